// Python entry of the worker-side operators: checks the tensors, makes the outputs that the caller did not pass, and calls
// the C functions of include/detox.h.
//
// A worker's small steps are bound by what a call costs on the host, and most of that is not the launch (2.3 us): from
// Python, each output tensor took 2 us and each tensor's checks 0.6.  Here they take a fraction of that: a norm of one row with
// all its outputs 20.8 -> 8.8 us, a step of 500 tokens 63 -> 39 us, and with outputs made past the dispatcher 7.7 and 38 today.
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "detox.h"

namespace {

PyObject* g_error = nullptr;   // the package's DetoxError(code, what)

// Thrown once a Python exception has been set.
struct Raised {};

template <typename... A>
[[noreturn]] void raise(PyObject* type, const char* format, A... args) {
    PyErr_Format(type, format, args...);
    throw Raised{};
}

void check(detox_status st, const char* what) {
    if (st == DETOX_OK) return;
    PyObject* e = g_error ? PyObject_CallFunction(g_error, "is", (int)st, what) : nullptr;
    if (e) {
        PyErr_SetObject(g_error, e);
        Py_DECREF(e);
    } else if (!PyErr_Occurred()) {
        PyErr_Format(PyExc_RuntimeError, "%s: status %d", what, (int)st);
    }
    throw Raised{};
}

constexpr int64_t kBlock = DETOX_KEEP_BLOCK;
constexpr at::ScalarType kValues = at::kFloat8_e4m3fn, kScales = at::kFloat8_e8m0fnu;
int64_t blocks(int64_t cols) { return (cols + kBlock - 1) / kBlock; }

int code_of(at::ScalarType t, const char* what) {
    if (t == at::kFloat) return DETOX_DTYPE_FLOAT;
    if (t == at::kHalf) return DETOX_DTYPE_HALF;
    if (t == at::kBFloat16) return DETOX_DTYPE_BFLOAT;
    raise(PyExc_TypeError, "%s: expected float32, float16 or bfloat16, got %s", what, c10::toString(t));
}
at::ScalarType type_of(int code) {
    return code == DETOX_DTYPE_FLOAT ? at::kFloat : code == DETOX_DTYPE_HALF ? at::kHalf : at::kBFloat16;
}

// None or a tensor.  The operators record no graph (their backward passes are functions of their own), so an input that asks for one is
// refused rather than cut off in silence.
const at::Tensor* optional_tensor(PyObject* o, const char* what) {
    if (o == Py_None) return nullptr;
    if (!THPVariable_Check(o)) raise(PyExc_TypeError, "%s: expected a tensor", what);
    const at::Tensor& t = THPVariable_Unpack(o);
    if (t.requires_grad() && at::GradMode::is_enabled())
        raise(PyExc_RuntimeError, "%s requires grad, but no graph is recorded here: call under torch.no_grad(), or pass a detached tensor", what);
    return &t;
}
const at::Tensor& tensor(PyObject* o, const char* what) {
    const at::Tensor* t = optional_tensor(o, what);
    if (!t) raise(PyExc_TypeError, "%s: expected a tensor", what);
    return *t;
}

// The device of the present call, -1 until its first tensor has been looked at: all tensors of a call lie on one device, which is
// where it is launched, whatever the current device is.
thread_local c10::DeviceIndex g_device = -1;
void on_device(const at::Tensor& t, const char* what) {
    if (!t.is_cuda()) raise(PyExc_TypeError, "%s: expected a CUDA tensor", what);
    const c10::DeviceIndex d = t.device().index();
    if (g_device < 0) g_device = d;
    if (d != g_device) raise(PyExc_ValueError, "%s: on cuda:%d, the tensors before it on cuda:%d", what, (int)d, (int)g_device);
}

// A matrix with contiguous rows.
struct Rows {
    at::Tensor t;
    void* p = nullptr;
    int64_t ld = 0, rows = 0, cols = 0;
};
Rows rows_of(const at::Tensor& t, const char* what) {
    if (!t.is_cuda() || t.dim() != 2) raise(PyExc_TypeError, "%s: expected a 2-D CUDA tensor", what);
    on_device(t, what);
    Rows r{t, t.data_ptr(), t.stride(0), t.size(0), t.size(1)};
    if (t.stride(1) != 1 && r.cols > 1) raise(PyExc_ValueError, "%s: rows must be contiguous", what);
    if (r.ld < r.cols) {
        if (r.rows > 1) raise(PyExc_ValueError, "%s: rows overlap", what);
        r.ld = r.cols;
    }
    return r;
}
Rows rows_of(const at::Tensor& t, const char* what, at::ScalarType type) {
    const Rows r = rows_of(t, what);
    if (t.scalar_type() != type) raise(PyExc_TypeError, "%s: expected %s, got %s", what, c10::toString(type), c10::toString(t.scalar_type()));
    return r;
}
Rows rows_of(const at::Tensor& t, const char* what, at::ScalarType type, int64_t rows, int64_t cols) {
    const Rows r = rows_of(t, what, type);
    if (r.rows != rows || r.cols != cols)
        raise(PyExc_ValueError, "%s: expected shape (%lld, %lld), got (%lld, %lld)", what, (long long)rows, (long long)cols,
              (long long)r.rows, (long long)r.cols);
    return r;
}
void* vector_of(const at::Tensor& t, const char* what, at::ScalarType type, int64_t n) {
    if (!t.is_cuda() || t.scalar_type() != type || t.dim() != 1 || t.size(0) != n || !t.is_contiguous())
        raise(PyExc_TypeError, "%s: expected a contiguous CUDA vector of %lld entries of %s", what, (long long)n, c10::toString(type));
    on_device(t, what);
    return t.data_ptr();
}

// A new tensor on `like`'s device, without a way through the dispatcher for each.
at::Tensor new_tensor(at::IntArrayRef sizes, at::IntArrayRef strides, at::ScalarType type, const at::Tensor& like) {
    return at::detail::empty_strided_cuda(sizes, strides, type, like.device());
}

// A new matrix; rows a multiple of 16 bytes apart, so that the kernels can use 16-byte accesses.
Rows new_rows(int64_t rows, int64_t cols, at::ScalarType type, const at::Tensor& like) {
    const int64_t n = 16 / (int64_t)c10::elementSize(type), ld = (cols + n - 1) / n * n;
    at::Tensor t = new_tensor({rows, cols}, {ld, 1}, type, like);
    void* p = t.data_ptr();
    return Rows{std::move(t), p, ld, rows, cols};
}
at::Tensor new_vector(int64_t n, at::ScalarType type, const at::Tensor& like) { return new_tensor({n}, {1}, type, like); }

// Values and scales of the 8-bit form.
struct Pair {
    Rows q, e;
};
Pair new_pair(int64_t rows, int64_t cols, const at::Tensor& like) {
    at::Tensor e = new_tensor({rows, blocks(cols)}, {blocks(cols), 1}, kScales, like);
    void* p = e.data_ptr();
    return Pair{new_rows(rows, cols, kValues, like), Rows{std::move(e), p, blocks(cols), rows, blocks(cols)}};
}
Pair pair_of(const at::Tensor& q, const at::Tensor& e, const char* what, const char* scales) {
    Pair p{rows_of(q, what, kValues), {}};
    p.e = rows_of(e, scales, kScales, p.q.rows, blocks(p.q.cols));
    return p;
}
uint8_t* bytes(const Rows& r) { return static_cast<uint8_t*>(r.p); }

// The stream of a call: the caller's, or the current one.  While this lives it is the current stream, so that the outputs and the
// workspace are made for it (and the tensors' device the current one): a workspace that came from another stream's pool could be handed out again there, at the call's
// return, while this stream's kernels still use it, and an output might still be in use there.
struct OnStream {
    cudaStream_t s;
    c10::cuda::OptionalCUDAStreamGuard guard;
    OnStream(PyObject* given, const at::Tensor& like) {
        const c10::DeviceIndex device = like.device().index();
        const c10::cuda::CUDAStream current = c10::cuda::getCurrentCUDAStream(device);
        s = current.stream();
        if (device != c10::cuda::current_device()) guard.reset_stream(current);
        if (given == Py_None) return;
        void* const handle = PyLong_AsVoidPtr(given);
        if (PyErr_Occurred()) throw Raised{};
        if (static_cast<cudaStream_t>(handle) == s) return;
        s = static_cast<cudaStream_t>(handle);
        guard.reset_stream(c10::cuda::getStreamFromExternal(s, device));
    }
};
int64_t integer(PyObject* o) {
    const int64_t v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
}
// one of an enumeration's codes (what does not fit its type is none of them)
int32_t code(PyObject* o) {
    const int64_t v = integer(o);
    return v < INT32_MIN || v > INT32_MAX ? -1 : (int32_t)v;
}
bool truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Raised{};
    return v != 0;
}

// The caller's workspace, or a new one.
struct Workspace {
    at::Tensor t;
    void* p;
    size_t bytes;
};
Workspace workspace(PyObject* given, size_t need, const at::Tensor& like) {
    if (const at::Tensor* t = optional_tensor(given, "ws")) {
        on_device(*t, "ws");
        if (!t->is_contiguous()) raise(PyExc_ValueError, "ws: expected a contiguous tensor");
        return Workspace{*t, t->data_ptr(), (size_t)t->nbytes()};
    }
    at::Tensor t = new_vector((int64_t)(need < 256 ? 256 : need), at::kByte, like);
    return Workspace{t, t.data_ptr(), (size_t)t.nbytes()};
}

PyObject* wrap(const at::Tensor& t) {
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}
template <typename... T>
PyObject* wrap_all(const T&... t) {
    PyObject* out = PyTuple_New(sizeof...(T));
    if (!out) throw Raised{};
    Py_ssize_t i = 0;
    (PyTuple_SET_ITEM(out, i++, wrap(t)), ...);
    return out;
}

// Runs a function's body; C++ exceptions (torch's own, out of memory) become Python's.
template <typename F>
PyObject* guarded(const char* name, Py_ssize_t n, Py_ssize_t want, F body) {
    HANDLE_TH_ERRORS
    g_device = -1;
    if (n != want) return PyErr_Format(PyExc_TypeError, "%s: %zd arguments, got %zd", name, want, n);
    try {
        return body();
    } catch (const Raised&) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// (x, q, e, stream)
PyObject* checkpoint_pack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("checkpoint_pack", n, 4, [&] {
        const Rows x = rows_of(tensor(a[0], "x"), "x");
        const int code = code_of(x.t.scalar_type(), "x");
        const OnStream on(a[3], x.t);
        Pair to;
        if (const at::Tensor* q = optional_tensor(a[1], "out")) {
            to = pair_of(*q, tensor(a[2], "out scales"), "out", "out scales");
            if (to.q.rows != x.rows || to.q.cols != x.cols) raise(PyExc_ValueError, "out: not of x's shape");
        } else {
            to = new_pair(x.rows, x.cols, x.t);
        }
        check(detox_checkpoint_pack(code, x.p, x.ld, x.rows, x.cols, bytes(to.q), to.q.ld, bytes(to.e), to.e.ld, on.s),
              "detox_checkpoint_pack");
        return wrap_all(to.q.t, to.e.t);
    });
}

// (q, e, dtype code, out, stream)
PyObject* checkpoint_unpack(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("checkpoint_unpack", n, 5, [&] {
        const Pair from = pair_of(tensor(a[0], "q"), tensor(a[1], "e"), "q", "e");
        const OnStream on(a[4], from.q.t);
        Rows x;
        if (const at::Tensor* t = optional_tensor(a[3], "out")) x = rows_of(*t, "out", t->scalar_type(), from.q.rows, from.q.cols);
        else x = new_rows(from.q.rows, from.q.cols, type_of((int)integer(a[2])), from.q.t);
        check(detox_checkpoint_unpack(code_of(x.t.scalar_type(), "out"), bytes(from.q), from.q.ld, bytes(from.e), from.e.ld, x.rows,
                                      x.cols, x.p, x.ld, on.s),
              "detox_checkpoint_unpack");
        return wrap(x.t);
    });
}

// (x, w, residual, eps, want_y, want_q, sum_out, stream) -> (sum, y, q, e, rstd)
PyObject* rmsnorm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("rmsnorm", n, 8, [&] {
        const Rows x = rows_of(tensor(a[0], "x"), "x");
        const at::ScalarType type = x.t.scalar_type();
        const int code = code_of(type, "x");
        void* w = vector_of(tensor(a[1], "w"), "w", type, x.cols);
        const double eps = PyFloat_AsDouble(a[3]);
        if (PyErr_Occurred()) throw Raised{};
        const OnStream on(a[7], x.t);
        Rows r, s, y;
        Pair q;
        if (const at::Tensor* t = optional_tensor(a[2], "residual")) {
            r = rows_of(*t, "residual", type, x.rows, x.cols);
            if (const at::Tensor* o = optional_tensor(a[6], "sum_out")) s = rows_of(*o, "sum_out", type, x.rows, x.cols);
            else s = new_rows(x.rows, x.cols, type, x.t);
        } else if (a[6] != Py_None) {
            raise(PyExc_ValueError, "sum_out: there is no residual to add");
        }
        if (truth(a[4])) y = new_rows(x.rows, x.cols, type, x.t);
        if (truth(a[5])) q = new_pair(x.rows, x.cols, x.t);
        const at::Tensor rstd = new_vector(x.rows, at::kFloat, x.t);
        check(detox_rmsnorm(code, x.p, x.ld, r.p, r.ld, w, x.rows, x.cols, (float)eps, s.p, s.ld, y.p, y.ld, bytes(q.q), q.q.ld,
                            bytes(q.e), q.e.ld, static_cast<float*>(rstd.data_ptr()), on.s),
              "detox_rmsnorm");
        return wrap_all(s.t, y.t, q.q.t, q.e.t, rstd);
    });
}

// (dy, s, w, rstd, ds, dx, dw, ws, stream) -> (dx, dw)
PyObject* rmsnorm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("rmsnorm_backward", n, 9, [&] {
        const Rows s = rows_of(tensor(a[1], "s"), "s");
        const at::ScalarType type = s.t.scalar_type();
        const int code = code_of(type, "s");
        const Rows dy = rows_of(tensor(a[0], "dy"), "dy", type, s.rows, s.cols);
        void* w = vector_of(tensor(a[2], "w"), "w", type, s.cols);
        void* rstd = vector_of(tensor(a[3], "rstd"), "rstd", at::kFloat, s.rows);
        const OnStream on(a[8], s.t);
        Rows ds, dx;
        if (const at::Tensor* t = optional_tensor(a[4], "ds")) ds = rows_of(*t, "ds", type, s.rows, s.cols);
        if (const at::Tensor* t = optional_tensor(a[5], "dx")) dx = rows_of(*t, "dx", type, s.rows, s.cols);
        else dx = new_rows(s.rows, s.cols, type, s.t);
        const at::Tensor* given = optional_tensor(a[6], "dw");
        const at::Tensor dw = given ? *given : new_vector(s.cols, at::kFloat, s.t);
        void* dwp = vector_of(dw, "dw", at::kFloat, s.cols);
        const Workspace ws = workspace(a[7], detox_rmsnorm_backward_workspace_bytes(s.rows, s.cols), s.t);
        check(detox_rmsnorm_backward(code, dy.p, dy.ld, ds.p, ds.ld, s.p, s.ld, w, static_cast<const float*>(rstd), s.rows, s.cols, dx.p,
                                     dx.ld, static_cast<float*>(dwp), ws.p, ws.bytes, on.s),
              "detox_rmsnorm_backward");
        return wrap_all(dx.t, dw);
    });
}

// The descriptor of the gated projections from (x, xe, wg, wu, act, kept q, kept e); x is a matrix, or with xe its 8-bit form.
struct Gated {
    detox_gated_desc d{};
    at::Tensor like;
    at::ScalarType type;
};
Gated gated_desc(PyObject* const* a) {
    Gated g;
    const Rows wg = rows_of(tensor(a[2], "wg"), "wg");
    g.like = wg.t;
    g.type = wg.t.scalar_type();
    const Rows wu = rows_of(tensor(a[3], "wu"), "wu", g.type, wg.rows, wg.cols);
    detox_gated_desc& d = g.d;
    d.dtype = code_of(g.type, "wg");
    d.act = code(a[4]);
    d.hidden = wg.rows;
    d.in_dim = wg.cols;
    d.Wg = wg.p; d.ldwg = wg.ld;
    d.Wu = wu.p; d.ldwu = wu.ld;
    int64_t cols;
    if (const at::Tensor* e = optional_tensor(a[1], "x scales")) {
        const Pair x = pair_of(tensor(a[0], "x"), *e, "x", "x scales");
        d.XQ = bytes(x.q); d.ldxq = x.q.ld;
        d.XE = bytes(x.e); d.ldxe = x.e.ld;
        d.tokens = x.q.rows;
        cols = x.q.cols;
    } else {
        const Rows x = rows_of(tensor(a[0], "x"), "x", g.type);
        d.X = x.p; d.ldx = x.ld;
        d.tokens = x.rows;
        cols = x.cols;
    }
    if (cols != d.in_dim) raise(PyExc_ValueError, "x has %lld columns, the weights %lld", (long long)cols, (long long)d.in_dim);
    if (const at::Tensor* q = optional_tensor(a[5], "kept")) {
        const at::Tensor& e = tensor(a[6], "kept scales");
        on_device(*q, "kept");
        on_device(e, "kept scales");
        if (q->scalar_type() != kValues || e.scalar_type() != kScales)
            raise(PyExc_TypeError, "kept: expected float8_e4m3fn values and float8_e8m0fnu scales on the GPU");
        const int64_t nb = blocks(d.hidden);
        if (q->dim() != 3 || q->size(0) != 2 || q->size(1) != d.tokens || q->size(2) != d.hidden || e.dim() != 3 || e.size(0) != 2 ||
            e.size(1) != d.tokens || e.size(2) != nb)
            raise(PyExc_ValueError, "kept: expected values [2, %lld, %lld] and their scales", (long long)d.tokens, (long long)d.hidden);
        if ((q->stride(2) != 1 && d.hidden > 1) || (e.stride(2) != 1 && nb > 1)) raise(PyExc_ValueError, "kept: rows must be contiguous");
        d.GQ = static_cast<uint8_t*>(q->data_ptr());
        d.GE = static_cast<uint8_t*>(e.data_ptr());
        d.UQ = d.GQ + q->stride(0);
        d.UE = d.GE + e.stride(0);
        d.ldq = q->stride(1);
        d.lde = e.stride(1);
    }
    return g;
}

// (x, xe, wg, wu, act, kept q, kept e, backward) -> bytes
PyObject* gated_workspace_bytes(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("gated_workspace_bytes", n, 8, [&] {
        const Gated g = gated_desc(a);
        return PyLong_FromSize_t(truth(a[7]) ? detox_gated_backward_workspace_bytes(&g.d) : detox_gated_workspace_bytes(&g.d));
    });
}

// (x, xe, wg, wu, act, None, None, keep, h, ws, stream) -> (h, kept q, kept e)
PyObject* gated(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("gated", n, 11, [&] {
        Gated g = gated_desc(a);
        detox_gated_desc& d = g.d;
        const OnStream on(a[10], g.like);
        at::Tensor q, e;
        if (truth(a[7])) {
            const int64_t ld = (d.hidden + 15) / 16 * 16, nb = blocks(d.hidden);
            q = new_tensor({2, d.tokens, d.hidden}, {d.tokens * ld, ld, 1}, kValues, g.like);
            e = new_tensor({2, d.tokens, nb}, {d.tokens * nb, nb, 1}, kScales, g.like);
            d.GQ = static_cast<uint8_t*>(q.data_ptr());
            d.GE = static_cast<uint8_t*>(e.data_ptr());
            d.UQ = d.GQ + d.tokens * ld;
            d.UE = d.GE + d.tokens * nb;
            d.ldq = ld;
            d.lde = nb;
        }
        Rows h;
        if (const at::Tensor* t = optional_tensor(a[8], "h")) h = rows_of(*t, "h", g.type, d.tokens, d.hidden);
        else h = new_rows(d.tokens, d.hidden, g.type, g.like);
        const Workspace ws = workspace(a[9], detox_gated_workspace_bytes(&d), g.like);
        check(detox_gated(&d, h.p, h.ld, ws.p, ws.bytes, on.s), "detox_gated");
        return wrap_all(h.t, q, e);
    });
}

// (x, xe, wg, wu, act, kept q, kept e, dh, dx, dwg, dwu, dw dtype code or -1, ws, stream) -> (dx, dwg, dwu)
PyObject* gated_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("gated_backward", n, 14, [&] {
        const Gated g = gated_desc(a);
        const detox_gated_desc& d = g.d;
        const Rows dh = rows_of(tensor(a[7], "dh"), "dh", g.type, d.tokens, d.hidden);
        const OnStream on(a[13], g.like);
        Rows dx, dwg, dwu;
        if (const at::Tensor* t = optional_tensor(a[8], "dx")) dx = rows_of(*t, "dx", g.type, d.tokens, d.in_dim);
        else dx = new_rows(d.tokens, d.in_dim, g.type, g.like);
        const int64_t code = integer(a[11]);
        const at::Tensor *tg = optional_tensor(a[9], "dwg"), *tu = optional_tensor(a[10], "dwu");
        if ((tg == nullptr) != (tu == nullptr)) raise(PyExc_ValueError, "give both weight gradients or none");
        if (tg) {
            dwg = rows_of(*tg, "dwg", code >= 0 ? type_of((int)code) : tg->scalar_type(), d.hidden, d.in_dim);
            dwu = rows_of(*tu, "dwu", tg->scalar_type(), d.hidden, d.in_dim);
            if (dwg.ld != dwu.ld) raise(PyExc_ValueError, "dwg and dwu must have the same stride");
        } else {
            const at::ScalarType type = code >= 0 ? type_of((int)code) : g.type;
            dwg = new_rows(d.hidden, d.in_dim, type, g.like);
            dwu = new_rows(d.hidden, d.in_dim, type, g.like);
        }
        const Workspace ws = workspace(a[12], detox_gated_backward_workspace_bytes(&d), g.like);
        check(detox_gated_backward(&d, dh.p, dh.ld, dx.p, dx.ld, dwg.p, dwu.p, dwg.ld, code_of(dwg.t.scalar_type(), "dwg"), ws.p, ws.bytes,
                                   on.s),
              "detox_gated_backward");
        return wrap_all(dx.t, dwg.t, dwu.t);
    });
}

PyObject* set_error(PyObject*, PyObject* type) {
    Py_INCREF(type);
    Py_XDECREF(g_error);
    g_error = type;
    Py_RETURN_NONE;
}

#define DETOX_METHOD(name) \
    { #name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr }
PyMethodDef methods[] = {
    DETOX_METHOD(checkpoint_pack), DETOX_METHOD(checkpoint_unpack), DETOX_METHOD(rmsnorm), DETOX_METHOD(rmsnorm_backward),
    DETOX_METHOD(gated_workspace_bytes), DETOX_METHOD(gated), DETOX_METHOD(gated_backward),
    {"set_error", set_error, METH_O, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_worker", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__worker() { return PyModule_Create(&module); }
