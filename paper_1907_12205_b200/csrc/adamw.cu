// One AdamW step over many tensors, with states in 32 bits or in 8.
//
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p - lr (wd p + (m / c1) / (sqrt(v / c2) + eps)),  c_i = 1 - b_i^step
//
// Bound by HBM: every buffer is read once and written once (fp32 weights and states: 28 bytes an entry; bf16 weights, fp32 masters and
// gradients, 8-bit states: 18).  The tensors' pointers travel as kernel parameters, so a step is one launch for each few hundred of them,
// with nothing to copy and nothing to set up, and a captured one keeps them.  A warp takes 4 blocks of 128 entries at a time, 4 entries a lane and
// block, so that a block's scale is one warp-wide reduction and every access of a warp is contiguous: 16 bytes a lane in fp32, and where a buffer is not aligned for
// that, single entries dealt round the lanes.
//
// 8 bits: m and sqrt(v) as e4m3 numbers with a power-of-two scale for each block.  Of v the root is kept, since its range is half as
// wide (v's would leave the form's 18 binary orders).  Rounding is random: added to the bits that the form drops, 16 random ones round up or down with
// the right mean; a sum of thousands of steps that each change an entry by less than its spacing keeps its mean that way.
#include <cmath>

#include "worker.cuh"

namespace detox {

namespace {

constexpr int kThreads = 256;
constexpr int kBlocks = 4;                       // blocks of 128 entries that a warp has in flight
constexpr int kUnit = kBlocks * kKeepBlock;

struct Tensor {
    void* P;
    const void* G;
    float* master;
    void* M;
    uint8_t* ME;
    void* V;
    uint8_t* VE;
    int64_t n;
    float weight_decay;
    uint32_t key;
    uint8_t p_dtype, g_dtype, vec;               // vec: every buffer is aligned for a lane's 4 entries
};
struct Numbers {
    float lr, beta1, beta2, rest1, rest2, eps, grad_scale;   // rest: 1 - beta
    float c1, root_c2;                           // 1 / (1 - beta1^step), 1 / sqrt(1 - beta2^step)
    float log_beta1, log_beta2;
    uint32_t seed, step;
    const float* lr_dev;
    const int64_t* step_dev;
};
// Units are numbered through the tensors of a launch; end[i]: the first one behind tensor i.
template <int CAP>
struct Table {
    int32_t count;
    int64_t end[CAP];
    Tensor of[CAP];
};
// Two sizes of launch: most of a launch's parameters are the table, and a small one's call is quicker.
constexpr int kFew = 32, kMany = 336;
static_assert(sizeof(Table<kMany>) + sizeof(Numbers) <= 32764, "kernel parameters");

__device__ __forceinline__ uint32_t mix(uint32_t x) {
    x ^= x >> 16;
    x *= 0x85ebca6bu;
    x ^= x >> 13;
    x *= 0xc2b2ae35u;
    return x ^ (x >> 16);
}

// 4 entries of a lane: contiguous ones (vec), or lane, lane + 32, ... of the block, where there are so many
template <typename T>
__device__ __forceinline__ void load4(const T* from, bool vec, int lane, int64_t left, float (&f)[4]) {
    if (vec) {
        if constexpr (sizeof(T) == 4) {
            const float4 x = ld_stream_f4(reinterpret_cast<const float*>(from) + 4 * lane);
            f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
        } else {
            const uint2 x = __ldcs(reinterpret_cast<const uint2*>(from + 4 * lane));
            const float2 a = unpack2<T>(x.x), b = unpack2<T>(x.y);
            f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = 32 * j + lane < left ? to_f32(from[32 * j + lane]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void store4(T* to, bool vec, int lane, int64_t left, const float (&f)[4]) {
    if (vec) {
        if constexpr (sizeof(T) == 4) st_stream_f4(reinterpret_cast<float*>(to) + 4 * lane, make_float4(f[0], f[1], f[2], f[3]));
        else __stcs(reinterpret_cast<uint2*>(to + 4 * lane), make_uint2(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3])));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (32 * j + lane < left) to[32 * j + lane] = from_f32<T>(f[j]);
    }
}
__device__ __forceinline__ void load4(const void* from, int dtype, int64_t at, bool vec, int lane, int64_t left, float (&f)[4]) {
    if (dtype == DETOX_DTYPE_FLOAT) load4(static_cast<const float*>(from) + at, vec, lane, left, f);
    else if (dtype == DETOX_DTYPE_HALF) load4(static_cast<const __half*>(from) + at, vec, lane, left, f);
    else load4(static_cast<const __nv_bfloat16*>(from) + at, vec, lane, left, f);
}
__device__ __forceinline__ void store4(void* to, int dtype, int64_t at, bool vec, int lane, int64_t left, const float (&f)[4]) {
    if (dtype == DETOX_DTYPE_FLOAT) store4(static_cast<float*>(to) + at, vec, lane, left, f);
    else if (dtype == DETOX_DTYPE_HALF) store4(static_cast<__half*>(to) + at, vec, lane, left, f);
    else store4(static_cast<__nv_bfloat16*>(to) + at, vec, lane, left, f);
}
// 4 bytes of a lane, as one word
__device__ __forceinline__ uint32_t load_bytes(const uint8_t* from, bool vec, int lane, int64_t left) {
    if (vec) return __ldcs(reinterpret_cast<const unsigned int*>(from) + lane);
    uint32_t q = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (32 * j + lane < left) q |= (uint32_t)from[32 * j + lane] << (8 * j);
    return q;
}
__device__ __forceinline__ void store_bytes(uint8_t* to, bool vec, int lane, int64_t left, uint32_t q) {
    if (vec) {
        __stcs(reinterpret_cast<unsigned int*>(to) + lane, q);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (32 * j + lane < left) to[32 * j + lane] = (uint8_t)(q >> (8 * j));
}

// The 8-bit form of a block, 4 entries a lane, rounded at random with `bits` (16 of them an entry).  POSITIVE: entries > 0 stay so.
// Inf and NaN become NaN and do not count for the scale.
template <bool POSITIVE>
__device__ __forceinline__ uint32_t keep_at_random(const float (&x)[4], const uint32_t (&bits)[4], uint32_t* q) {
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t a = __float_as_uint(x[j]) & 0x7fffffffu;
        if (a < 0x7f800000u && a > top) top = a;
    }
    const uint32_t e = keep_exponent(__uint_as_float(__reduce_max_sync(0xffffffffu, top)));
    const float inverse = keep_inverse(e);
    float r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float a = fabsf(x[j]) * inverse;           // at most 448: e4m3 keeps 3 of fp32's 23 bits behind the first
        const float lift = a < 0.015625f ? 0.015625f : 0.f;   // below 2^-6 the form's steps are 2^-9 wide, as they are from there to 2^-5
        const uint32_t b = (__float_as_uint(a + lift) + (bits[j] << 4)) & 0xfff00000u;
        float k = __uint_as_float(b) - lift;
        if (POSITIVE && a > 0.f && k == 0.f) k = 0.001953125f;
        r[j] = a <= 448.f ? copysignf(k, x[j]) : __int_as_float(0x7fc00000);
    }
    *q = keep4(r[0], r[1], r[2], r[3]);
    return e;
}

template <bool EIGHT, int CAP>
__global__ void __launch_bounds__(kThreads, 4) adamw_kernel(const __grid_constant__ Table<CAP> table, const __grid_constant__ Numbers number) {
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x % 32;
    float lr = number.lr, c1 = number.c1, root_c2 = number.root_c2;
    uint32_t step = number.step;
    if (number.lr_dev) lr = *number.lr_dev;
    if (number.step_dev) {
        const int64_t t = *number.step_dev;
        step = (uint32_t)t;
        const float count = t < 1 ? 1.f : (float)t;
        // 1 - b^t = -(e^(t log b) - 1), without the difference's loss of bits (b = 0: log b = -Inf)
        c1 = 1.f / -expm1f(count * number.log_beta1);
        root_c2 = sqrtf(1.f / -expm1f(count * number.log_beta2));
    }
    const uint32_t start = EIGHT ? mix(number.seed + 0x9e3779b9u * step) : 0u;
    const int64_t units = table.end[table.count - 1], stride = (int64_t)gridDim.x * (kThreads / 32);
    int which = 0;
    for (int64_t unit = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32; unit < units; unit += stride) {
        if (unit >= table.end[which]) {
            // the first tensor that ends behind this unit
            int lo = which + 1, hi = table.count - 1;
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (unit < table.end[mid]) hi = mid;
                else lo = mid + 1;
            }
            which = lo;
        }
        const Tensor& t = table.of[which];
        const int64_t at = (unit - (which ? table.end[which - 1] : 0)) * kUnit;
        float g[kBlocks][4], p[kBlocks][4], m[kBlocks][4], v[kBlocks][4];
        uint32_t mq[kBlocks], vq[kBlocks];
        float ms[kBlocks], vs[kBlocks];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const int64_t i = at + b * kKeepBlock, left = t.n - i;
            if (left <= 0) continue;
            const bool vec = t.vec && left >= kKeepBlock;
            load4(t.G, t.g_dtype, i, vec, lane, left, g[b]);
            if (t.master) load4(t.master + i, vec, lane, left, p[b]);
            else load4(t.P, t.p_dtype, i, vec, lane, left, p[b]);
            if constexpr (EIGHT) {
                mq[b] = load_bytes(static_cast<const uint8_t*>(t.M) + i, vec, lane, left);
                vq[b] = load_bytes(static_cast<const uint8_t*>(t.V) + i, vec, lane, left);
                ms[b] = keep_scale_of_byte(t.ME[i / kKeepBlock]);
                vs[b] = keep_scale_of_byte(t.VE[i / kKeepBlock]);
            } else {
                load4(static_cast<const float*>(t.M) + i, vec, lane, left, m[b]);
                load4(static_cast<const float*>(t.V) + i, vec, lane, left, v[b]);
            }
        }
        const uint32_t seed = EIGHT ? mix(start + t.key) : 0u;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const int64_t i = at + b * kKeepBlock, left = t.n - i;
            if (left <= 0) continue;
            const bool vec = t.vec && left >= kKeepBlock;
            if constexpr (EIGHT) {
                taken4(mq[b], m[b]);
                taken4(vq[b], v[b]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    m[b][j] *= ms[b];
                    const float root = v[b][j] * vs[b];
                    v[b][j] = root * root;
                }
            }
            float root[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x = g[b][j] * number.grad_scale;
                m[b][j] = fmaf(number.beta1, m[b][j], number.rest1 * x);
                v[b][j] = fmaf(number.beta2, v[b][j], number.rest2 * (x * x));
                root[j] = sqrtf(v[b][j]);
                const float direction = __fdividef(m[b][j] * c1, fmaf(root[j], root_c2, number.eps));
                p[b][j] = fmaf(-lr, fmaf(t.weight_decay, p[b][j], direction), p[b][j]);
            }
            if (t.master) store4(t.master + i, vec, lane, left, p[b]);
            store4(t.P, t.p_dtype, i, vec, lane, left, p[b]);
            if constexpr (EIGHT) {
                uint32_t rm[4], rv[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t h = mix(seed ^ (uint32_t)(i + (vec ? 4 * lane + j : 32 * j + lane)));
                    rm[j] = h & 0xffffu;
                    rv[j] = h >> 16;
                }
                uint32_t q;
                const uint32_t me = keep_at_random<false>(m[b], rm, &q);
                store_bytes(static_cast<uint8_t*>(t.M) + i, vec, lane, left, q);
                const uint32_t ve = keep_at_random<true>(root, rv, &q);
                store_bytes(static_cast<uint8_t*>(t.V) + i, vec, lane, left, q);
                if (lane == 0) {
                    t.ME[i / kKeepBlock] = (uint8_t)me;
                    t.VE[i / kKeepBlock] = (uint8_t)ve;
                }
            } else {
                store4(static_cast<float*>(t.M) + i, vec, lane, left, m[b]);
                store4(static_cast<float*>(t.V) + i, vec, lane, left, v[b]);
            }
        }
    }
}

bool aligned_for(const void* p, int size) { return aligned_to(p, (size_t)size * 4); }

template <bool EIGHT, int CAP>
detox_status step_of(const Numbers& number, const detox_adamw_tensor* from, const detox_adamw_tensor* end, const detox_adamw_tensor** next,
                     cudaStream_t s) {
    static thread_local Table<CAP> table;
    int64_t units = 0;
    int n = 0;
    for (; from != end && n < CAP; ++from) {
        if (from->n == 0) continue;
        const int ps = from->p_dtype == DETOX_DTYPE_FLOAT ? 4 : 2, gs = from->g_dtype == DETOX_DTYPE_FLOAT ? 4 : 2, ss = EIGHT ? 1 : 4;
        Tensor& t = table.of[n];
        t.P = from->P; t.G = from->G; t.master = from->master;
        t.M = from->M; t.ME = from->ME; t.V = from->V; t.VE = from->VE;
        t.n = from->n;
        t.weight_decay = from->weight_decay;
        t.key = from->key;
        t.p_dtype = (uint8_t)from->p_dtype;
        t.g_dtype = (uint8_t)from->g_dtype;
        t.vec = aligned_for(t.P, ps) && aligned_for(t.G, gs) && aligned_for(t.master, 4) && aligned_for(t.M, ss) && aligned_for(t.V, ss);
        units += ceil_div(t.n, (int64_t)kUnit);
        table.end[n++] = units;
    }
    *next = from;
    if (n == 0) return DETOX_OK;
    table.count = n;
    const int64_t need = ceil_div(units, (int64_t)(kThreads / 32)), most = (int64_t)kSMs * 4;
    return launch_chained(adamw_kernel<EIGHT, CAP>, (unsigned)(need < most ? need : most), kThreads, 0, 1, s, table, number);
}

}  // namespace

detox_status launch_adamw(const detox_adamw_desc& d, const detox_adamw_tensor* tensors, int64_t count, cudaStream_t s) {
    Numbers number = {};
    number.lr = (float)d.lr;
    number.beta1 = (float)d.beta1; number.beta2 = (float)d.beta2;
    number.rest1 = (float)(1.0 - d.beta1); number.rest2 = (float)(1.0 - d.beta2);
    number.eps = (float)d.eps;
    number.grad_scale = d.grad_scale;
    number.log_beta1 = (float)log(d.beta1); number.log_beta2 = (float)log(d.beta2);
    number.c1 = (float)(1.0 / (1.0 - pow(d.beta1, (double)d.step)));
    number.root_c2 = (float)sqrt(1.0 / (1.0 - pow(d.beta2, (double)d.step)));
    number.seed = d.seed;
    number.step = (uint32_t)d.step;
    number.lr_dev = d.lr_dev;
    number.step_dev = d.step_dev;
    const detox_adamw_tensor* end = tensors + count;
    while (tensors != end) {
        const bool few = end - tensors <= kFew;
        detox_status st;
        if (d.bits == 8) st = few ? step_of<true, kFew>(number, tensors, end, &tensors, s) : step_of<true, kMany>(number, tensors, end, &tensors, s);
        else st = few ? step_of<false, kFew>(number, tensors, end, &tensors, s) : step_of<false, kMany>(number, tensors, end, &tensors, s);
        if (st != DETOX_OK) return st;
    }
    return DETOX_OK;
}

}  // namespace detox
