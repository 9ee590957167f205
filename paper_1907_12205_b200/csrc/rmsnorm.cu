// Root-mean-square norm with the residual's addition, and its backward pass.
//
// Forward:   s = x + r;  rstd = 1 / sqrt(mean(s^2) + eps);  y = s rstd w, as it is and / or in the 8-bit form.
// Backward:  with hat = s rstd:  dx = dS + rstd (w dy - hat mean(w dy hat));  dw = sum over rows of dy hat.
//
// Both are bound by HBM, so a row is read once and stays in registers: TPR threads hold it, EPT entries each, in 16-byte
// pieces dealt round the threads (piece t, t + TPR, ...).  With the 8-bit output a block of 128 columns then lies in 16
// neighbouring lanes (fp32: 32), which agree on its largest entry by shuffles.  Up to 512 columns a warp takes a row
// and no barrier is needed; above that a CTA does.  The grid is persistent: the next row's pieces are asked for before the
// present row's sum is formed, so that memory stays busy through the reductions.
//
// dw adds in a fixed order: a CTA takes every gridDim-th row and adds in registers, leaves one row of partial sums, and a
// second kernel adds those column by column.
#include "worker.cuh"

namespace detox {

namespace {

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// Sum over the TPR threads of a row (the same value in all of them; fixed order).  TPR > 32: the whole CTA; `turn`
// alternates between two halves of `sm`, so that one barrier a sum is enough.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* sm, int turn) {
    v = warp_sum(v);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        float* at = sm + (turn & 1) * W;
        if ((threadIdx.x & 31) == 0) at[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += at[i];
    }
    return v;
}

// 1 / sqrt(x) to about half a unit: rsqrtf is off by up to two, which moved a whole row's 8-bit entries over their rounding
// boundaries more often than the rest of the arithmetic; one Newton step, its residual 1 - x r^2 without a rounding that counts.
__device__ __forceinline__ float inverse_root(float x) {
    const float r = rsqrtf(x);
    if (!(r > 0.f && r < 3.402823466e38f)) return r;
    const float h = x * r, l = fmaf(x, r, -h);
    return fmaf(0.5f * r, fmaf(-l, r, fmaf(-h, r, 1.f)), r);
}

template <int TPR> constexpr int kBlockOf = TPR < 128 ? 256 : TPR;   // threads of a CTA
// Persistent CTAs on an SM: as many as the registers of a row's entries allow (64 or 128 a thread), with the next row waiting in
// registers too.  CTAs of 1024 threads with more than 8 entries each have no registers for that.
template <int TPR, int EPT> constexpr int kForwardCtas = 1024 / kBlockOf<TPR>;
template <int TPR, int EPT> constexpr int kBackwardCtas = TPR == 1024 ? 1 : (EPT == 8 ? 1024 : 512) / kBlockOf<TPR>;
template <int TPR, int EPT> constexpr bool kAhead = TPR < 1024 || EPT == 8;

struct NormOut {
    void* S; int64_t lds;
    void* Y; int64_t ldy;
    uint8_t* Q; int64_t ldq;
    uint8_t* E; int64_t lde;
    float* rstd;
    bool s_vec, y_vec, q_vec;   // 16-byte (8-bit form: 8-byte) stores
};
struct NormIn {
    const void* X; int64_t ldx;
    const void* R; int64_t ldr;
    const void* w;
    Span x, r, weight;
};

// X, R and S may be the same buffer: a row is in registers before any of it is written.
template <typename T, int TPR, int EPT, bool ANY>
__global__ void __launch_bounds__(kBlockOf<TPR>, (kForwardCtas<TPR, EPT>))
rmsnorm_kernel(const __grid_constant__ NormIn in, int64_t rows, int cols, float eps, const __grid_constant__ NormOut o) {
    constexpr int N = Piece<T>::N, P = EPT / N, RPB = kBlockOf<TPR> / TPR;
    __shared__ float sm[TPR > 32 ? 2 * (TPR / 32) : 1];
    pdl_trigger();
    pdl_wait();
    const int t = threadIdx.x % TPR;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    if (row >= rows) return;                   // (TPR = 32: whole warps; else never: a CTA has a row)
    uint4 weight[P], x[P], r[P];
    const T *w = static_cast<const T*>(in.w), *from_x = static_cast<const T*>(in.X) + row * in.ldx;
    const T* from_r = in.R ? static_cast<const T*>(in.R) + row * in.ldr : nullptr;
    auto fetch = [&] {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int c = (t + i * TPR) * N;
            x[i] = load_piece<ANY>(from_x, c, cols, in.x);
            if (from_r) r[i] = load_piece<ANY>(from_r, c, cols, in.r);
        }
        from_x += stride * in.ldx;
        if (from_r) from_r += stride * in.ldr;
    };
#pragma unroll
    for (int i = 0; i < P; ++i)
        if ((kAhead<TPR, EPT>)) weight[i] = load_piece<ANY>(w, (t + i * TPR) * N, cols, in.weight);
    if ((kAhead<TPR, EPT>)) fetch();
    for (int turn = 0;; ++turn) {
        if (!(kAhead<TPR, EPT>)) fetch();
        uint64_t v[P][N / 2];
        uint64_t sum2 = 0ull;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            Piece<T>::split(x[i], v[i]);
            if (from_r) {
                uint64_t f[N / 2];
                Piece<T>::split(r[i], f);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) v[i][j] = add2(v[i][j], f[j]);
            }
#pragma unroll
            for (int j = 0; j < N / 2; ++j) sum2 = fma2(v[i][j], v[i][j], sum2);
        }
        const int64_t next = row + stride;
        if ((kAhead<TPR, EPT>) && next < rows) fetch();
        const float sum = row_sum<TPR>(pair_lo(sum2) + pair_hi(sum2), sm, turn);
        const float rstd = inverse_root(sum / (float)cols + eps);
        const uint64_t rstd2 = pair_of(rstd, rstd);
        if (o.rstd && t == 0) o.rstd[row] = rstd;
        if (o.S) {
            T* s = static_cast<T*>(o.S) + row * o.lds;
#pragma unroll
            for (int i = 0; i < P; ++i) store_piece(s, (t + i * TPR) * N, cols, !ANY || o.s_vec, v[i]);
        }
        if (o.Y || o.Q) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                // (beyond the row's end: zeros, or NaN from 0 * Inf, which a block's largest entry passes over)
                const int c = (t + i * TPR) * N;
                uint64_t f[N / 2];
                Piece<T>::split((kAhead<TPR, EPT>) ? weight[i] : load_piece<ANY>(w, c, cols, in.weight), f);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) v[i][j] = mul2(mul2(v[i][j], rstd2), f[j]);
                if (o.Y) store_piece(static_cast<T*>(o.Y) + row * o.ldy, c, cols, !ANY || o.y_vec, v[i]);
                if (o.Q) {
                    constexpr int kLanes = kKeepBlock / N;   // 16, or 32 in fp32: the lanes of a block lie side by side
                    uint32_t q[N / 4];
                    const uint32_t e = keep_pairs<N / 2, kLanes>(v[i], q);
                    uint8_t* to = o.Q + row * o.ldq + c;
                    if ((!ANY || o.q_vec) && c + N <= cols) {
                        if constexpr (N == 8) __stcs(reinterpret_cast<uint2*>(to), make_uint2(q[0], q[1]));
                        else __stcs(reinterpret_cast<unsigned int*>(to), q[0]);
                    } else {
#pragma unroll
                        for (int j = 0; j < N; ++j)
                            if (c + j < cols) to[j] = (uint8_t)(q[j / 4] >> (8 * (j % 4)));
                    }
                    if (c < cols && t % kLanes == 0) o.E[row * o.lde + c / kKeepBlock] = (uint8_t)e;
                }
            }
        }
        if (next >= rows) break;
        row = next;
    }
}

struct BackwardSpans {
    Span dy, ds, s, weight;
};

template <typename T, int TPR, int EPT, bool ANY>
__global__ void __launch_bounds__(kBlockOf<TPR>, (kBackwardCtas<TPR, EPT>)) rmsnorm_backward_kernel(
    const T* dY, int64_t lddy, const T* dS, int64_t ldds, const T* __restrict__ S, int64_t lds, const T* __restrict__ w,
    const float* __restrict__ rstd_of, const __grid_constant__ BackwardSpans in, int64_t rows, int cols, T* dX, int64_t lddx, bool dx_vec, float* __restrict__ parts,
    int64_t ldp) {
    constexpr int N = Piece<T>::N, P = EPT / N, RPB = kBlockOf<TPR> / TPR;
    __shared__ float sm[TPR > 32 ? 2 * (TPR / 32) : 1];
    pdl_trigger();
    pdl_wait();
    const int t = threadIdx.x % TPR;
    const float inv_cols = 1.f / (float)cols;
    const int64_t stride = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    uint64_t acc[P][N / 2];
    uint4 weight[P], dy[P], s[P], ds[P];
    float rstd = 0.f;
    const T *from_dy = dY + row * lddy, *from_s = S + row * lds, *from_ds = dS ? dS + row * ldds : nullptr;
    const float* from_rstd = rstd_of + row;
    auto fetch = [&] {
        rstd = load_here(from_rstd);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int c = (t + i * TPR) * N;
            dy[i] = load_piece<ANY>(from_dy, c, cols, in.dy);
            s[i] = load_piece<ANY>(from_s, c, cols, in.s);
            if (from_ds) ds[i] = load_piece<ANY>(from_ds, c, cols, in.ds);
        }
        from_rstd += stride;
        from_dy += stride * lddy;
        from_s += stride * lds;
        if (from_ds) from_ds += stride * ldds;
    };
#pragma unroll
    for (int i = 0; i < P; ++i) {
        if ((kAhead<TPR, EPT>)) weight[i] = load_piece<ANY>(w, (t + i * TPR) * N, cols, in.weight);
        ds[i] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int j = 0; j < N / 2; ++j) acc[i][j] = 0ull;
    }
    if ((kAhead<TPR, EPT>) && row < rows) fetch();
    for (int turn = 0; row < rows; ++turn) {
        if (!(kAhead<TPR, EPT>)) fetch();
        uint64_t dyw[P][N / 2], hat[P][N / 2];
        const uint64_t scale2 = pair_of(rstd, rstd);
        uint4 extra[P];
        uint64_t dot2 = 0ull;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            extra[i] = ds[i];
            uint64_t f[N / 2];
            Piece<T>::split((kAhead<TPR, EPT>) ? weight[i] : load_piece<ANY>(w, (t + i * TPR) * N, cols, in.weight), f);
            Piece<T>::split(dy[i], dyw[i]);
            Piece<T>::split(s[i], hat[i]);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                hat[i][j] = mul2(hat[i][j], scale2);
                acc[i][j] = fma2(dyw[i][j], hat[i][j], acc[i][j]);
                dyw[i][j] = mul2(dyw[i][j], f[j]);
                dot2 = fma2(dyw[i][j], hat[i][j], dot2);
            }
        }
        const int64_t next = row + stride;
        if ((kAhead<TPR, EPT>) && next < rows) fetch();
        if (dX) {
            const float dot = row_sum<TPR>(pair_lo(dot2) + pair_hi(dot2), sm, turn) * -inv_cols;
            const uint64_t ndot2 = pair_of(dot, dot);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                uint64_t out[N / 2];
                Piece<T>::split(extra[i], out);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) out[j] = fma2(scale2, fma2(hat[i][j], ndot2, dyw[i][j]), out[j]);
                store_piece(dX + row * lddx, (t + i * TPR) * N, cols, !ANY || dx_vec, out);
            }
        }
        row = next;
    }
    if (!parts) return;
    float* part = parts + (int64_t)blockIdx.x * ldp;
    if constexpr (RPB == 1) {
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int j = 0; j < N; j += 4) {
                const int c = (t + i * TPR) * N + j;
                if (c < ldp) *reinterpret_cast<ulonglong2*>(part + c) = make_ulonglong2(acc[i][j / 2], acc[i][j / 2 + 1]);
            }
    } else {
        // the CTA's warps one after another
        __shared__ float all[TPR * EPT];
        for (int k = 0; k < RPB; ++k) {
            if (threadIdx.x / TPR == k) {
#pragma unroll
                for (int i = 0; i < P; ++i)
#pragma unroll
                    for (int j = 0; j < N; ++j) {
                        const int c = (t + i * TPR) * N + j;
                        const float a = j & 1 ? pair_hi(acc[i][j / 2]) : pair_lo(acc[i][j / 2]);
                        all[c] = k == 0 ? a : all[c] + a;
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += kBlockOf<TPR>) part[c] = all[c];
    }
}

// dw[c] = sum over the partial rows: a CTA has 32 columns, a thread 4 of them and every 128th row
constexpr int kDwThreads = 1024, kDwCols = 32;
__global__ void __launch_bounds__(kDwThreads) rmsnorm_dw_kernel(const float* __restrict__ parts, int nparts, int64_t ldp,
                                                                int cols, float* __restrict__ dw) {
    constexpr int kQuads = kDwCols / 4, kGroups = kDwThreads / kQuads;
    __shared__ float sm[kGroups][kDwCols + 1];
    pdl_trigger();
    pdl_wait();
    const int x = threadIdx.x % kQuads, y = threadIdx.x / kQuads;
    const float* from = parts + (int64_t)blockIdx.x * kDwCols + 4 * x;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 5
    for (int r = y; r < nparts; r += kGroups) {
        const float4 v = *reinterpret_cast<const float4*>(from + (int64_t)r * ldp);
        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
    }
    sm[y][4 * x] = sum.x; sm[y][4 * x + 1] = sum.y; sm[y][4 * x + 2] = sum.z; sm[y][4 * x + 3] = sum.w;
    __syncthreads();
    // a warp for each column
    const int c = threadIdx.x / 32, lane = threadIdx.x % 32;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < kGroups / 32; ++k) v += sm[lane + 32 * k][c];
    v = warp_sum(v);
    const int64_t col = (int64_t)blockIdx.x * kDwCols + c;
    if (lane == 0 && col < cols) dw[col] = v;
}
static_assert(kDwThreads / 32 == kDwCols, "a warp for each column");
int64_t parts_pitch(int64_t cols) { return (cols + kDwCols - 1) / kDwCols * kDwCols; }

// Calls f<TPR, EPT>() with the threads and entries for rows of this width: up to 512 columns (fp32: 256) a warp, without
// barriers; then 8 entries a thread where that is enough, since registers are what limits the rows in flight.
template <typename T, typename F>
detox_status by_width(int64_t cols, F f) {
    if (cols <= 32 * 8) return f.template operator()<32, 8>();
    if (sizeof(T) == 2 && cols <= 32 * 16) return f.template operator()<32, 16>();
    if (cols <= 128 * 8) return f.template operator()<128, 8>();
    if (cols <= 256 * 8) return f.template operator()<256, 8>();
    if constexpr (sizeof(T) == 2) {
        if (cols <= 256 * 16) return f.template operator()<256, 16>();
        if (cols <= 512 * 16) return f.template operator()<512, 16>();
    } else {
        if (cols <= 512 * 8) return f.template operator()<512, 8>();
        if (cols <= 1024 * 8) return f.template operator()<1024, 8>();
    }
    if (cols <= 1024 * 16) return f.template operator()<1024, 16>();
    return f.template operator()<1024, 32>();
}
// 16-byte pieces can be stored: base and stride
template <typename T>
bool pieces(const void* p, int64_t ld) {
    return aligned16(p) && ld % Piece<T>::N == 0;
}

// CTAs of the backward pass, each leaving one row of partial sums of dw
struct CountParts {
    int64_t rows;
    int* out;
    template <int TPR, int EPT>
    detox_status operator()() const {
        const int64_t need = ceil_div(rows, (int64_t)(kBlockOf<TPR> / TPR)), most = (int64_t)kSMs * kBackwardCtas<TPR, EPT>;
        *out = (int)(need < most ? need : most);
        return DETOX_OK;
    }
};
template <typename T>
int parts_of(int64_t rows, int64_t cols) {
    int n = 0;
    by_width<T>(cols, CountParts{rows, &n});
    return n;
}

template <typename T, bool ANY>
struct Forward {
    NormIn in;
    int64_t rows, cols;
    float eps;
    NormOut o;
    cudaStream_t s;
    template <int TPR, int EPT>
    detox_status operator()() const {
        constexpr int RPB = kBlockOf<TPR> / TPR;
        const int64_t need = ceil_div(rows, (int64_t)RPB), most = (int64_t)kSMs * kForwardCtas<TPR, EPT>;
        return launch_chained(rmsnorm_kernel<T, TPR, EPT, ANY>, (unsigned)(need < most ? need : most), kBlockOf<TPR>, 0, 1, s, in, rows,
                              (int)cols, eps, o);
    }
};

struct BackwardIn {
    const void* dY; int64_t lddy;
    const void* dS; int64_t ldds;
    const void* S; int64_t lds;
    const void* w;
    const float* rstd;
    BackwardSpans span;
};
template <typename T, bool ANY>
struct Backward {
    BackwardIn in;
    int64_t rows, cols;
    void* dX; int64_t lddx;
    float* parts;
    int nparts;
    cudaStream_t s;
    template <int TPR, int EPT>
    detox_status operator()() const {
        return launch_chained(rmsnorm_backward_kernel<T, TPR, EPT, ANY>, (unsigned)nparts, kBlockOf<TPR>, 0, 1, s,
                              static_cast<const T*>(in.dY), in.lddy, static_cast<const T*>(in.dS), in.ldds, static_cast<const T*>(in.S),
                              in.lds, static_cast<const T*>(in.w), in.rstd, in.span, rows, (int)cols, static_cast<T*>(dX), lddx, pieces<T>(dX, lddx), parts, parts_pitch(cols));
    }
};

template <typename T>
detox_status forward(NormIn in, int64_t rows, int64_t cols, float eps, NormOut o, cudaStream_t s) {
    in.x = span_of<T>(in.X, in.ldx, rows, cols);
    in.r = span_of<T>(in.R, in.ldr, rows, cols);
    in.weight = span_of<T>(in.w, 0, 1, cols);
    o.s_vec = pieces<T>(o.S, o.lds);
    o.y_vec = pieces<T>(o.Y, o.ldy);
    o.q_vec = aligned_to(o.Q, 8) && o.ldq % 8 == 0;
    if (cols % Piece<T>::N == 0 && in.x.vec && (!in.R || in.r.vec) && in.weight.vec && (!o.S || o.s_vec) && (!o.Y || o.y_vec) && (!o.Q || o.q_vec))
        return by_width<T>(cols, Forward<T, false>{in, rows, cols, eps, o, s});
    return by_width<T>(cols, Forward<T, true>{in, rows, cols, eps, o, s});
}

template <typename T>
detox_status backward(BackwardIn in, int64_t rows, int64_t cols, void* dX, int64_t lddx, float* parts, cudaStream_t s) {
    const int nparts = parts_of<T>(rows, cols);
    in.span.dy = span_of<T>(in.dY, in.lddy, rows, cols);
    in.span.ds = span_of<T>(in.dS, in.ldds, rows, cols);
    in.span.s = span_of<T>(in.S, in.lds, rows, cols);
    in.span.weight = span_of<T>(in.w, 0, 1, cols);
    if (cols % Piece<T>::N == 0 && in.span.dy.vec && (!in.dS || in.span.ds.vec) && in.span.s.vec && in.span.weight.vec && (!dX || pieces<T>(dX, lddx)))
        return by_width<T>(cols, Backward<T, false>{in, rows, cols, dX, lddx, parts, nparts, s});
    return by_width<T>(cols, Backward<T, true>{in, rows, cols, dX, lddx, parts, nparts, s});
}

}  // namespace

detox_status launch_rmsnorm(int dtype, const void* X, int64_t ldx, const void* R, int64_t ldr, const void* w,
                            int64_t rows, int64_t cols, float eps, void* S, int64_t lds, void* Y, int64_t ldy,
                            uint8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, float* rstd, cudaStream_t s) {
    if (rows == 0) return DETOX_OK;
    const NormIn in{X, ldx, R, ldr, w, {}, {}, {}};
    const NormOut o{S, lds, Y, ldy, Q, ldq, E, lde, rstd, false, false, false};
    if (dtype == DETOX_DTYPE_FLOAT) return forward<float>(in, rows, cols, eps, o, s);
    if (dtype == DETOX_DTYPE_HALF) return forward<__half>(in, rows, cols, eps, o, s);
    return forward<__nv_bfloat16>(in, rows, cols, eps, o, s);
}

size_t rmsnorm_backward_ws_bytes(int64_t rows, int64_t cols) {
    int n = 1;   // (whatever the type)
    if (rows > 0) n = parts_of<float>(rows, cols) > parts_of<__half>(rows, cols) ? parts_of<float>(rows, cols) : parts_of<__half>(rows, cols);
    return align_up((size_t)n * (size_t)parts_pitch(cols) * sizeof(float));
}

detox_status launch_rmsnorm_backward(int dtype, const void* dY, int64_t lddy, const void* dS, int64_t ldds, const void* S,
                                     int64_t lds, const void* w, const float* rstd, int64_t rows, int64_t cols, void* dX,
                                     int64_t lddx, float* dw, void* ws, cudaStream_t s) {
    if (rows == 0) {
        if (dw && cudaMemsetAsync(dw, 0, (size_t)cols * sizeof(float), s) != cudaSuccess) return DETOX_ERR_CUDA;
        return DETOX_OK;
    }
    float* parts = dw ? static_cast<float*>(ws) : nullptr;
    const BackwardIn in{dY, lddy, dS, ldds, S, lds, w, rstd, {}};
    detox_status st;
    if (dtype == DETOX_DTYPE_FLOAT) st = backward<float>(in, rows, cols, dX, lddx, parts, s);
    else if (dtype == DETOX_DTYPE_HALF) st = backward<__half>(in, rows, cols, dX, lddx, parts, s);
    else st = backward<__nv_bfloat16>(in, rows, cols, dX, lddx, parts, s);
    if (st != DETOX_OK || !dw) return st;
    return launch_chained(rmsnorm_dw_kernel, (unsigned)ceil_div(cols, (int64_t)kDwCols), kDwThreads, 0, 1, s, parts,
                          dtype == DETOX_DTYPE_FLOAT ? parts_of<float>(rows, cols) : parts_of<__half>(rows, cols), parts_pitch(cols), (int)cols, dw);
}

}  // namespace detox
