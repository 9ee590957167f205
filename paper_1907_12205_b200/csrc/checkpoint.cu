// Activation checkpoints in 8 bits: e4m3 entries with a power-of-two scale for each block of 128 columns of a row.
//
// Pack:  amax = max |v| over the block;  e = the smallest integer with amax <= 448 * 2^e;  q = e4m3(v * 2^-e).
// Bound by HBM: 2 + 1 (fp32: 4 + 1) bytes an entry and a byte for each block.  One pass: eight neighbouring lanes hold
// a block, 16 entries each, and agree on its largest entry by three shuffles, so the entries never leave the registers.
#include "worker.cuh"

namespace detox {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 16;                         // entries of a lane
constexpr int kLanes = kKeepBlock / kPer;        // lanes of a block

// Blocks are numbered row by row; a group of eight lanes takes every `groups`-th one.  The row and the block's place in
// it are carried along instead of divided out of the number.
struct Walk {
    int64_t row;
    int blk;
    __device__ __forceinline__ Walk(int64_t item, int nblk) : row(item / nblk), blk((int)(item % nblk)) {}
    __device__ __forceinline__ void step(int64_t drow, int dblk, int nblk) {
        row += drow;
        blk += dblk;
        if (blk >= nblk) { blk -= nblk; ++row; }
    }
};

template <typename T, bool ANY>
__global__ void __launch_bounds__(kThreads) pack_kernel(const T* __restrict__ X, int64_t ld, Span span, int64_t rows, int64_t cols,
                                                        int nblk, uint8_t* __restrict__ Q, int64_t ldq, bool q_vec,
                                                        uint8_t* __restrict__ E, int64_t lde) {
    constexpr int N = Piece<T>::N;
    pdl_trigger();
    pdl_wait();
    const int64_t groups = (int64_t)gridDim.x * (kThreads / kLanes);
    const int part = threadIdx.x % kLanes;
    const int64_t drow = groups / nblk;
    const int dblk = (int)(groups % nblk);
    Walk w(((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes, nblk);
    for (; __any_sync(0xffffffffu, w.row < rows); w.step(drow, dblk, nblk)) {
        const bool live = w.row < rows;
        const int64_t c0 = (int64_t)w.blk * kKeepBlock + part * kPer;
        const bool full = live && c0 + kPer <= cols;
        const T* x = X + w.row * ld;
        uint4 raw[kPer / N];
#pragma unroll
        for (int i = 0; i < kPer / N; ++i) raw[i] = load_piece<ANY>(x, c0 + i * N, live ? cols : (int64_t)0, span);
        uint64_t v[kPer / 2];
#pragma unroll
        for (int i = 0; i < kPer / N; ++i) {
            uint64_t f[N / 2];
            Piece<T>::split(raw[i], f);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) v[i * (N / 2) + j] = f[j];
        }
        uint32_t q[kPer / 4];
        const uint32_t e = keep_pairs<kPer / 2, kLanes>(v, q);
        uint8_t* to = Q + w.row * ldq + c0;
        if (full && (!ANY || q_vec)) {
            st_stream_u4(to, make_uint4(q[0], q[1], q[2], q[3]));
        } else if (live) {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (c0 + i < cols) to[i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
        }
        if (live && part == 0) E[w.row * lde + w.blk] = (uint8_t)e;
    }
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads) unpack_kernel(const uint8_t* __restrict__ Q, int64_t ldq,
                                                          const uint8_t* __restrict__ E, int64_t lde, int64_t rows,
                                                          int64_t cols, int nblk, T* __restrict__ X, int64_t ld) {
    constexpr int N = Piece<T>::N;
    pdl_trigger();
    pdl_wait();
    const int64_t groups = (int64_t)gridDim.x * (kThreads / kLanes);
    const int part = threadIdx.x % kLanes;
    const int64_t drow = groups / nblk;
    const int dblk = (int)(groups % nblk);
    Walk w(((int64_t)blockIdx.x * kThreads + threadIdx.x) / kLanes, nblk);
    for (; w.row < rows; w.step(drow, dblk, nblk)) {
        const int64_t c0 = (int64_t)w.blk * kKeepBlock + part * kPer;
        if (c0 >= cols) continue;
        const bool full = VEC && c0 + kPer <= cols;
        const uint8_t* from = Q + w.row * ldq + c0;
        const float scale = keep_scale_of_byte(E[w.row * lde + w.blk]);
        uint32_t q[kPer / 4] = {0u, 0u, 0u, 0u};
        if (full) {
            const uint4 p = ld_stream_u4(from);
            q[0] = p.x; q[1] = p.y; q[2] = p.z; q[3] = p.w;
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (c0 + i < cols) q[i / 4] |= (uint32_t)from[i] << (8 * (i % 4));
        }
        float v[kPer];
#pragma unroll
        for (int i = 0; i < kPer / 4; ++i) {
            float f[4];
            taken4(q[i], f);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = taken_clamp<T>(f[j] * scale);
        }
        T* x = X + w.row * ld + c0;
        if (full) {
#pragma unroll
            for (int i = 0; i < kPer / N; ++i) {
                float f[N];
#pragma unroll
                for (int j = 0; j < N; ++j) f[j] = v[i * N + j];
                st_stream_u4(x + i * N, Piece<T>::join(f));
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (c0 + i < cols) x[i] = from_f32<T>(v[i]);
        }
    }
}

unsigned grid_for(int64_t rows, int nblk) {
    const int64_t need = ceil_div(rows * nblk, (int64_t)(kThreads / kLanes));
    const int64_t most = (int64_t)kSMs * 16;
    return (unsigned)(need < most ? need : most);
}

template <typename T>
detox_status pack(const void* X, int64_t ld, int64_t rows, int64_t cols, uint8_t* Q, int64_t ldq, uint8_t* E, int64_t lde,
                  cudaStream_t s) {
    const int nblk = (int)ceil_div(cols, (int64_t)kKeepBlock);
    const Span span = span_of<T>(X, ld, rows, cols);
    const bool q_vec = aligned16(Q) && ldq % 16 == 0;
    return launch_chained(cols % Piece<T>::N == 0 && span.vec && q_vec ? pack_kernel<T, false> : pack_kernel<T, true>, grid_for(rows, nblk), kThreads, 0, 1, s,
                          static_cast<const T*>(X), ld, span, rows, cols, nblk, Q, ldq, q_vec, E, lde);
}
template <typename T>
detox_status unpack(const uint8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t rows, int64_t cols, void* X,
                    int64_t ld, cudaStream_t s) {
    const int nblk = (int)ceil_div(cols, (int64_t)kKeepBlock);
    const bool vec = aligned16(X) && ld % Piece<T>::N == 0 && aligned16(Q) && ldq % 16 == 0;
    auto* k = vec ? unpack_kernel<T, true> : unpack_kernel<T, false>;
    return launch_chained(k, grid_for(rows, nblk), kThreads, 0, 1, s, Q, ldq, E, lde, rows, cols, nblk, static_cast<T*>(X), ld);
}

}  // namespace

detox_status launch_checkpoint_pack(int dtype, const void* X, int64_t ld, int64_t rows, int64_t cols, uint8_t* Q,
                                    int64_t ldq, uint8_t* E, int64_t lde, cudaStream_t s) {
    if (rows == 0) return DETOX_OK;
    if (dtype == DETOX_DTYPE_FLOAT) return pack<float>(X, ld, rows, cols, Q, ldq, E, lde, s);
    if (dtype == DETOX_DTYPE_HALF) return pack<__half>(X, ld, rows, cols, Q, ldq, E, lde, s);
    return pack<__nv_bfloat16>(X, ld, rows, cols, Q, ldq, E, lde, s);
}

detox_status launch_checkpoint_unpack(int dtype, const uint8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde,
                                      int64_t rows, int64_t cols, void* X, int64_t ld, cudaStream_t s) {
    if (rows == 0) return DETOX_OK;
    if (dtype == DETOX_DTYPE_FLOAT) return unpack<float>(Q, ldq, E, lde, rows, cols, X, ld, s);
    if (dtype == DETOX_DTYPE_HALF) return unpack<__half>(Q, ldq, E, lde, rows, cols, X, ld, s);
    return unpack<__nv_bfloat16>(Q, ldq, E, lde, rows, cols, X, ld, s);
}

}  // namespace detox
