// Shared by the worker-side operators and the optimizer (rmsnorm.cu, checkpoint.cu, gated.cu, embedding.cu, token_loss.cu, adamw.cu): element types, the 8-bit form of kept
// activations, and the launcher declarations (internal).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "tcgen05.cuh"

namespace detox {

constexpr int kKeepBlock = DETOX_KEEP_BLOCK;   // columns that share a scale

// ---- element types ----------------------------------------------------------------------------
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// two fp32 values rounded and packed (a in the low half), and back
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t v);
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t v) {
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

// packed pairs of fp32
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
    return ((uint64_t)__float_as_uint(hi) << 32) | __float_as_uint(lo);
}
__device__ __forceinline__ float pair_lo(uint64_t p) { return __uint_as_float((uint32_t)p); }
__device__ __forceinline__ float pair_hi(uint64_t p) { return __uint_as_float((uint32_t)(p >> 32)); }

// the 16 / sizeof(T) entries of a 16-byte piece
template <typename T>
struct Piece {
    static constexpr int N = 16 / (int)sizeof(T);
    static __device__ __forceinline__ void split(uint4 v, float (&f)[N]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) {
                f[i] = __uint_as_float(w[i]);
            } else {
                const float2 p = unpack2<T>(w[i]);
                f[2 * i] = p.x;
                f[2 * i + 1] = p.y;
            }
        }
    }
    // the same as packed pairs of fp32, which the two-lane instructions work on
    static __device__ __forceinline__ void split(uint4 v, uint64_t (&p)[N / 2]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            if constexpr (sizeof(T) == 4) {
                p[i] = ((uint64_t)w[2 * i + 1] << 32) | w[2 * i];
            } else {
                const float2 f = unpack2<T>(w[i]);
                p[i] = pair_of(f.x, f.y);
            }
        }
    }
    static __device__ __forceinline__ uint4 join(const uint64_t (&p)[N / 2]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            if constexpr (sizeof(T) == 4) {
                w[2 * i] = (uint32_t)p[i];
                w[2 * i + 1] = (uint32_t)(p[i] >> 32);
            } else {
                w[i] = pack2<T>(pair_lo(p[i]), pair_hi(p[i]));
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    static __device__ __forceinline__ uint4 join(const float (&f)[N]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f[i]);
            else w[i] = pack2<T>(f[2 * i], f[2 * i + 1]);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// ---- rows of any alignment ----------------------------------------------------------------------
// A matrix as the kernels that take any alignment read it: `vec` says that its rows are 16-byte aligned; otherwise `lo` and
// `hi` bound its bytes.
struct Span {
    uintptr_t lo, hi;
    bool vec;
};
template <typename T>
Span span_of(const void* p, int64_t ld, int64_t rows, int64_t cols) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return Span{at, at + ((uintptr_t)(rows - 1) * (uintptr_t)ld + (uintptr_t)cols) * sizeof(T), aligned16(p) && ld % Piece<T>::N == 0};
}
// entries [c, c + N) of a row as they lie in memory, bit for bit, zeros beyond `cols`
template <typename T, typename I>
__device__ __forceinline__ uint4 gather_piece(const T* row, I c, I cols) {
    uint32_t w[4];
    if constexpr (sizeof(T) == 4) {
        const uint32_t* x = reinterpret_cast<const uint32_t*>(row);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = c + i < cols ? x[c + i] : 0u;
    } else {
        const uint16_t* x = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = (c + 2 * i < cols ? (uint32_t)x[c + 2 * i] : 0u) | (c + 2 * i + 1 < cols ? (uint32_t)x[c + 2 * i + 1] << 16 : 0u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// 16 bytes, or zeros.  Volatile: the load is issued where it is written.  The compiler otherwise moves the loads of the next row
// behind the reduction of the present one, which they are there to overlap (norm's backward pass 28.4 instead of 25.7 us).
__device__ __forceinline__ uint4 load_here(const void* from, bool want) {
    uint4 v;
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t"
        "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
        "@p ld.global.cs.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
        : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
        : "l"(from), "r"((uint32_t)want)
        : "memory");
    return v;
}
__device__ __forceinline__ float load_here(const float* from) {
    float v;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(from) : "memory");
    return v;
}
// The same.  ANY = false: the rows are 16-byte aligned and whole pieces long.  ANY = true: see span; where they are not aligned a piece is two aligned loads,
// shifted together (a norm of 4928 x 1087 bf16 with such rows: 27 us with a load for each entry), and only at the ends of
// the matrix, where those would reach outside it, a load for each entry.
template <bool ANY, typename T, typename I>
__device__ __forceinline__ uint4 load_piece(const T* row, I c, I cols, const Span& span) {
    if constexpr (!ANY) return load_here(row + c, c < cols);
    if (c + Piece<T>::N > cols) return gather_piece(row, c, cols);
    if (span.vec) return ld_stream_u4(row + c);
    const uintptr_t at = reinterpret_cast<uintptr_t>(row + c), a = at & ~(uintptr_t)15;
    if (a < span.lo || a + 32 > span.hi) return gather_piece(row, c, cols);
    const uint4 x = *reinterpret_cast<const uint4*>(a), y = *reinterpret_cast<const uint4*>(a + 16);
    uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
    const uint32_t by = (uint32_t)(at & 15);
    if (by & 8) {
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
    }
    if (by & 4) {
#pragma unroll
        for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
    }
    const uint32_t bits = (by & 3) * 8;
    return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                      __funnelshift_r(w[3], w[4], bits));
}
// ... and stored
template <typename T>
__device__ __forceinline__ void store_piece(T* row, int c, int cols, bool vec, const uint64_t (&p)[Piece<T>::N / 2]) {
    constexpr int N = Piece<T>::N;
    if (vec && c + N <= cols) {
        st_stream_u4(row + c, Piece<T>::join(p));
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c + j < cols) row[c + j] = from_f32<T>(j & 1 ? pair_hi(p[j / 2]) : pair_lo(p[j / 2]));
    }
}

// ---- the 8-bit form ---------------------------------------------------------------------------
// Biased exponent (e + 127) of the scale: the smallest e with amax <= 448 * 2^e = 1.75 * 2^(e+8), at least -126.
// Adding 0x1fffff carries into the exponent exactly when the mantissa is above 1.75.
__device__ __forceinline__ uint32_t keep_exponent(float amax) {
    const int e = (int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8;
    return (uint32_t)(e < 1 ? 1 : e);
}
// 2^e and 2^-e of a biased exponent in 1 .. 247 (both are normal numbers)
__device__ __forceinline__ float keep_scale(uint32_t e) { return __uint_as_float(e << 23); }
__device__ __forceinline__ float keep_inverse(uint32_t e) { return __uint_as_float((254u - e) << 23); }
// A scale byte as it is read back: 0 (never written by this library) stands for 2^-127, 255 for NaN.
__device__ __forceinline__ float keep_scale_of_byte(uint32_t e) {
    return __uint_as_float(e == 0u ? 0x00400000u : (e == 255u ? 0x7fc00000u : e << 23));
}
// A block's largest entry is taken as max |v|, which passes over NaN.  Only when that comes out as Inf is it taken again
// after the Infs have been turned into NaN (v + 0 v), which is also how they are kept.
__device__ __forceinline__ bool is_inf(float amax) { return amax > 3.402823466e38f; }
__device__ __forceinline__ float inf_to_nan(float v) { return fmaf(v, 0.f, v); }
// Four values, already divided by the scale (so at most 448, or NaN), to four e4m3 bytes (a first).
__device__ __forceinline__ uint32_t keep4(float a, float b, float c, float d) {
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
}
// The 8-bit form of 2 * PAIRS entries of a block that lies in LANES neighbouring lanes of a warp (whole warps call this).
// Returns the biased exponent; v is used up.
template <int PAIRS, int LANES>
__device__ __forceinline__ uint32_t keep_pairs(uint64_t (&v)[PAIRS], uint32_t (&q)[PAIRS / 2]) {
    auto largest = [&] {
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) amax = fmaxf(amax, fmaxf(fabsf(pair_lo(v[i])), fabsf(pair_hi(v[i]))));
#pragma unroll
        for (int s = LANES / 2; s > 0; s >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, s));
        return amax;
    };
    float amax = largest();
    if (__any_sync(0xffffffffu, is_inf(amax))) {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) v[i] = pair_of(inf_to_nan(pair_lo(v[i])), inf_to_nan(pair_hi(v[i])));
        amax = largest();
    }
    const uint32_t e = keep_exponent(amax);
    const float inv = keep_inverse(e);
    const uint64_t inv2 = pair_of(inv, inv);
#pragma unroll
    for (int i = 0; i < PAIRS; ++i) v[i] = mul2(v[i], inv2);
#pragma unroll
    for (int i = 0; i < PAIRS / 2; ++i) q[i] = keep4(pair_lo(v[2 * i]), pair_hi(v[2 * i]), pair_lo(v[2 * i + 1]), pair_hi(v[2 * i + 1]));
    return e;
}
// ... and back (not yet multiplied by the scale)
__device__ __forceinline__ void taken4(uint32_t q, float (&f)[4]) {
    uint32_t lo, hi;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)(q & 0xffffu)));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(q >> 16)));
    const float2 a = unpack2<__half>(lo), b = unpack2<__half>(hi);
    f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
}
// A taken-out value in its type: exact in fp32 and bf16; fp16 is clamped to its largest number (NaN stays NaN).
template <typename T> __device__ __forceinline__ float taken_clamp(float v) { return v; }
template <> __device__ __forceinline__ float taken_clamp<__half>(float v) {
    return v > 65504.f ? 65504.f : (v < -65504.f ? -65504.f : v);
}

// ---- launches that overlap the end of the kernel before them -------------------------------------
// A step is a chain of short kernels, so each is launched while the one before it drains: its setup (barriers, tensor
// memory) runs early, and pdl_wait holds it until everything before it in the stream has finished and is visible.
// pdl_trigger lets the next one in as soon as all of this kernel's CTAs have started.
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_trigger() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// chained = false: a launch without overlap, for a kernel that must have the GPU to itself.
template <typename... P, typename... A>
detox_status launch(bool chained, void (*kernel)(P...), dim3 grid, unsigned block, size_t smem, unsigned cluster, cudaStream_t s,
                    const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    unsigned n = 0;
    if (chained) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    const bool ok = cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) == cudaSuccess;
    return launch_status() == DETOX_OK && ok ? DETOX_OK : DETOX_ERR_CUDA;
}
template <typename... P, typename... A>
detox_status launch_chained(void (*kernel)(P...), dim3 grid, unsigned block, size_t smem, unsigned cluster, cudaStream_t s,
                            const A&... args) {
    return launch(true, kernel, grid, block, smem, cluster, s, args...);
}

inline bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// ---- launchers (each enqueues on `s`; none synchronises) ---------------------------------------

// checkpoint.cu
detox_status launch_checkpoint_pack(int dtype, const void* X, int64_t ld, int64_t rows, int64_t cols, uint8_t* Q,
                                    int64_t ldq, uint8_t* E, int64_t lde, cudaStream_t s);
detox_status launch_checkpoint_unpack(int dtype, const uint8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde,
                                      int64_t rows, int64_t cols, void* X, int64_t ld, cudaStream_t s);

// rmsnorm.cu
detox_status launch_rmsnorm(int dtype, const void* X, int64_t ldx, const void* R, int64_t ldr, const void* w,
                            int64_t rows, int64_t cols, float eps, void* S, int64_t lds, void* Y, int64_t ldy,
                            uint8_t* Q, int64_t ldq, uint8_t* E, int64_t lde, float* rstd, cudaStream_t s);
size_t rmsnorm_backward_ws_bytes(int64_t rows, int64_t cols);
detox_status launch_rmsnorm_backward(int dtype, const void* dY, int64_t lddy, const void* dS, int64_t ldds, const void* S,
                                     int64_t lds, const void* w, const float* rstd, int64_t rows, int64_t cols, void* dX,
                                     int64_t lddx, float* dw, void* ws, cudaStream_t s);

// embedding.cu
detox_status launch_embedding(int dtype, const void* W, int64_t ldw, int64_t vocab, int64_t cols, int index, const void* tokens,
                              int64_t rows, float scale, void* Y, int64_t ldy, cudaStream_t s);
size_t embedding_backward_ws_bytes(int64_t rows, int64_t vocab, int64_t cols);
detox_status launch_embedding_backward(int dtype, const void* dY, int64_t lddy, int index, const void* tokens, int64_t rows, int64_t vocab,
                                       int64_t cols, float scale, void* dW, int64_t lddw, int dw_dtype, bool add, void* ws, cudaStream_t s);

// token_loss.cu
detox_status launch_token_logp(int dtype, const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y, float scale,
                               float* logp, float* lse, cudaStream_t s);
detox_status launch_token_logp_backward(int dtype, const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y,
                                        float scale, const float* lse, const float* dlogp, void* dZ, int64_t lddz, cudaStream_t s);
size_t policy_loss_ws_bytes(int64_t rows);
detox_status launch_policy_loss(const detox_policy_desc& d, float* stats, float* logp, void* dZ, int64_t lddz, void* ws, cudaStream_t s);
size_t preference_loss_ws_bytes(int64_t rows, int64_t pairs);
detox_status launch_preference_loss(const detox_preference_desc& d, float* loss, float* margin, float* sums, void* dZ, int64_t lddz, void* ws,
                                    cudaStream_t s);

// adamw.cu
detox_status launch_adamw(const detox_adamw_desc& d, const detox_adamw_tensor* tensors, int64_t count, cudaStream_t s);

// gated.cu
size_t gated_ws_bytes(const detox_gated_desc& g);
size_t gated_backward_ws_bytes(const detox_gated_desc& g);
long long gated_wait_limit(long long clocks);
unsigned long long gated_expired_waits(int32_t* first, bool clear);
detox_status launch_gated(const detox_gated_desc& g, void* H, int64_t ldh, void* ws, cudaStream_t s);
detox_status launch_gated_backward(const detox_gated_desc& g, const void* dH, int64_t lddh, void* dX, int64_t lddx,
                                   void* dWg, void* dWu, int64_t lddw, int dw_dtype, void* ws, cudaStream_t s);

}  // namespace detox
