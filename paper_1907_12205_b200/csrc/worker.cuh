// Shared by the worker-side operators (rmsnorm.cu, checkpoint.cu, gated.cu): element types, the 8-bit form of kept
// activations, and the launcher declarations (internal).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

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

// ---- the 8-bit form ---------------------------------------------------------------------------
// |v| where v is finite, else 0: what a block's largest entry is taken over
__device__ __forceinline__ float finite_abs(float v) {
    const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
    return b < 0x7f800000u ? __uint_as_float(b) : 0.f;
}
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
// Four values, already divided by the scale, to four e4m3 bytes (a first).  The conversion saturates, and scaled
// finite values are at most 448, so only an Inf could come out as a number: v + 0 v turns it into NaN beforehand.
__device__ __forceinline__ uint32_t keep4(float a, float b, float c, float d) {
    uint16_t lo, hi;
    a = fmaf(a, 0.f, a); b = fmaf(b, 0.f, b); c = fmaf(c, 0.f, c); d = fmaf(d, 0.f, d);
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return (uint32_t)lo | ((uint32_t)hi << 16);
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

template <typename... P, typename... A>
detox_status launch_chained(void (*kernel)(P...), unsigned grid, unsigned block, size_t smem, unsigned cluster, cudaStream_t s,
                            const A&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const bool ok = cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) == cudaSuccess;
    return launch_status() == DETOX_OK && ok ? DETOX_OK : DETOX_ERR_CUDA;
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

// gated.cu
size_t gated_ws_bytes(const detox_gated_desc& g);
size_t gated_backward_ws_bytes(const detox_gated_desc& g);
detox_status launch_gated(const detox_gated_desc& g, void* H, int64_t ldh, void* ws, cudaStream_t s);
detox_status launch_gated_backward(const detox_gated_desc& g, const void* dH, int64_t lddh, void* dX, int64_t lddx,
                                   void* dWg, void* dWu, int64_t lddw, int dw_dtype, void* ws, cudaStream_t s);

}  // namespace detox
