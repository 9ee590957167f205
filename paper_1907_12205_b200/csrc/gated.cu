// Gated pair of projections, h = act(x Wg^T) * (x Wu^T), and its backward pass, on the tensor cores (tcgen05).
//
// All products are one kernel, a GEMM with fp32 accumulators in tensor memory, in four forms:
//   forward    C = x [Wg ; Wu]^T: an output tile holds 128 columns of g and the same 128 columns of u side by side, so
//              the epilogue has both factors of h in hand, and g and u never travel to HBM in full.  The 128 columns
//              are also exactly one block of the 8-bit form, so a thread (one row) finds the block's scale by itself.
//   recompute  the same product; the epilogue reads dh and leaves dg and du
//   dgrad      dx = dg Wg + du Wu: one accumulator over both products
//   wgrad      dWg = dg^T x, dWu = du^T x
// The reduction runs along the rows of memory in the first two (K-major operands); dgrad's weights and both operands of wgrad
// lie the other way round and are read as MN-major tiles: nothing is transposed in memory.
//
// CTA: one warp issues the TMA copies of 64-wide slices of both operands into a ring of stages, one thread issues
// the MMAs, four warps drain the accumulator.  Two accumulators of 128 x 256 fill the tensor memory, so a tile is drained
// while the next one is multiplied.  The grid is persistent.  Ragged edges: TMA fills with zeros outside a matrix and
// the epilogue masks its stores.
#include <cuda.h>

#include <type_traits>

#include "gram_tc.cuh"
#include "tcgen05.cuh"
#include "worker.cuh"

namespace detox {

namespace {

enum Form { kForward = 0, kRecompute = 1, kDgrad = 2, kWgrad = 3 };

constexpr int kSlice = 64;                       // entries of the reduction per stage: one 128-byte swizzled row
constexpr int kTileM = 128, kTileN = 256;
constexpr uint32_t kChunkBytes = 64 * 128;       // 64 rows of 128 bytes
constexpr uint32_t kABytes = kTileM * 128, kBBytes = kTileN * 128, kStageBytes = kABytes + kBBytes;
constexpr int kStages = 4;
constexpr int kEpiWarps = 4, kThreads = 32 * (2 + kEpiWarps);
constexpr int kTmemCols = 2 * kTileN;

struct GemmSmem {
    uint64_t full[kStages];        // a stage's copies have landed
    uint64_t empty[kStages];       // the MMAs that read it are done
    uint64_t accum_full[2];        // an accumulator is complete
    uint64_t accum_empty[2];       // ... and drained
    uint32_t tmem_base;
    int abort_flag;
};
constexpr size_t kSmemBytes = kStages * (size_t)kStageBytes + sizeof(GemmSmem) + 1024;

struct GemmArgs {
    int mt, nt;                    // output tiles (wgrad: mt counts those of dWg and of dWu)
    int kb0, kb1;                  // slices of the first and of the second product that are added up
    int act;
    int64_t rows, cols;            // of the output (forward, recompute: of h)
    void* out0; void* out1;        // forward: h, -; recompute: dg, du; dgrad: dx, -; wgrad: dWg, dWu
    int64_t ldo;
    bool out_vec;                  // 16-byte stores
    uint8_t *gq, *ge, *uq, *ue;    // forward: the kept g and u, or null
    int64_t ldq, lde;
    bool q_vec;
    const void* dh;                // recompute
    int64_t lddh;
    bool dh_vec;
};

// Shared-memory descriptor of an MN-major operand: chunks of 64 entries (128 swizzled bytes) by 64 steps of the
// reduction; 8 steps lie 1024 bytes apart, the next 64 entries kChunkBytes.
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t addr) {
    uint64_t desc = (uint64_t)((addr & 0x3FFFFu) >> 4);
    desc |= (uint64_t)(kChunkBytes >> 4) << 16;             // leading byte offset: next 64 entries
    desc |= (uint64_t)(1024 >> 4) << 32;                    // stride byte offset: next 8 steps
    desc |= (uint64_t)1 << 46;
    desc |= (uint64_t)2 << 61;                              // 128-byte swizzle
    return desc;
}

__device__ __forceinline__ void tmem_load32(uint32_t taddr, float (&f)[32]) {
    uint32_t v[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(taddr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(v[i]);
}

// ---- activations: a = act(g), da = act'(g) -----------------------------------------------------
template <int ACT>
__device__ __forceinline__ float act_of(float g) {
    if constexpr (ACT == DETOX_ACT_SILU) return __fdividef(g, 1.f + __expf(-g));
    if constexpr (ACT == DETOX_ACT_GELU) return 0.5f * g * (1.f + erff(g * 0.70710678f));
    return fmaxf(g, 0.f);
}
template <int ACT>
__device__ __forceinline__ void act_both(float g, float& a, float& da) {
    if constexpr (ACT == DETOX_ACT_SILU) {
        const float s = __fdividef(1.f, 1.f + __expf(-g));
        a = g * s;
        da = fmaf(a, 1.f - s, s);
    } else if constexpr (ACT == DETOX_ACT_GELU) {
        const float c = fmaf(0.5f, erff(g * 0.70710678f), 0.5f);
        a = g * c;
        da = fmaf(g * 0.39894228f, __expf(-0.5f * g * g), c);
    } else {
        a = fmaxf(g, 0.f);
        da = g > 0.f ? 1.f : 0.f;
    }
}
// calls f<ACT>()
template <typename F>
__device__ __forceinline__ void by_act(int act, F f) {
    if (act == DETOX_ACT_SILU) f.template operator()<DETOX_ACT_SILU>();
    else if (act == DETOX_ACT_GELU) f.template operator()<DETOX_ACT_GELU>();
    else f.template operator()<DETOX_ACT_RELU>();
}
template <int NV>
struct HOf {   // h = act(g) u, into u
    const float (&g)[NV];
    float (&u)[NV];
    template <int ACT> __device__ __forceinline__ void operator()() {
#pragma unroll
        for (int i = 0; i < NV; ++i) u[i] *= act_of<ACT>(g[i]);
    }
};
template <int NV>
struct DguOf {   // (g, u, dh) -> (dg, du, -)
    float (&g)[NV];
    float (&u)[NV];
    const float (&dh)[NV];
    template <int ACT> __device__ __forceinline__ void operator()() {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float a, da;
            act_both<ACT>(g[i], a, da);
            g[i] = dh[i] * u[i] * da;
            u[i] = dh[i] * a;
        }
    }
};

// ---- 32 consecutive entries of an output row ----------------------------------------------------
template <typename OT>
__device__ __forceinline__ void store32(OT* row, int64_t c, int64_t cols, bool vec, const float (&f)[32]) {
    constexpr int N = Piece<OT>::N;
    if (vec && c + 32 <= cols) {
#pragma unroll
        for (int i = 0; i < 32 / N; ++i) {
            float p[N];
#pragma unroll
            for (int j = 0; j < N; ++j) p[j] = f[i * N + j];
            *reinterpret_cast<uint4*>(row + c + i * N) = Piece<OT>::join(p);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (c + i < cols) row[c + i] = from_f32<OT>(f[i]);
    }
}
template <typename T>
__device__ __forceinline__ void load32(const T* row, int64_t c, int64_t cols, bool vec, float (&f)[32]) {
    constexpr int N = Piece<T>::N;
    if (vec && c + 32 <= cols) {
#pragma unroll
        for (int i = 0; i < 32 / N; ++i) {
            float p[N];
            Piece<T>::split(*reinterpret_cast<const uint4*>(row + c + i * N), p);
#pragma unroll
            for (int j = 0; j < N; ++j) f[i * N + j] = p[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) f[i] = c + i < cols ? to_f32(row[c + i]) : 0.f;
    }
}
// 32 entries of the 8-bit form
__device__ __forceinline__ void keep32(uint8_t* row, int64_t c, int64_t cols, bool vec, float inv, const float (&f)[32]) {
    uint32_t q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = keep4(f[4 * i] * inv, f[4 * i + 1] * inv, f[4 * i + 2] * inv, f[4 * i + 3] * inv);
    if (vec && c + 32 <= cols) {
        *reinterpret_cast<uint4*>(row + c) = make_uint4(q[0], q[1], q[2], q[3]);
        *reinterpret_cast<uint4*>(row + c + 16) = make_uint4(q[4], q[5], q[6], q[7]);
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (c + i < cols) row[c + i] = (uint8_t)(q[i / 4] >> (8 * (i % 4)));
    }
}

// Maps: forward, recompute: a0 = x, b0 = Wg, b1 = Wu; dgrad: a0 = dg, a1 = du, b0 = Wg, b1 = Wu; wgrad: a0 = dg,
// a1 = du, b0 = x.
template <typename T, typename OT, int FORM>
__global__ void __launch_bounds__(kThreads, 1)
gated_gemm_kernel(const __grid_constant__ CUtensorMap a0, const __grid_constant__ CUtensorMap a1,
                  const __grid_constant__ CUtensorMap b0, const __grid_constant__ CUtensorMap b1,
                  const __grid_constant__ GemmArgs p, int* __restrict__ status) {
    extern __shared__ uint8_t smem_raw[];
    uint8_t* stages = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);   // swizzled tiles need 1024-byte alignment
    GemmSmem* sm = reinterpret_cast<GemmSmem*>(stages + (size_t)kStages * kStageBytes);
    volatile int* abort_flag = &sm->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm->full[s], 1);
            mbar_init(&sm->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm->accum_full[b], 1);
            mbar_init(&sm->accum_empty[b], kEpiWarps);
        }
        sm->abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 0) tmem_alloc(&sm->tmem_base, kTmemCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sm->tmem_base;

    const int nkb = p.kb0 + p.kb1;
    const int64_t tiles = (int64_t)p.mt * p.nt;

    if (warp == 0) {
        if (lane == 0) {
            // ------------------------------------------------ copies
            int s = 0;
            uint32_t ph = 0;
            int64_t issued = 0;
            bool ok = true;
            for (int64_t tile = blockIdx.x; ok && tile < tiles; tile += gridDim.x) {
                const int m = (int)(tile % p.mt), n = (int)(tile / p.mt);
                for (int kb = 0; kb < nkb; ++kb) {
                    if (!mbar_wait(&sm->empty[s], ph ^ 1u, abort_flag, status)) { ok = false; break; }
                    uint8_t* a = stages + (size_t)s * kStageBytes;
                    uint8_t* b = a + kABytes;
                    uint64_t* bar = &sm->full[s];
                    mbar_expect_tx(bar, kStageBytes);
                    if constexpr (FORM == kForward || FORM == kRecompute) {
                        tma_load_2d(a, &a0, kb * kSlice, m * kTileM, bar);
                        tma_load_2d(b, &b0, kb * kSlice, n * 128, bar);
                        tma_load_2d(b + 128 * 128, &b1, kb * kSlice, n * 128, bar);
                    } else if constexpr (FORM == kDgrad) {
                        const bool second = kb >= p.kb0;
                        const int k = (second ? kb - p.kb0 : kb) * kSlice;
                        tma_load_2d(a, second ? &a1 : &a0, k, m * kTileM, bar);
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            tma_load_2d(b + c * kChunkBytes, second ? &b1 : &b0, n * kTileN + c * 64, k, bar);
                    } else {
                        const int half = p.mt / 2;
                        const bool second = m >= half;
                        const int row = (second ? m - half : m) * kTileM;
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            tma_load_2d(a + c * kChunkBytes, second ? &a1 : &a0, row + c * 64, kb * kSlice, bar);
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            tma_load_2d(b + c * kChunkBytes, &b0, n * kTileN + c * 64, kb * kSlice, bar);
                    }
                    ++issued;
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
            if (*abort_flag) {
                // give the copies still in flight a bounded time to land before the CTA goes away
                for (int64_t i = issued > kStages ? issued - kStages : 0; i < issued; ++i)
                    for (uint32_t spin = 0; spin < (1u << 16) && !mbar_test(&sm->full[i % kStages], (uint32_t)(i / kStages) & 1u); ++spin)
                        __nanosleep(64);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            // ------------------------------------------------ MMAs
            constexpr bool kAmn = FORM == kWgrad, kBmn = FORM == kDgrad || FORM == kWgrad;
            constexpr uint32_t fmt = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;   // A and B: fp16 or bf16
            constexpr uint32_t idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((kAmn ? 1u : 0u) << 15) | ((kBmn ? 1u : 0u) << 16) |
                                       ((uint32_t)(kTileN >> 3) << 17) | ((uint32_t)(kTileM >> 4) << 24);
            // 16 steps of the reduction: 32 bytes along a K-major row, 16 rows of an MN-major chunk
            constexpr uint64_t kAstep = kAmn ? 16 * 128 / 16 : 2, kBstep = kBmn ? 16 * 128 / 16 : 2;
            int s = 0, buf = 0;
            uint32_t ph = 0, aph = 0;
            bool ok = true;
            for (int64_t tile = blockIdx.x; ok && tile < tiles; tile += gridDim.x) {
                if (!mbar_wait(&sm->accum_empty[buf], aph ^ 1u, abort_flag, status)) break;
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(buf * kTileN);
                for (int kb = 0; kb < nkb; ++kb) {
                    if (!mbar_wait(&sm->full[s], ph, abort_flag, status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t addr = smem_u32(stages + (size_t)s * kStageBytes);
                    const uint64_t ad = kAmn ? smem_desc_mn(addr) : smem_desc(addr);
                    const uint64_t bd = kBmn ? smem_desc_mn(addr + kABytes) : smem_desc(addr + kABytes);
#pragma unroll
                    for (int kk = 0; kk < kSlice / 16; ++kk)
                        mma_f16(d, ad + kk * kAstep, bd + kk * kBstep, idesc, (kb | kk) != 0 ? 1u : 0u);
                    mma_commit(&sm->empty[s]);
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
                if (ok) mma_commit(&sm->accum_full[buf]);
                if (++buf == 2) { buf = 0; aph ^= 1u; }
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------- epilogue: a thread has one row of the tile
        const int part = warp & 3;   // the 32 accumulator lanes that this warp may read
        int buf = 0;
        uint32_t ph = 0;
        for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
            int m = (int)(tile % p.mt);
            const int n = (int)(tile / p.mt);
            if (!__all_sync(0xffffffffu, mbar_wait(&sm->accum_full[buf], ph, abort_flag, status))) break;
            tc_fence_after();
            const uint32_t at = tmem + ((uint32_t)(part * 32) << 16) + (uint32_t)(buf * kTileN);
            if constexpr (FORM == kForward || FORM == kRecompute) {
                const int64_t row = (int64_t)m * kTileM + part * 32 + lane, c0 = (int64_t)n * 128;
                const bool live = row < p.rows;
                float gmax = 0.f, umax = 0.f;
#pragma unroll 1
                for (int c = 0; c < 128; c += 32) {
                    float g[32], u[32];
                    tmem_load32(at + c, g);
                    tmem_load32(at + 128 + c, u);
                    if constexpr (FORM == kForward) {
                        if (p.gq) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                gmax = fmaxf(gmax, finite_abs(g[i]));
                                umax = fmaxf(umax, finite_abs(u[i]));
                            }
                        }
                        by_act(p.act, HOf<32>{g, u});
                        if (live) store32(static_cast<T*>(p.out0) + row * p.ldo, c0 + c, p.cols, p.out_vec, u);
                    } else if (live) {
                        float dh[32];
                        load32(static_cast<const T*>(p.dh) + row * p.lddh, c0 + c, p.cols, p.dh_vec, dh);
                        by_act(p.act, DguOf<32>{g, u, dh});
                        store32(static_cast<T*>(p.out0) + row * p.ldo, c0 + c, p.cols, true, g);
                        store32(static_cast<T*>(p.out1) + row * p.ldo, c0 + c, p.cols, true, u);
                    }
                }
                if (FORM == kForward && p.gq) {
                    const uint32_t ge = keep_exponent(gmax), ue = keep_exponent(umax);
                    const float ginv = keep_inverse(ge), uinv = keep_inverse(ue);
#pragma unroll 1
                    for (int c = 0; c < 128; c += 32) {
                        float f[32];
                        tmem_load32(at + c, f);
                        if (live) keep32(p.gq + row * p.ldq, c0 + c, p.cols, p.q_vec, ginv, f);
                        tmem_load32(at + 128 + c, f);
                        if (live) keep32(p.uq + row * p.ldq, c0 + c, p.cols, p.q_vec, uinv, f);
                    }
                    if (live) {
                        p.ge[row * p.lde + n] = (uint8_t)ge;
                        p.ue[row * p.lde + n] = (uint8_t)ue;
                    }
                }
            } else {
                void* out = p.out0;
                if (FORM == kWgrad && m >= p.mt / 2) { m -= p.mt / 2; out = p.out1; }
                const int64_t row = (int64_t)m * kTileM + part * 32 + lane, c0 = (int64_t)n * kTileN;
#pragma unroll 1
                for (int c = 0; c < kTileN; c += 32) {
                    float f[32];
                    tmem_load32(at + c, f);
                    if (row < p.rows) store32(static_cast<OT*>(out) + row * p.ldo, c0 + c, p.cols, p.out_vec, f);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm->accum_empty[buf]);
            if (++buf == 2) { buf = 0; ph ^= 1u; }
        }
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, kTmemCols);
}

// ---- dg and du from the kept g and u ------------------------------------------------------------
// One pass: dh, both 8-bit matrices with their scales in, dg and du out.  A thread has 8 columns of a row.
template <typename T>
__global__ void __launch_bounds__(256) dgu_kernel(const T* __restrict__ dH, int64_t lddh, bool dh_vec,
                                                  const uint8_t* __restrict__ GQ, const uint8_t* __restrict__ GE,
                                                  const uint8_t* __restrict__ UQ, const uint8_t* __restrict__ UE, int64_t ldq,
                                                  int64_t lde, bool q_vec, int act, int64_t rows, int64_t cols,
                                                  T* __restrict__ dG, T* __restrict__ dU, int64_t ldo) {
    const int64_t per_row = (cols + 7) / 8;
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    int64_t item = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    int64_t row = item / per_row, k = item % per_row;
    const int64_t drow = stride / per_row, dk = stride % per_row;
    while (row < rows) {
        const int64_t c = k * 8;
        const bool full = c + 8 <= cols;
        float dh[8], g[8], u[8];
        if (full && dh_vec) {
            Piece<T>::split(ld_stream_u4(dH + row * lddh + c), dh);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) dh[i] = c + i < cols ? to_f32(dH[row * lddh + c + i]) : 0.f;
        }
        uint2 gq = make_uint2(0u, 0u), uq = make_uint2(0u, 0u);
        if (full && q_vec) {
            gq = __ldcs(reinterpret_cast<const uint2*>(GQ + row * ldq + c));
            uq = __ldcs(reinterpret_cast<const uint2*>(UQ + row * ldq + c));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (c + i < cols) {
                    const uint32_t a = (uint32_t)GQ[row * ldq + c + i] << (8 * (i % 4)), b = (uint32_t)UQ[row * ldq + c + i] << (8 * (i % 4));
                    if (i < 4) { gq.x |= a; uq.x |= b; } else { gq.y |= a; uq.y |= b; }
                }
            }
        }
        const float gs = keep_scale_of_byte(GE[row * lde + c / kKeepBlock]), us = keep_scale_of_byte(UE[row * lde + c / kKeepBlock]);
        float f[4];
        taken4(gq.x, f);
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = f[i] * gs;
        taken4(gq.y, f);
#pragma unroll
        for (int i = 0; i < 4; ++i) g[4 + i] = f[i] * gs;
        taken4(uq.x, f);
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = f[i] * us;
        taken4(uq.y, f);
#pragma unroll
        for (int i = 0; i < 4; ++i) u[4 + i] = f[i] * us;
        by_act(act, DguOf<8>{g, u, dh});
        // (the workspace rows are padded to whole pieces)
        *reinterpret_cast<uint4*>(dG + row * ldo + c) = Piece<T>::join(g);
        *reinterpret_cast<uint4*>(dU + row * ldo + c) = Piece<T>::join(u);
        row += drow;
        k += dk;
        if (k >= per_row) { k -= per_row; ++row; }
    }
}

// A matrix that TMA cannot address, copied to 16-byte aligned rows.
__global__ void __launch_bounds__(256) align_rows_kernel(const uint16_t* __restrict__ X, int64_t ld, int64_t rows,
                                                         int64_t cols, uint16_t* __restrict__ Y, int64_t ldy) {
    const int64_t per_row = (cols + 7) / 8;
    const int64_t stride = (int64_t)gridDim.x * blockDim.x;
    int64_t item = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    int64_t row = item / per_row, k = item % per_row;
    const int64_t drow = stride / per_row, dk = stride % per_row;
    while (row < rows) {
        const int64_t c = k * 8;
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = c + 2 * i < cols ? X[row * ld + c + 2 * i] : 0u, hi = c + 2 * i + 1 < cols ? X[row * ld + c + 2 * i + 1] : 0u;
            v[i] = lo | (hi << 16);
        }
        *reinterpret_cast<uint4*>(Y + row * ldy + c) = make_uint4(v[0], v[1], v[2], v[3]);
        row += drow;
        k += dk;
        if (k >= per_row) { k -= per_row; ++row; }
    }
}

// ---- host ---------------------------------------------------------------------------------------
struct Mat {
    const void* p;
    int64_t ld;
};

bool tma_ok(const void* p, int64_t ld) { return aligned16(p) && ld % 8 == 0; }
int64_t padded(int64_t cols) { return (cols + 63) / 64 * 64; }

// The workspace: status word | aligned copies where TMA needs them (x also when it comes in 8 bits) | dg | du
struct GatedPlan {
    bool copy_x, copy_wg, copy_wu;
    size_t x, wg, wu, dg, du, total;
};
GatedPlan gated_plan(const detox_gated_desc& g, bool backward) {
    GatedPlan q;
    size_t off = 256;
    auto take = [&](bool want, int64_t rows, int64_t cols) {
        const size_t at = off;
        if (want) off += align_up((size_t)rows * (size_t)padded(cols) * 2);
        return at;
    };
    q.copy_x = !g.X || !tma_ok(g.X, g.ldx);
    q.copy_wg = !tma_ok(g.Wg, g.ldwg);
    q.copy_wu = !tma_ok(g.Wu, g.ldwu);
    q.x = take(q.copy_x, g.tokens, g.in_dim);
    q.wg = take(q.copy_wg, g.hidden, g.in_dim);
    q.wu = take(q.copy_wu, g.hidden, g.in_dim);
    q.dg = take(backward, g.tokens, g.hidden);
    q.du = take(backward, g.tokens, g.hidden);
    q.total = off;
    return q;
}

unsigned items_grid(int64_t items) {
    const int64_t need = ceil_div(items, (int64_t)256), most = (int64_t)kSMs * 8;
    return (unsigned)(need < most ? need : most);
}

detox_status aligned_copy(const void* X, int64_t ld, int64_t rows, int64_t cols, void* to, Mat* out, cudaStream_t s) {
    align_rows_kernel<<<items_grid(rows * ceil_div(cols, (int64_t)8)), 256, 0, s>>>(
        static_cast<const uint16_t*>(X), ld, rows, cols, static_cast<uint16_t*>(to), padded(cols));
    *out = Mat{to, padded(cols)};
    return launch_status();
}

detox_status input_matrix(const detox_gated_desc& g, const GatedPlan& q, char* ws, Mat* out, cudaStream_t s) {
    if (!q.copy_x) {
        *out = Mat{g.X, g.ldx};
        return DETOX_OK;
    }
    if (g.X) return aligned_copy(g.X, g.ldx, g.tokens, g.in_dim, ws + q.x, out, s);
    *out = Mat{ws + q.x, padded(g.in_dim)};
    return launch_checkpoint_unpack(g.dtype, g.XQ, g.ldxq, g.XE, g.ldxe, g.tokens, g.in_dim, ws + q.x, padded(g.in_dim), s);
}
detox_status weight_matrices(const detox_gated_desc& g, const GatedPlan& q, char* ws, Mat* wg, Mat* wu, cudaStream_t s) {
    *wg = Mat{g.Wg, g.ldwg};
    *wu = Mat{g.Wu, g.ldwu};
    if (q.copy_wg) {
        const detox_status st = aligned_copy(g.Wg, g.ldwg, g.hidden, g.in_dim, ws + q.wg, wg, s);
        if (st != DETOX_OK) return st;
    }
    if (q.copy_wu) return aligned_copy(g.Wu, g.ldwu, g.hidden, g.in_dim, ws + q.wu, wu, s);
    return DETOX_OK;
}

// One product: maps, grid, launch.  Each map's matrix is rows x cols with boxes of `box` rows.
struct MapOf {
    Mat m;
    int64_t rows, cols;
    int box;
};
template <typename T, typename OT, int FORM>
detox_status launch_gemm(const MapOf& a0, const MapOf& a1, const MapOf& b0, const MapOf& b1, const GemmArgs& args, int* status,
                         cudaStream_t s) {
    CUtensorMap maps[4];
    const MapOf* of[4] = {&a0, &a1, &b0, &b1};
    for (int i = 0; i < 4; ++i) {
        const detox_status st = make_map_16bit(&maps[i], std::is_same<T, __nv_bfloat16>::value, of[i]->m.p, of[i]->m.ld, of[i]->rows,
                                               of[i]->cols, of[i]->box);
        if (st != DETOX_OK) return st;
    }
    auto* k = gated_gemm_kernel<T, OT, FORM>;
    if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes) != cudaSuccess) return DETOX_ERR_CUDA;
    const int64_t tiles = (int64_t)args.mt * args.nt;
    k<<<(unsigned)(tiles < kSMs ? tiles : kSMs), kThreads, kSmemBytes, s>>>(maps[0], maps[1], maps[2], maps[3], args, status);
    return launch_status();
}

template <typename T>
detox_status forward(const detox_gated_desc& g, void* H, int64_t ldh, char* ws, cudaStream_t s) {
    const GatedPlan q = gated_plan(g, false);
    int* status = reinterpret_cast<int*>(ws);
    if (cudaMemsetAsync(status, 0, sizeof(int), s) != cudaSuccess) return DETOX_ERR_CUDA;
    Mat x, wg, wu;
    detox_status st = input_matrix(g, q, ws, &x, s);
    if (st == DETOX_OK) st = weight_matrices(g, q, ws, &wg, &wu, s);
    if (st != DETOX_OK) return st;
    GemmArgs a{};
    a.mt = (int)ceil_div(g.tokens, (int64_t)kTileM);
    a.nt = (int)ceil_div(g.hidden, (int64_t)128);
    a.kb0 = (int)ceil_div(g.in_dim, (int64_t)kSlice);
    a.act = g.act;
    a.rows = g.tokens;
    a.cols = g.hidden;
    a.out0 = H;
    a.ldo = ldh;
    a.out_vec = tma_ok(H, ldh);
    a.gq = g.GQ; a.ge = g.GE; a.uq = g.UQ; a.ue = g.UE;
    a.ldq = g.ldq; a.lde = g.lde;
    a.q_vec = aligned16(g.GQ) && aligned16(g.UQ) && g.ldq % 16 == 0;
    const MapOf mx{x, g.tokens, g.in_dim, 128}, mg{wg, g.hidden, g.in_dim, 128}, mu{wu, g.hidden, g.in_dim, 128};
    return launch_gemm<T, T, kForward>(mx, mx, mg, mu, a, status, s);
}

template <typename T, typename OT>
detox_status weight_gradients(const detox_gated_desc& g, const Mat& dg, const Mat& du, const Mat& x, void* dWg, void* dWu,
                              int64_t lddw, int* status, cudaStream_t s) {
    GemmArgs a{};
    a.mt = 2 * (int)ceil_div(g.hidden, (int64_t)kTileM);
    a.nt = (int)ceil_div(g.in_dim, (int64_t)kTileN);
    a.kb0 = (int)ceil_div(g.tokens, (int64_t)kSlice);
    a.rows = g.hidden;
    a.cols = g.in_dim;
    a.out0 = dWg;
    a.out1 = dWu;
    a.ldo = lddw;
    a.out_vec = aligned16(dWg) && aligned16(dWu) && lddw % Piece<OT>::N == 0;
    const MapOf mg{dg, g.tokens, g.hidden, 64}, mu{du, g.tokens, g.hidden, 64}, mx{x, g.tokens, g.in_dim, 64};
    return launch_gemm<T, OT, kWgrad>(mg, mu, mx, mx, a, status, s);
}

template <typename T>
detox_status backward(const detox_gated_desc& g, const void* dH, int64_t lddh, void* dX, int64_t lddx, void* dWg, void* dWu,
                      int64_t lddw, int dw_dtype, char* ws, cudaStream_t s) {
    const GatedPlan q = gated_plan(g, true);
    int* status = reinterpret_cast<int*>(ws);
    if (cudaMemsetAsync(status, 0, sizeof(int), s) != cudaSuccess) return DETOX_ERR_CUDA;
    const bool kept = g.GQ != nullptr;
    const int64_t ldf = padded(g.hidden);
    const Mat dg{ws + q.dg, ldf}, du{ws + q.du, ldf};
    Mat x{nullptr, 0}, wg{nullptr, 0}, wu{nullptr, 0};
    detox_status st = DETOX_OK;
    if (dWg || !kept) st = input_matrix(g, q, ws, &x, s);
    if (st == DETOX_OK && (dX || !kept)) st = weight_matrices(g, q, ws, &wg, &wu, s);
    if (st != DETOX_OK) return st;
    if (kept) {
        const bool q_vec = aligned_to(g.GQ, 8) && aligned_to(g.UQ, 8) && g.ldq % 8 == 0;
        dgu_kernel<T><<<items_grid(g.tokens * ceil_div(g.hidden, (int64_t)8)), 256, 0, s>>>(
            static_cast<const T*>(dH), lddh, tma_ok(dH, lddh), g.GQ, g.GE, g.UQ, g.UE, g.ldq, g.lde, q_vec, g.act, g.tokens,
            g.hidden, static_cast<T*>(const_cast<void*>(dg.p)), static_cast<T*>(const_cast<void*>(du.p)), ldf);
        st = launch_status();
    } else {
        GemmArgs a{};
        a.mt = (int)ceil_div(g.tokens, (int64_t)kTileM);
        a.nt = (int)ceil_div(g.hidden, (int64_t)128);
        a.kb0 = (int)ceil_div(g.in_dim, (int64_t)kSlice);
        a.act = g.act;
        a.rows = g.tokens;
        a.cols = g.hidden;
        a.out0 = const_cast<void*>(dg.p);
        a.out1 = const_cast<void*>(du.p);
        a.ldo = ldf;
        a.dh = dH;
        a.lddh = lddh;
        a.dh_vec = tma_ok(dH, lddh);
        const MapOf mx{x, g.tokens, g.in_dim, 128}, mg{wg, g.hidden, g.in_dim, 128}, mu{wu, g.hidden, g.in_dim, 128};
        st = launch_gemm<T, T, kRecompute>(mx, mx, mg, mu, a, status, s);
    }
    if (st != DETOX_OK) return st;
    if (dX) {
        GemmArgs a{};
        a.mt = (int)ceil_div(g.tokens, (int64_t)kTileM);
        a.nt = (int)ceil_div(g.in_dim, (int64_t)kTileN);
        a.kb0 = a.kb1 = (int)ceil_div(g.hidden, (int64_t)kSlice);
        a.rows = g.tokens;
        a.cols = g.in_dim;
        a.out0 = dX;
        a.ldo = lddx;
        a.out_vec = tma_ok(dX, lddx);
        const MapOf mdg{dg, g.tokens, g.hidden, 128}, mdu{du, g.tokens, g.hidden, 128};
        const MapOf mg{wg, g.hidden, g.in_dim, 64}, mu{wu, g.hidden, g.in_dim, 64};
        st = launch_gemm<T, T, kDgrad>(mdg, mdu, mg, mu, a, status, s);
        if (st != DETOX_OK) return st;
    }
    if (!dWg) return DETOX_OK;
    if (dw_dtype == DETOX_DTYPE_FLOAT) return weight_gradients<T, float>(g, dg, du, x, dWg, dWu, lddw, status, s);
    return weight_gradients<T, T>(g, dg, du, x, dWg, dWu, lddw, status, s);
}

}  // namespace

size_t gated_ws_bytes(const detox_gated_desc& g) { return gated_plan(g, false).total; }
size_t gated_backward_ws_bytes(const detox_gated_desc& g) { return gated_plan(g, true).total; }

detox_status launch_gated(const detox_gated_desc& g, void* H, int64_t ldh, void* ws, cudaStream_t s) {
    if (g.tokens == 0) return cudaMemsetAsync(ws, 0, sizeof(int), s) == cudaSuccess ? DETOX_OK : DETOX_ERR_CUDA;
    if (g.dtype == DETOX_DTYPE_HALF) return forward<__half>(g, H, ldh, static_cast<char*>(ws), s);
    return forward<__nv_bfloat16>(g, H, ldh, static_cast<char*>(ws), s);
}

detox_status launch_gated_backward(const detox_gated_desc& g, const void* dH, int64_t lddh, void* dX, int64_t lddx,
                                   void* dWg, void* dWu, int64_t lddw, int dw_dtype, void* ws, cudaStream_t s) {
    if (g.tokens == 0) {
        const size_t size = dw_dtype == DETOX_DTYPE_FLOAT ? 4 : 2;
        bool ok = cudaMemsetAsync(ws, 0, sizeof(int), s) == cudaSuccess;
        void* const dw[2] = {dWg, dWu};
        for (void* w : dw)
            if (w) ok = ok && cudaMemset2DAsync(w, (size_t)lddw * size, 0, (size_t)g.in_dim * size, (size_t)g.hidden, s) == cudaSuccess;
        return ok ? DETOX_OK : DETOX_ERR_CUDA;
    }
    if (g.dtype == DETOX_DTYPE_HALF)
        return backward<__half>(g, dH, lddh, dX, lddx, dWg, dWu, lddw, dw_dtype, static_cast<char*>(ws), s);
    return backward<__nv_bfloat16>(g, dH, lddh, dX, lddx, dWg, dWu, lddw, dw_dtype, static_cast<char*>(ws), s);
}

}  // namespace detox
