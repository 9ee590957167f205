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
// A CTA: one warp issues the TMA copies of 64-wide slices of both operands into a ring of stages, one thread issues
// the MMAs, eight warps drain the accumulator (two to each quarter of its rows).  Two accumulators share the tensor memory, so
// a tile is drained while the next one is multiplied.  Ragged edges: TMA fills with zeros outside a matrix and the epilogue
// masks its stores.
// Three shapes of the work (shape_of chooses):
//   pair     two CTAs of a cluster multiply one 256 x 256 tile (cta_group::2): each holds 128 rows of either operand, so
//            a byte of shared memory feeds twice the MMA work that a CTA on its own gets out of it; persistent grid
//   single   one CTA, 128 x 256 or 128 x 128; persistent grid
//   split    few tiles: the CTAs of a cluster take a share of one tile's reduction each, leave fp32 sums in shared memory
//            and then finish a share of its rows each, adding the others' sums over distributed shared memory in
//            the order of their ranks
//
// A pair's kernel runs alone: it is launched without overlap with the kernel before it, and lets none in before it ends.  While it
// took part in the chain of overlapping launches, steps of 8192 tokens stopped making progress about once in some thousand steps.
// No order of events in this code explains that; on their own, 80,000 such steps finished.  It costs nothing that shows in a step
// of 8192 tokens (0.97 ms either way) and 4 us in a backward pass of 1001 (70.9 -> 74.4, two pairs), so the other shapes stay chained.
//
// Every wait on a barrier is bounded (Waits below).  One that runs out ends its CTAs' work and leaves a record, the outputs of those
// CTAs become NaN, and the products that follow in the call give up at once.
#include <cuda.h>

#include <atomic>
#include <type_traits>

#include "gram_tc.cuh"
#include "tcgen05.cuh"
#include "worker.cuh"

namespace detox {

namespace {

enum Form { kForward = 0, kRecompute = 1, kDgrad = 2, kWgrad = 3 };

constexpr int kSlice = 64;                       // entries of the reduction per stage: one 128-byte swizzled row
constexpr uint32_t kChunkBytes = 64 * 128;       // 64 rows of 128 bytes
constexpr int kEpiWarps = 8, kThreads = 32 * (2 + kEpiWarps);
constexpr int kMaxSplit = 8;                     // CTAs of a portable cluster
constexpr int kMaxStages = 6;
constexpr int kRowBytes = 64, kRowPitch = 80, kWarpBuffer = 32 * kRowPitch;   // an epilogue warp's output rows, see flush_rows

// CG: CTAs that multiply one tile together.  BN: columns of the tile (forward, recompute: half of g, half of u).
template <int CG, int BN>
struct Tile {
    static constexpr int M = 128 * CG, N = BN;
    static constexpr int rows_b = BN / CG;                                    // rows of B that a CTA holds
    static constexpr uint32_t a_bytes = 128 * 128, b_bytes = rows_b * 128, stage_bytes = a_bytes + b_bytes;
    static constexpr int stages = stage_bytes > 32768 ? 4 : 6;
    static constexpr int tmem_cols = 2 * BN;
    static constexpr int pitch = BN + 4;                                      // floats between rows of a split's sums
};

struct GemmSmem {
    uint64_t full[kMaxStages];     // a stage's copies have landed (pair: both CTAs', counted at the first one)
    uint64_t empty[kMaxStages];    // the MMAs that read it are done
    uint64_t accum_full[2];        // an accumulator is complete
    uint64_t accum_empty[2];       // ... and drained (pair: by both CTAs, counted at the first one)
    uint32_t tmem_base;
    int abort_flag;
};
template <int CG, int BN>
constexpr size_t kSmemBytes = Tile<CG, BN>::stages * (size_t)Tile<CG, BN>::stage_bytes + kEpiWarps * kWarpBuffer + sizeof(GemmSmem) + 1024;
static_assert(kSmemBytes<2, 256> <= 227 * 1024 && kSmemBytes<1, 256> <= 227 * 1024 && kSmemBytes<1, 128> <= 227 * 1024, "fits an SM");
static_assert(128 * Tile<1, 256>::pitch * 4 <= Tile<1, 256>::stages * Tile<1, 256>::stage_bytes, "a split's sums fit the stages");
static_assert(128 * Tile<1, 128>::pitch * 4 <= Tile<1, 128>::stages * Tile<1, 128>::stage_bytes, "a split's sums fit the stages");

struct GemmArgs {
    int mt, nt;                    // output tiles (wgrad: mt counts those of dWg and of dWu)
    int kb0, kb1;                  // slices of the first and of the second product that are added up
    int split;                     // CTAs that share a tile's reduction
    bool clear_status;             // first kernel of the call that may set the status word; the later ones look at it
    long long wait_limit;          // SM clocks
    bool n_first;                  // neighbouring tiles lie along a row of the output (else along a column)
    int act;
    int64_t rows, cols;            // of the output (forward, recompute: of h)
    void* out0; void* out1;        // forward: h, -; recompute: dg, du; dgrad: dx, -; wgrad: dWg, dWu
    int64_t ldo;
    bool out_vec;                  // 16-byte stores
    uint8_t *gq, *ge, *uq, *ue;    // forward: the kept g and u, or null
    int64_t ldq, lde;
    bool q_vec;
    const void* dh;                // recompute (16-byte aligned rows)
    int64_t lddh;
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

// ---- bounded waits ------------------------------------------------------------------------------
enum Barrier { kEmpty = 0, kFull = 1, kAccumEmpty = 2, kAccumFull = 3 };
// Waits that ran out on this device, and what the first of them waited for: only the host clears it.
struct Expired {
    unsigned long long count;
    int32_t first[DETOX_EXPIRED_WORDS];   // form, CTAs of a tile's MMA, columns, split, rank, barrier, stage or accumulator, tile
};
__device__ Expired g_expired;
// (Out of line, like leave_nan below: what a product does not run should not lie between what it does.  48 tokens of 1024 -> 2816: 8.32 us,
// with both inline 8.42, without either 8.1; 500 of 512 -> 1408, a step: 38.3, 38.9 and 38.9.)
__device__ __noinline__ void note_expired(int* status, int form, int cg, int bn, int split, int rank, int which, int index, int tile) {
    if (atomicAdd(&g_expired.count, 1ull) == 0) {
        const int32_t what[DETOX_EXPIRED_WORDS] = {form, cg, bn, split, rank, which, index, tile};
#pragma unroll
        for (int i = 0; i < DETOX_EXPIRED_WORDS; ++i) g_expired.first[i] = what[i];
    }
    atomicExch(status, (int)DETOX_ERR_TIMEOUT);
}
struct Waits {
    int* abort_flag;               // this CTA's
    uint32_t peer_flag;            // the pair's other CTA's (an address in the cluster's shared memory), or 0
    int* status;
    long long limit;
    int form, cg, bn, split, rank;
    // False when the limit passed, or when another wait of this CTA or pair has already given up.
    __device__ __forceinline__ bool operator()(uint64_t* bar, uint32_t parity, Barrier which, int index, int64_t tile) const {
        if (mbar_try(bar, parity)) return true;
        const long long start = clock64();
        for (;;) {
            if (mbar_try(bar, parity)) return true;
            if (*static_cast<volatile int*>(abort_flag)) return false;
            if (clock64() - start > limit) break;
        }
        give_up();
        note_expired(status, form, cg, bn, split, rank, which, index, (int)tile);
        return false;
    }
    __device__ __forceinline__ void give_up() const {
        *static_cast<volatile int*>(abort_flag) = 1;
        if (peer_flag) asm volatile("st.shared::cluster.b32 [%0], %1;" ::"r"(peer_flag), "r"(1) : "memory");
    }
};
// Copies, MMAs and arrivals in flight end within microseconds; a CTA that has given up stays this long before it goes away, so that none
// of them meets the next kernel's shared memory.
__device__ __forceinline__ void let_flights_land() {
    const long long start = clock64();
    while (clock64() - start < 4000000) __nanosleep(1000);   // two milliseconds at the highest clock
}

// ---- the forms of the tcgen05 / cluster instructions that a pair of CTAs needs -------------------
template <int CG>
__device__ __forceinline__ void tmem_alloc_cg(uint32_t* slot, uint32_t ncols) {
    if constexpr (CG == 1) {
        tmem_alloc(slot, ncols);
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(ncols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CG>
__device__ __forceinline__ void tmem_dealloc_cg(uint32_t taddr, uint32_t ncols) {
    if constexpr (CG == 1) tmem_dealloc(taddr, ncols);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_f16_cg(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1) {
        mma_f16(tmem_d, adesc, bdesc, idesc, accumulate);
    } else {
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
            : "memory");
    }
}
// arrive on `bar` (pair: on the barrier at this place in both CTAs) once the MMAs issued so far have finished
template <int CG>
__device__ __forceinline__ void mma_commit_cg(uint64_t* bar) {
    if constexpr (CG == 1) mma_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
// the address, in the cluster's shared memory, of what lies at `addr` in the CTA of rank `rank`
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// 2-D TMA load into this CTA, completion counted on `bar`: a barrier of this CTA, or (pair) of the first CTA
template <int CG>
__device__ __forceinline__ void tma_load_cg(uint8_t* dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
            ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
            ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 ld_cluster_f2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

// kChunk columns of this thread's accumulator row, or two times as many.  Load and wait are one statement, so that nothing that
// uses the values can be moved between them.  Sixteen columns at a time: a CTA with one tile runs its epilogue once, and the
// longer a body is unrolled, the more of it goes into fetching instructions (a tile of 128 x 256: 2.6 us with 32, 2.1 with 16).
constexpr int kChunk = 16;
__device__ __forceinline__ void tmem_load(uint32_t at, float (&f)[kChunk]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]),
          "=f"(f[8]), "=f"(f[9]), "=f"(f[10]), "=f"(f[11]), "=f"(f[12]), "=f"(f[13]), "=f"(f[14]), "=f"(f[15])
        : "r"(at)
        : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t at_f, uint32_t at_g, float (&f)[kChunk], float (&g)[kChunk]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]),
          "=f"(f[8]), "=f"(f[9]), "=f"(f[10]), "=f"(f[11]), "=f"(f[12]), "=f"(f[13]), "=f"(f[14]), "=f"(f[15]),
          "=f"(g[0]), "=f"(g[1]), "=f"(g[2]), "=f"(g[3]), "=f"(g[4]), "=f"(g[5]), "=f"(g[6]), "=f"(g[7]),
          "=f"(g[8]), "=f"(g[9]), "=f"(g[10]), "=f"(g[11]), "=f"(g[12]), "=f"(g[13]), "=f"(g[14]), "=f"(g[15])
        : "r"(at_f), "r"(at_g)
        : "memory");
}

// ---- activations: a = act(g), da = act'(g) -----------------------------------------------------
// gelu: the normal distribution function and e = exp(-g^2 / 2).  For negative g it is small, and (1 + erf) / 2 would lose its bits
// there, 0.1% at -4 and all of them below -5.5.  With x = |g| and t = 1 / (1 + 0.3 x), the distribution function at -x is e R(x), and
// R(x) / t a polynomial in t: fitted to the least largest relative error over 0 <= x <= 14, 1.5e-7; with the arithmetic's own
// error 3e-6 of its size down to g = -8.  (erfcf is as good and made a step of 500 tokens 2.4 us of 38.6 slower.)
__device__ __forceinline__ float normal_cdf(float g, float& e) {
    const float x = fabsf(g), t = __fdividef(1.f, fmaf(0.3f, x, 1.f));
    e = __expf(-0.5f * x * x);
    float q = 0.035674829f;
    q = fmaf(q, t, -0.157203287f);
    q = fmaf(q, t, 0.206353813f);
    q = fmaf(q, t, -0.0536838956f);
    q = fmaf(q, t, 0.12856175f);
    q = fmaf(q, t, 0.099913463f);
    q = fmaf(q, t, 0.120753959f);
    q = fmaf(q, t, 0.119629301f);
    const float tail = e * (t * q);
    return g < 0.f ? tail : 1.f - tail;
}
template <int ACT>
__device__ __forceinline__ float act_of(float g) {
    if constexpr (ACT == DETOX_ACT_SILU) return __fdividef(g, 1.f + __expf(-g));
    if constexpr (ACT == DETOX_ACT_GELU) {
        float e;
        return g * normal_cdf(g, e);
    }
    return g < 0.f ? 0.f : g;   // (NaN stays NaN)
}
template <int ACT>
__device__ __forceinline__ void act_both(float g, float& a, float& da) {
    if constexpr (ACT == DETOX_ACT_SILU) {
        const float s = __fdividef(1.f, 1.f + __expf(-g));
        a = g * s;
        da = fmaf(a, 1.f - s, s);
    } else if constexpr (ACT == DETOX_ACT_GELU) {
        float e;
        const float c = normal_cdf(g, e);
        a = g * c;
        da = fmaf(g * 0.39894228f, e, c);
    } else {
        a = act_of<ACT>(g);
        da = g > 0.f ? 1.f : 0.f;
    }
}
// The same for two entries at a time.
template <int ACT>
__device__ __forceinline__ void act_both(uint64_t g, uint64_t& a, uint64_t& da) {
    if constexpr (ACT == DETOX_ACT_SILU) {
        const uint64_t one = pair_of(1.f, 1.f);
        const uint64_t s = pair_of(__fdividef(1.f, 1.f + __expf(-pair_lo(g))), __fdividef(1.f, 1.f + __expf(-pair_hi(g))));
        a = mul2(g, s);
        da = fma2(a, sub2(one, s), s);
    } else {
        float al, ah, dl, dh;
        act_both<ACT>(pair_lo(g), al, dl);
        act_both<ACT>(pair_hi(g), ah, dh);
        a = pair_of(al, ah);
        da = pair_of(dl, dh);
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

template <int NP>
struct DguPairsOf {   // the same on pairs
    uint64_t (&g)[NP];
    uint64_t (&u)[NP];
    const uint64_t (&dh)[NP];
    template <int ACT> __device__ __forceinline__ void operator()() {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            uint64_t a, da;
            act_both<ACT>(g[i], a, da);
            g[i] = mul2(mul2(dh[i], u[i]), da);
            u[i] = mul2(dh[i], a);
        }
    }
};

// ---- output rows through shared memory ------------------------------------------------------------
// A lane has a row of the accumulator, but 32 lanes that store 16 bytes each into 32 rows keep the load-store unit
// busy for 32 cycles.  So a warp collects 64 bytes of each of its 32 rows in shared memory (rows 80 bytes apart: eight
// lanes' 16-byte accesses meet no bank twice) and stores 8 rows of 64 bytes with one instruction.
__device__ __forceinline__ uint4* own_row(uint8_t* buf, int lane) { return reinterpret_cast<uint4*>(buf + lane * kRowPitch); }

// rows x cols: the part of `out` that exists, with the warp's first row at row 0 and the buffer's first column at column 0
template <typename OT>
__device__ __forceinline__ void flush_rows(uint8_t* buf, OT* out, int64_t ld, int64_t rows, int64_t cols, bool vec, int lane) {
    constexpr int W = kRowBytes / (int)sizeof(OT);
    __syncwarp();
    if (vec && cols >= W) {
        const int r0 = lane / 4, part = lane % 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + 8 * i;
            if (r < rows) {
                const uint4 v = *reinterpret_cast<const uint4*>(buf + r * kRowPitch + part * 16);
                *reinterpret_cast<uint4*>(out + r * ld + part * (W / 4)) = v;
            }
        }
    } else {
        const int n = (int)(rows < 32 ? rows : 32);
#pragma unroll 1
        for (int r = 0; r < n; ++r)
            for (int c = lane; c < W && c < cols; c += 32) out[r * ld + c] = reinterpret_cast<const OT*>(buf + r * kRowPitch)[c];
    }
    __syncwarp();
}
// the way in, for 16-byte aligned rows: entries beyond the matrix read as zeros
template <typename T>
__device__ __forceinline__ void fetch_rows(uint8_t* buf, const T* in, int64_t ld, int64_t rows, int64_t cols, int lane) {
    constexpr int N = Piece<T>::N;
    const int r0 = lane / 4, c = lane % 4 * N;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 8 * i;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows) {
            if (c + N <= cols) {
                v = *reinterpret_cast<const uint4*>(in + r * ld + c);
            } else {
                float f[N];
#pragma unroll
                for (int j = 0; j < N; ++j) f[j] = c + j < cols ? to_f32(in[r * ld + c + j]) : 0.f;
                v = Piece<T>::join(f);
            }
        }
        *reinterpret_cast<uint4*>(buf + r * kRowPitch + lane % 4 * 16) = v;
    }
    __syncwarp();
}
// kChunk entries as 16-byte pieces of a row, and kChunk 8-bit ones
template <typename OT>
__device__ __forceinline__ void put_chunk(uint4* to, const float (&f)[kChunk]) {
    constexpr int N = Piece<OT>::N;
#pragma unroll
    for (int i = 0; i < kChunk / N; ++i) {
        float p[N];
#pragma unroll
        for (int j = 0; j < N; ++j) p[j] = f[i * N + j];
        to[i] = Piece<OT>::join(p);
    }
}
__device__ __forceinline__ uint4 keep_chunk(bool odd, float inv, float (&f)[kChunk]) {
    uint32_t q[4];
    if (odd) {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) f[i] = inf_to_nan(f[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = keep4(f[4 * i] * inv, f[4 * i + 1] * inv, f[4 * i + 2] * inv, f[4 * i + 3] * inv);
    return make_uint4(q[0], q[1], q[2], q[3]);
}

// E consecutive entries of an output row (E = 2 or 4), as the lanes of a warp store a split's finished row
template <typename OT, int E>
__device__ __forceinline__ void store_few(OT* row, int64_t c, int64_t cols, bool vec, const float (&f)[E]) {
    if (vec && c + E <= cols) {
        if constexpr (sizeof(OT) == 2) {
            if constexpr (E == 4) *reinterpret_cast<uint2*>(row + c) = make_uint2(pack2<OT>(f[0], f[1]), pack2<OT>(f[2], f[3]));
            else *reinterpret_cast<uint32_t*>(row + c) = pack2<OT>(f[0], f[1]);
        } else {
            if constexpr (E == 4) *reinterpret_cast<float4*>(row + c) = make_float4(f[0], f[1], f[2], f[3]);
            else *reinterpret_cast<float2*>(row + c) = make_float2(f[0], f[1]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (c + i < cols) row[c + i] = from_f32<OT>(f[i]);
    }
}

// The end of a split: the CTA of rank `rank` finishes its share of the tile's rows.  A warp takes B of them at a time, a lane
// E columns of the tile's first half and E of the second; the S sums of an entry lie in the S CTAs' shared memory and are all
// asked for before the first is used (one round trip over the cluster's network), then added in the order of the ranks.
template <typename T, typename OT, int FORM, int BN, int S>
__device__ __forceinline__ void finish_split(const GemmArgs& p, int m, int n, uint32_t rank, uint32_t sums, int warp, int lane) {
    using TL = Tile<1, BN>;
    constexpr bool kGated = FORM == kForward || FORM == kRecompute;
    constexpr int kHalf = BN / 2, E = BN / 64, B = S <= 2 ? 4 : 2;
    void* out = p.out0;
    if (FORM == kWgrad && m >= p.mt / 2) { m -= p.mt / 2; out = p.out1; }
    const int64_t row0 = (int64_t)m * TL::M;
    const int live = (int)(p.rows - row0 < TL::M ? p.rows - row0 : TL::M);
    const int share = (live + S - 1) / S;
    const int last = (int)(rank + 1) * share < live ? (int)(rank + 1) * share : live;
    uint32_t from[S];
#pragma unroll
    for (int k = 0; k < S; ++k) from[k] = cluster_addr(sums, k) + (uint32_t)lane * (E * 4);
    for (int r0 = (int)rank * share + warp * B; r0 < last; r0 += kThreads / 32 * B) {
        float va[B][S][E], vb[B][S][E];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const uint32_t off = (uint32_t)(r0 + i < last ? r0 + i : r0) * (TL::pitch * 4);
#pragma unroll
            for (int k = 0; k < S; ++k) {
                if constexpr (E == 4) {
                    const float4 x = ld_cluster_f4(from[k] + off), y = ld_cluster_f4(from[k] + off + kHalf * 4);
                    va[i][k][0] = x.x; va[i][k][1] = x.y; va[i][k][2] = x.z; va[i][k][3] = x.w;
                    vb[i][k][0] = y.x; vb[i][k][1] = y.y; vb[i][k][2] = y.z; vb[i][k][3] = y.w;
                } else {
                    const float2 x = ld_cluster_f2(from[k] + off), y = ld_cluster_f2(from[k] + off + kHalf * 4);
                    va[i][k][0] = x.x; va[i][k][1] = x.y;
                    vb[i][k][0] = y.x; vb[i][k][1] = y.y;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < B; ++i) {
            if (r0 + i >= last) break;
            float a[E], b[E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                a[j] = va[i][0][j];
                b[j] = vb[i][0][j];
#pragma unroll
                for (int k = 1; k < S; ++k) { a[j] += va[i][k][j]; b[j] += vb[i][k][j]; }
            }
            const int64_t row = row0 + r0 + i;
            if constexpr (kGated) {
                const int64_t c = (int64_t)n * kHalf + lane * E;
                if constexpr (FORM == kForward) {
                    if (BN == 256 && p.gq) {
                        uint64_t ga[2] = {pair_of(a[0], a[1]), pair_of(a[E - 2], a[E - 1])};
                        uint64_t ub[2] = {pair_of(b[0], b[1]), pair_of(b[E - 2], b[E - 1])};
                        uint32_t gq[1], uq[1];
                        const uint32_t ge = keep_pairs<2, 32>(ga, gq), ue = keep_pairs<2, 32>(ub, uq);
                        if (p.q_vec && c + E <= p.cols) {
                            *reinterpret_cast<uint32_t*>(p.gq + row * p.ldq + c) = gq[0];
                            *reinterpret_cast<uint32_t*>(p.uq + row * p.ldq + c) = uq[0];
                        } else {
#pragma unroll
                            for (int j = 0; j < E; ++j)
                                if (c + j < p.cols) {
                                    p.gq[row * p.ldq + c + j] = (uint8_t)(gq[0] >> (8 * j));
                                    p.uq[row * p.ldq + c + j] = (uint8_t)(uq[0] >> (8 * j));
                                }
                        }
                        if (lane == 0) {
                            p.ge[row * p.lde + n] = (uint8_t)ge;
                            p.ue[row * p.lde + n] = (uint8_t)ue;
                        }
                    }
                    by_act(p.act, HOf<E>{a, b});
                    store_few<T, E>(static_cast<T*>(out) + row * p.ldo, c, p.cols, p.out_vec, b);
                } else {
                    float dh[E];
#pragma unroll
                    for (int j = 0; j < E; ++j)
                        dh[j] = c + j < p.cols ? to_f32(static_cast<const T*>(p.dh)[row * p.lddh + c + j]) : 0.f;
                    by_act(p.act, DguOf<E>{a, b, dh});
                    store_few<T, E>(static_cast<T*>(p.out0) + row * p.ldo, c, p.cols, true, a);
                    store_few<T, E>(static_cast<T*>(p.out1) + row * p.ldo, c, p.cols, true, b);
                }
            } else {
                const int64_t c = (int64_t)n * BN + lane * E;
                store_few<OT, E>(static_cast<OT*>(out) + row * p.ldo, c, p.cols, p.out_vec, a);
                store_few<OT, E>(static_cast<OT*>(out) + row * p.ldo, c + kHalf, p.cols, p.out_vec, b);
            }
        }
    }
}

// NaN in place of a tile that was given up, so that its outputs cannot be taken for results: all of it (split: every CTA of
// the cluster writes the same), or a pair's CTA its rows.
template <typename V>
__device__ __noinline__ void fill(V* out, int64_t ld, int64_t r0, int64_t r1, int64_t c0, int64_t c1, V value) {
    const int64_t cols = c1 - c0;
    for (int64_t i = threadIdx.x; i < (r1 - r0) * cols; i += kThreads) out[(r0 + i / cols) * ld + c0 + i % cols] = value;
}
template <typename T, typename OT, int FORM, int CG, int BN>
__device__ __noinline__ void leave_nan(const GemmArgs& p, int m, int n, uint32_t rank) {
    constexpr bool kGated = FORM == kForward || FORM == kRecompute;
    void* out = p.out0;
    if (FORM == kWgrad && m >= p.mt / 2) { m -= p.mt / 2; out = p.out1; }
    const int64_t r0 = (int64_t)m * Tile<CG, BN>::M + (CG == 2 ? (int)rank * 128 : 0), c0 = (int64_t)n * (kGated ? BN / 2 : BN);
    const int64_t r1 = r0 + 128 < p.rows ? r0 + 128 : p.rows, c1 = c0 + (kGated ? BN / 2 : BN) < p.cols ? c0 + (kGated ? BN / 2 : BN) : p.cols;
    if (r0 >= r1) return;
    if constexpr (sizeof(OT) == 4) fill<uint32_t>(static_cast<uint32_t*>(out), p.ldo, r0, r1, c0, c1, 0x7fffffffu);
    else fill<uint16_t>(static_cast<uint16_t*>(out), p.ldo, r0, r1, c0, c1, (uint16_t)0x7fff);   // (NaN in fp16 and in bf16)
    if (FORM == kRecompute) fill<uint16_t>(static_cast<uint16_t*>(p.out1), p.ldo, r0, r1, c0, c1, (uint16_t)0x7fff);
    if (FORM == kForward && BN == 256 && p.gq) {
        fill<uint8_t>(p.gq, p.ldq, r0, r1, c0, c1, (uint8_t)0x7f);
        fill<uint8_t>(p.uq, p.ldq, r0, r1, c0, c1, (uint8_t)0x7f);
        fill<uint8_t>(p.ge, p.lde, r0, r1, n, n + 1, (uint8_t)127);
        fill<uint8_t>(p.ue, p.lde, r0, r1, n, n + 1, (uint8_t)127);
    }
}

// Maps: forward, recompute: a0 = x, b0 = Wg, b1 = Wu; dgrad: a0 = dg, a1 = du, b0 = Wg, b1 = Wu; wgrad: a0 = dg,
// a1 = du, b0 = x.
template <typename T, typename OT, int FORM, int CG, int BN>
__global__ void __launch_bounds__(kThreads, 1)
gated_gemm_kernel(const __grid_constant__ CUtensorMap a0, const __grid_constant__ CUtensorMap a1,
                  const __grid_constant__ CUtensorMap b0, const __grid_constant__ CUtensorMap b1,
                  const __grid_constant__ GemmArgs p, int* __restrict__ status) {
    using TL = Tile<CG, BN>;
    constexpr int kStages = TL::stages;
    constexpr bool kGated = FORM == kForward || FORM == kRecompute;
    constexpr int kHalf = BN / 2;                    // columns of g (and of u) in a tile
    extern __shared__ uint8_t smem_raw[];
    uint8_t* stages = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);   // swizzled tiles need 1024-byte alignment
    uint8_t* buffers = stages + (size_t)kStages * TL::stage_bytes;
    GemmSmem* sm = reinterpret_cast<GemmSmem*>(buffers + kEpiWarps * kWarpBuffer);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 || p.split > 1 ? cluster_rank() : 0u;
    const Waits wait{&sm->abort_flag, CG == 2 ? cluster_addr(smem_u32(&sm->abort_flag), rank ^ 1u) : 0u, status, p.wait_limit,
                     FORM, CG, BN, p.split, (int)rank};

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&sm->full[s], 1);
            mbar_init(&sm->empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&sm->accum_full[b], 1);
            mbar_init(&sm->accum_empty[b], kEpiWarps * CG);
        }
        sm->abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 1) tmem_alloc_cg<CG>(&sm->tmem_base, TL::tmem_cols);
    tc_fence_before();
    if constexpr (CG == 2) {
        __syncthreads();
        cluster_sync();                              // the other CTA's barriers are there before anything arrives on them
    } else {
        // the copies need only the barriers, which their own warp has set up: they start without waiting for the others
        __syncwarp();
        if (warp == 0) asm volatile("bar.arrive 1, %0;" ::"n"(kThreads) : "memory");
        else asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
    }
    tc_fence_after();
    // The next kernel is let in only after this one's own wait, so by then all that came before this one is finished.
    pdl_wait();
    if constexpr (CG == 1) pdl_trigger();
    if (p.clear_status && blockIdx.x == 0 && threadIdx.x == 0) *status = 0;   // (a wait that runs out sets it far later)
    // A product whose operands an expired wait has left undone gives up at once.  (Warp 2 looks: its own first wait is long.)
    if (!p.clear_status && threadIdx.x == 64 && *static_cast<volatile int*>(status) != 0) wait.give_up();

    // A unit is the CTAs that work on a tile together: the pair, or the split's cluster; it takes every units-th tile.
    const int unit_ctas = CG == 2 ? 2 : p.split;
    const int64_t unit = blockIdx.x / unit_ctas, units = gridDim.x / unit_ctas;
    const int64_t tiles = (int64_t)p.mt * p.nt;
    const int nkb = p.kb0 + p.kb1;
    // this CTA's slices of the reduction
    const int kb_begin = CG == 2 ? 0 : (int)((int64_t)nkb * rank / p.split);
    const int kb_end = CG == 2 ? nkb : (int)((int64_t)nkb * (rank + 1) / p.split);
    auto place = [&](int64_t tile, int& m, int& n) {
        if (p.n_first) { n = (int)(tile % p.nt); m = (int)(tile / p.nt); }
        else { m = (int)(tile % p.mt); n = (int)(tile / p.mt); }
    };

    if (warp == 0) {
        if (lane == 0) {
            // ------------------------------------------------ copies
            const int cta_m = CG == 2 ? (int)rank * 128 : 0;          // first row of this CTA's part of A in the tile
            int s = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int64_t tile = unit; ok && tile < tiles; tile += units) {
                int m, n;
                place(tile, m, n);
                for (int kb = kb_begin; kb < kb_end; ++kb) {
                    if (!wait(&sm->empty[s], ph ^ 1u, kEmpty, s, tile)) { ok = false; break; }
                    uint8_t* a = stages + (size_t)s * TL::stage_bytes;
                    uint8_t* b = a + TL::a_bytes;
                    uint32_t bar = smem_u32(&sm->full[s]);
                    if constexpr (CG == 2) {
                        if (rank == 0) mbar_expect_tx(&sm->full[s], 2 * TL::stage_bytes);
                        bar = cluster_addr(bar, 0);
                    } else {
                        mbar_expect_tx(&sm->full[s], TL::stage_bytes);
                    }
                    if constexpr (kGated) {
                        tma_load_cg<CG>(a, &a0, kb * kSlice, m * TL::M + cta_m, bar);
                        if constexpr (CG == 2) {                       // the first CTA brings Wg, the second Wu
                            tma_load_cg<CG>(b, rank == 0 ? &b0 : &b1, kb * kSlice, n * kHalf, bar);
                        } else {
                            tma_load_cg<CG>(b, &b0, kb * kSlice, n * kHalf, bar);
                            tma_load_cg<CG>(b + kHalf * 128, &b1, kb * kSlice, n * kHalf, bar);
                        }
                    } else {
                        const int col = n * BN + (CG == 2 ? (int)rank * TL::rows_b : 0);
                        if constexpr (FORM == kDgrad) {
                            const bool second = kb >= p.kb0;
                            const int k = (second ? kb - p.kb0 : kb) * kSlice;
                            tma_load_cg<CG>(a, second ? &a1 : &a0, k, m * TL::M + cta_m, bar);
#pragma unroll
                            for (int c = 0; c < TL::rows_b / 64; ++c)
                                tma_load_cg<CG>(b + c * kChunkBytes, second ? &b1 : &b0, col + c * 64, k, bar);
                        } else {
                            const int half = p.mt / 2;
                            const bool second = m >= half;
                            const int row = (second ? m - half : m) * TL::M + cta_m;
#pragma unroll
                            for (int c = 0; c < 2; ++c)
                                tma_load_cg<CG>(a + c * kChunkBytes, second ? &a1 : &a0, row + c * 64, kb * kSlice, bar);
#pragma unroll
                            for (int c = 0; c < TL::rows_b / 64; ++c)
                                tma_load_cg<CG>(b + c * kChunkBytes, &b0, col + c * 64, kb * kSlice, bar);
                        }
                    }
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
            }
            // The last MMAs' arrivals have to land before this CTA goes away: they may come from the pair's other CTA, and the next
            // kernel's barriers lie at the same place.
            for (int i = 0; ok && i < kStages; ++i) {
                ok = wait(&sm->empty[s], ph ^ 1u, kEmpty, s, -1);
                if (++s == kStages) { s = 0; ph ^= 1u; }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && (CG == 1 || rank == 0)) {
            // ------------------------------------------------ MMAs
            constexpr bool kAmn = FORM == kWgrad, kBmn = FORM == kDgrad || FORM == kWgrad;
            constexpr uint32_t fmt = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;   // A and B: fp16 or bf16
            constexpr uint32_t idesc = (1u << 4) | (fmt << 7) | (fmt << 10) | ((kAmn ? 1u : 0u) << 15) | ((kBmn ? 1u : 0u) << 16) |
                                       ((uint32_t)(TL::N >> 3) << 17) | ((uint32_t)(TL::M >> 4) << 24);
            // 16 steps of the reduction: 32 bytes along a K-major row, 16 rows of an MN-major chunk
            constexpr uint64_t kAstep = kAmn ? 16 * 128 / 16 : 2, kBstep = kBmn ? 16 * 128 / 16 : 2;
            const uint32_t tmem = sm->tmem_base;
            int s = 0, buf = 0;
            uint32_t ph = 0, aph = 0;
            bool ok = true;
            for (int64_t tile = unit; ok && tile < tiles; tile += units) {
                if (!wait(&sm->accum_empty[buf], aph ^ 1u, kAccumEmpty, buf, tile)) { ok = false; break; }
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)(buf * BN);
                for (int kb = kb_begin; kb < kb_end; ++kb) {
                    if (!wait(&sm->full[s], ph, kFull, s, tile)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t addr = smem_u32(stages + (size_t)s * TL::stage_bytes);
                    const uint64_t ad = kAmn ? smem_desc_mn(addr) : smem_desc(addr);
                    const uint64_t bd = kBmn ? smem_desc_mn(addr + TL::a_bytes) : smem_desc(addr + TL::a_bytes);
#pragma unroll
                    for (int kk = 0; kk < kSlice / 16; ++kk)
                        mma_f16_cg<CG>(d, ad + kk * kAstep, bd + kk * kBstep, idesc, kb != kb_begin || kk != 0 ? 1u : 0u);
                    mma_commit_cg<CG>(&sm->empty[s]);
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
                if (ok) mma_commit_cg<CG>(&sm->accum_full[buf]);
                if (++buf == 2) { buf = 0; aph ^= 1u; }
            }
            // ... and so do the last accumulators' arrivals, from both CTAs' epilogues
            for (int i = 0; ok && i < 2; ++i) {
                ok = wait(&sm->accum_empty[buf], aph ^ 1u, kAccumEmpty, buf, -1);
                if (++buf == 2) { buf = 0; aph ^= 1u; }
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------- epilogue: a thread has one row of the tile
        const uint32_t tmem = sm->tmem_base;
        const int part = warp & 3, half = (warp - 2) >> 2;   // the 32 accumulator lanes that this warp may read; its columns
        uint8_t* buf = buffers + (warp - 2) * kWarpBuffer;
        int acc = 0;
        uint32_t ph = 0;
        for (int64_t tile = unit; tile < tiles; tile += units) {
            int m, n;
            place(tile, m, n);
            if (!__all_sync(0xffffffffu, wait(&sm->accum_full[acc], ph, kAccumFull, acc, tile))) break;
            tc_fence_after();
            const uint32_t at = tmem + ((uint32_t)(part * 32) << 16) + (uint32_t)(acc * BN);
            const int in_tile = (CG == 2 ? (int)rank * 128 : 0) + part * 32 + lane;
            if (CG == 1 && p.split > 1) {
                // (the one tile of this cluster, all its MMAs done: the stages are free to take the sums)
                const int m_out = FORM == kWgrad && m >= p.mt / 2 ? m - p.mt / 2 : m;
                float* row = reinterpret_cast<float*>(stages) + (size_t)in_tile * TL::pitch;
                const bool live = (int64_t)m_out * TL::M + in_tile < p.rows;
                const int c_end = __any_sync(0xffffffffu, live) ? (half + 1) * kHalf : 0;
#pragma unroll 1
                for (int c = half * kHalf; c < c_end; c += kChunk) {
                    float f[kChunk];
                    tmem_load(at + c, f);
                    if (live) {
#pragma unroll
                        for (int i = 0; i < kChunk / 4; ++i)
                            *reinterpret_cast<float4*>(row + c + 4 * i) = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
                    }
                }
            } else if constexpr (kGated) {
                const int64_t row0 = (int64_t)m * TL::M + in_tile - lane, c0 = (int64_t)n * kHalf;
                const int64_t rows = p.rows - row0;                                      // of this warp's that exist
                constexpr int kOwn = kHalf / 2, W = kRowBytes / (int)sizeof(T);
#pragma unroll 1
                for (int c = half * kOwn; c < (half + 1) * kOwn; c += W) {               // this warp's columns of h
                    const int64_t col = c0 + c, cols = p.cols - col;
                    if constexpr (FORM == kForward) {
#pragma unroll 1
                        for (int k = 0; k < W; k += kChunk) {
                            float g[kChunk], u[kChunk];
                            tmem_load(at + c + k, at + kHalf + c + k, g, u);
                            by_act(p.act, HOf<kChunk>{g, u});
                            put_chunk<T>(own_row(buf, lane) + k / Piece<T>::N, u);
                        }
                        flush_rows(buf, static_cast<T*>(p.out0) + row0 * p.ldo + col, p.ldo, rows, cols, p.out_vec, lane);
                    } else {
                        fetch_rows(buf, static_cast<const T*>(p.dh) + row0 * p.lddh + col, p.lddh, rows, cols, lane);
                        uint4 du[kRowBytes / 16];
#pragma unroll
                        for (int k = 0; k < W; k += kChunk) {
                            float g[kChunk], u[kChunk], dh[kChunk];
                            uint4* mine = own_row(buf, lane) + k / Piece<T>::N;          // dh there becomes dg
#pragma unroll
                            for (int i = 0; i < kChunk / Piece<T>::N; ++i) {
                                float f[Piece<T>::N];
                                Piece<T>::split(mine[i], f);
#pragma unroll
                                for (int j = 0; j < Piece<T>::N; ++j) dh[i * Piece<T>::N + j] = f[j];
                            }
                            tmem_load(at + c + k, at + kHalf + c + k, g, u);
                            by_act(p.act, DguOf<kChunk>{g, u, dh});
                            put_chunk<T>(mine, g);
                            put_chunk<T>(du + k / Piece<T>::N, u);
                        }
                        flush_rows(buf, static_cast<T*>(p.out0) + row0 * p.ldo + col, p.ldo, rows, cols, true, lane);
#pragma unroll
                        for (int i = 0; i < kRowBytes / 16; ++i) own_row(buf, lane)[i] = du[i];
                        flush_rows(buf, static_cast<T*>(p.out1) + row0 * p.ldo + col, p.ldo, rows, cols, true, lane);
                    }
                }
                if (FORM == kForward && BN == 256 && p.gq) {
                    // half of the warps keep g, the others u: a thread finds the largest of its 128 entries, then converts them
                    const uint32_t from = at + half * kHalf;
                    float amax = 0.f;
#pragma unroll 1
                    for (int c = 0; c < kHalf; c += kChunk) {
                        float f[kChunk];
                        tmem_load(from + c, f);
#pragma unroll
                        for (int i = 0; i < kChunk; ++i) amax = fmaxf(amax, fabsf(f[i]));
                    }
                    const bool odd = __any_sync(0xffffffffu, is_inf(amax));   // an Inf somewhere: see keep_pairs
                    if (odd) {
                        amax = 0.f;
#pragma unroll 1
                        for (int c = 0; c < kHalf; c += kChunk) {
                            float f[kChunk];
                            tmem_load(from + c, f);
                            for (int i = 0; i < kChunk; ++i) amax = fmaxf(amax, fabsf(inf_to_nan(f[i])));
                        }
                    }
                    const uint32_t e = keep_exponent(amax);
                    const float inv = keep_inverse(e);
                    uint8_t* to = half ? p.uq : p.gq;
#pragma unroll 1
                    for (int c = 0; c < kHalf; c += kRowBytes) {
#pragma unroll 1
                        for (int k = 0; k < kRowBytes; k += kChunk) {
                            float f[kChunk];
                            tmem_load(from + c + k, f);
                            own_row(buf, lane)[k / kChunk] = keep_chunk(odd, inv, f);
                        }
                        flush_rows(buf, to + row0 * p.ldq + c0 + c, p.ldq, rows, p.cols - c0 - c, p.q_vec, lane);
                    }
                    if (lane < rows) (half ? p.ue : p.ge)[(row0 + lane) * p.lde + n] = (uint8_t)e;
                }
            } else {
                void* out = p.out0;
                if (FORM == kWgrad && m >= p.mt / 2) { m -= p.mt / 2; out = p.out1; }
                const int64_t row0 = (int64_t)m * TL::M + in_tile - lane, c0 = (int64_t)n * BN;
                constexpr int W = kRowBytes / (int)sizeof(OT);
#pragma unroll 1
                for (int c = half * kHalf; c < (half + 1) * kHalf; c += W) {
#pragma unroll 1
                    for (int k = 0; k < W; k += kChunk) {
                        float f[kChunk];
                        tmem_load(at + c + k, f);
                        put_chunk<OT>(own_row(buf, lane) + k / Piece<OT>::N, f);
                    }
                    flush_rows(buf, static_cast<OT*>(out) + row0 * p.ldo + c0 + c, p.ldo, p.rows - row0, p.cols - c0 - c, p.out_vec, lane);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (CG == 2) mbar_arrive_cluster(cluster_addr(smem_u32(&sm->accum_empty[acc]), 0));
                else mbar_arrive(&sm->accum_empty[acc]);
            }
            if (++acc == 2) { acc = 0; ph ^= 1u; }
        }
        __syncwarp();
    }

    // ---------------------------------------------------- the end
    tc_fence_before();
    __syncthreads();
    if (*static_cast<volatile int*>(&sm->abort_flag)) let_flights_land();
    __syncwarp();
    if (CG == 2 || p.split > 1) cluster_sync();      // all of the cluster's work is done, and no flag will be set any more
    bool gave_up = *static_cast<volatile int*>(&sm->abort_flag) != 0;
    if constexpr (CG == 1) {
        if (p.split > 1) {
            // the cluster's sums are added and the tile is finished (asked for here and used behind it: who gave up)
            const uint32_t flag = ld_cluster_u32(cluster_addr(smem_u32(&sm->abort_flag), lane < p.split ? lane : 0));
            int m, n;
            place(unit, m, n);
            const uint32_t sums = smem_u32(stages);
            if (p.split == 2) finish_split<T, OT, FORM, BN, 2>(p, m, n, rank, sums, warp, lane);
            else if (p.split == 3) finish_split<T, OT, FORM, BN, 3>(p, m, n, rank, sums, warp, lane);
            else if (p.split == 4) finish_split<T, OT, FORM, BN, 4>(p, m, n, rank, sums, warp, lane);
            else if (p.split == 6) finish_split<T, OT, FORM, BN, 6>(p, m, n, rank, sums, warp, lane);
            else finish_split<T, OT, FORM, BN, 8>(p, m, n, rank, sums, warp, lane);
            gave_up = __any_sync(0xffffffffu, flag != 0u);
            cluster_sync();                          // nobody leaves while its shared memory may still be reached
        }
    }
    if (gave_up) {
        for (int64_t tile = unit; tile < tiles; tile += units) {
            int m, n;
            place(tile, m, n);
            leave_nan<T, OT, FORM, CG, BN>(p, m, n, rank);
        }
    }
    if (warp == 1) tmem_dealloc_cg<CG>(sm->tmem_base, TL::tmem_cols);
}

// ---- what the backward pass lays out before its products -----------------------------------------
// dg and du from the kept g and u, in one pass: dh and both 8-bit matrices with their scales in, dg and du out; and,
// when the input comes in 8 bits, its entries for the weight gradients.
struct PrepareArgs {
    const void* dh; int64_t lddh;
    Span dh_span;
    const uint8_t *gq, *ge, *uq, *ue;
    int64_t ldq, lde;
    bool q_vec;
    int act;
    int64_t rows, cols;
    void *dg, *du;
    int64_t ldo;
    const uint8_t *xq, *xe;        // null: nothing to lay out
    int64_t ldxq, ldxe;
    bool xq_vec;
    int64_t x_cols;
    void* x; int64_t ldx;
};

// The pieces of `W` columns of a matrix, dealt to the threads of the grid; the row is carried along, not divided out.
template <int W>
struct Pieces {
    int64_t row, k, drow, dk, per_row;
    __device__ __forceinline__ explicit Pieces(int64_t cols) : per_row((cols + W - 1) / W) {
        const int64_t item = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, stride = (int64_t)gridDim.x * blockDim.x;
        row = item / per_row;
        k = item % per_row;
        drow = stride / per_row;
        dk = stride % per_row;
    }
    __device__ __forceinline__ void next() {
        row += drow;
        k += dk;
        if (k >= per_row) { k -= per_row; ++row; }
    }
};
constexpr int kWide = 16;   // columns of a thread: 16 bytes of the 8-bit form
// 16 bytes of a row of 8-bit entries, zeros beyond its end
__device__ __forceinline__ uint4 load_kept(const uint8_t* row, int64_t c, int64_t cols, bool vec) {
    if (vec && c + kWide <= cols) return ld_stream_u4(row + c);
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < kWide; ++i)
        if (c + i < cols) w[i / 4] |= (uint32_t)row[c + i] << (8 * (i % 4));
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void taken_pairs(uint4 q, uint8_t e, uint64_t (&p)[kWide / 2]) {
    const float scale = keep_scale_of_byte(e);
    const uint64_t scale2 = pair_of(scale, scale);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float f[4];
        taken4(w[i], f);
        p[2 * i] = mul2(pair_of(f[0], f[1]), scale2);
        p[2 * i + 1] = mul2(pair_of(f[2], f[3]), scale2);
    }
}
// two 16-byte pieces of a workspace row (padded to whole pieces)
template <typename T>
__device__ __forceinline__ void store_wide(T* to, const uint64_t (&p)[kWide / 2]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint64_t half[4] = {p[4 * k], p[4 * k + 1], p[4 * k + 2], p[4 * k + 3]};
        *reinterpret_cast<uint4*>(to + 8 * k) = Piece<T>::join(half);
    }
}

template <typename T>
__global__ void __launch_bounds__(256) gated_prepare_kernel(const __grid_constant__ PrepareArgs p) {
    pdl_trigger();
    pdl_wait();
    for (Pieces<kWide> it(p.cols); it.row < p.rows; it.next()) {
        const int64_t c = it.k * kWide;
        const T* dh_row = static_cast<const T*>(p.dh) + it.row * p.lddh;
        const int64_t at = it.row * p.ldq, block = it.row * p.lde + c / kKeepBlock;
        uint64_t dh[8], g[8], u[8];
        const uint4 gq = load_kept(p.gq + at, c, p.cols, p.q_vec), uq = load_kept(p.uq + at, c, p.cols, p.q_vec);
        const uint8_t ge = p.ge[block], ue = p.ue[block];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint64_t f[4];
            Piece<T>::split(load_piece<true>(dh_row, c + 8 * k, p.cols, p.dh_span), f);
#pragma unroll
            for (int i = 0; i < 4; ++i) dh[4 * k + i] = f[i];
        }
        taken_pairs(gq, ge, g);
        taken_pairs(uq, ue, u);
        by_act(p.act, DguPairsOf<8>{g, u, dh});
        store_wide(static_cast<T*>(p.dg) + it.row * p.ldo + c, g);
        store_wide(static_cast<T*>(p.du) + it.row * p.ldo + c, u);
    }
    if (!p.xq) return;
    for (Pieces<kWide> it(p.x_cols); it.row < p.rows; it.next()) {
        const int64_t c = it.k * kWide;
        uint64_t x[8];
        taken_pairs(load_kept(p.xq + it.row * p.ldxq, c, p.x_cols, p.xq_vec), p.xe[it.row * p.ldxe + c / kKeepBlock], x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = pair_of(taken_clamp<T>(pair_lo(x[i])), taken_clamp<T>(pair_hi(x[i])));
        store_wide(static_cast<T*>(p.x) + it.row * p.ldx + c, x);
    }
}

// Matrices whose rows are not 16-byte aligned, copied to rows that are (blockIdx.y says which).
constexpr int kMaxCopies = 4;
struct CopyArgs {
    const __half* from[kMaxCopies];                // (16-bit entries of either type)
    Span span[kMaxCopies];
    int64_t ld[kMaxCopies], rows[kMaxCopies], cols[kMaxCopies];
    uint16_t* to[kMaxCopies];
    int64_t ld_to[kMaxCopies];
};
__global__ void __launch_bounds__(256) align_rows_kernel(const __grid_constant__ CopyArgs p) {
    pdl_trigger();
    pdl_wait();
    const int which = blockIdx.y;
    const int64_t cols = p.cols[which];
    for (Pieces<8> it(cols); it.row < p.rows[which]; it.next()) {
        const int64_t c = it.k * 8;
        *reinterpret_cast<uint4*>(p.to[which] + it.row * p.ld_to[which] + c) =
            load_piece<true>(p.from[which] + it.row * p.ld[which], c, cols, p.span[which]);
    }
}

// ---- host ---------------------------------------------------------------------------------------
struct Mat {
    const void* p;
    int64_t ld;
};

bool tma_ok(const void* p, int64_t ld) { return aligned16(p) && ld % 8 == 0; }
int64_t padded(int64_t cols) { return (cols + 63) / 64 * 64; }

// The workspace: status word | aligned copies where a kernel needs them (x also when it comes in 8 bits) | dg | du
struct GatedPlan {
    bool copy_x, copy_wg, copy_wu;
    size_t x, wg, wu, dh, dg, du, total;
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
    q.dh = take(backward && !g.GQ, g.tokens, g.hidden);
    q.dg = take(backward, g.tokens, g.hidden);
    q.du = take(backward, g.tokens, g.hidden);
    q.total = off;
    return q;
}

unsigned items_grid(int64_t items) {
    const int64_t need = ceil_div(items, (int64_t)256), most = (int64_t)kSMs * 8;
    return (unsigned)(need < most ? need : most);
}

// The copies of a call, in one launch.
struct Copies {
    CopyArgs args{};
    int n = 0;
    int64_t items = 0;
    // `m` as it is, or where its copy will be
    Mat add(bool copy, const Mat& m, int64_t rows, int64_t cols, void* to) {
        if (!copy) return m;
        args.from[n] = static_cast<const __half*>(m.p);
        args.span[n] = span_of<__half>(m.p, m.ld, rows, cols);
        args.ld[n] = m.ld;
        args.rows[n] = rows;
        args.cols[n] = cols;
        args.to[n] = static_cast<uint16_t*>(to);
        args.ld_to[n] = padded(cols);
        const int64_t k = rows * ceil_div(cols, (int64_t)8);
        items = k > items ? k : items;
        ++n;
        return Mat{to, padded(cols)};
    }
    detox_status launch(cudaStream_t s) const {
        if (n == 0) return DETOX_OK;
        return launch_chained(align_rows_kernel, dim3(items_grid(items), (unsigned)n), 256, 0, 1, s, args);
    }
};
// x where the products can read it; an 8-bit x is laid out by a kernel of its own
detox_status input_matrix(const detox_gated_desc& g, const GatedPlan& q, char* ws, Copies* copies, Mat* out, cudaStream_t s) {
    if (g.X) {
        *out = copies->add(q.copy_x, Mat{g.X, g.ldx}, g.tokens, g.in_dim, ws + q.x);
        return DETOX_OK;
    }
    *out = Mat{ws + q.x, padded(g.in_dim)};
    return launch_checkpoint_unpack(g.dtype, g.XQ, g.ldxq, g.XE, g.ldxe, g.tokens, g.in_dim, ws + q.x, padded(g.in_dim), s);
}
void weight_matrices(const detox_gated_desc& g, const GatedPlan& q, char* ws, Copies* copies, Mat* wg, Mat* wu) {
    *wg = copies->add(q.copy_wg, Mat{g.Wg, g.ldwg}, g.hidden, g.in_dim, ws + q.wg);
    *wu = copies->add(q.copy_wu, Mat{g.Wu, g.ldwu}, g.hidden, g.in_dim, ws + q.wu);
}

// Which shape a product takes: the least of an estimate, in units of 10 ns, that was fitted to measurements of every shape on
// twenty problems from 1 to 8192 tokens, while pairs too were launched overlapping the kernel before.  (On the present code the shape it
// takes costs 3.3% more than the best one on average, 20% at worst, over the four products of eighteen of them.)
//   a slice of the reduction   pair 28, nearly the MMAs' own rate; 128 x 256 on one CTA 45, 128 x 128 27: a CTA takes in
//                  about 64 bytes a clock, and these need 48 and 32 KB a slice for 1/2 and 1/4 of a pair tile's work.
//                  With one row of tiles every byte of the weights comes from HBM for a single use, and the shapes differ
//                  little (36).
//   a tile's end   250 for 256 columns, half of it for 128; 100 more where g and u are kept, 100 more with a split,
//                  whose cluster meets
//   a launch       400
// The number of clusters that fit at once is that of a B200 (2 dies, GPCs of 14 to 20 SMs); it is a constant, so that
// every GPU takes the same shape and gives the same bits.
struct Shape {
    int cg, bn, split;
};
// `copies` outputs of rows x cols (forward and recompute: 2 x hidden columns), nkb slices each
struct Product {
    int64_t rows;
    int copies;
    int64_t cols;
    int nkb;
    bool keeps;        // leaves the 8-bit form, which needs a block of 128 columns in a tile
};
int64_t estimate(const Product& p, const Shape& s) {
    static const int kClusters[kMaxSplit + 1] = {0, 148, 74, 45, 33, 26, 22, 15, 15};
    const int64_t tiles = p.copies * ceil_div(p.rows, (int64_t)(128 * s.cg)) * ceil_div(p.cols, (int64_t)s.bn);
    const int slice = p.rows * p.copies <= 128 ? 36 : (s.cg == 2 ? 28 : (s.bn == 256 ? 45 : 27));
    const int64_t tile = ceil_div((int64_t)p.nkb, (int64_t)s.split) * slice + 250 * s.bn / 256 + (p.keeps ? 100 : 0) +
                         (s.split > 1 ? 100 : 0);
    return ceil_div(tiles, (int64_t)kClusters[s.cg * s.split]) * tile + 400;
}
template <typename F>
void each_shape(const Product& p, F f) {
    f(Shape{2, 256, 1});
    for (int split : {1, 2, 3, 4, 6, 8}) {   // (clusters of 5 and 7 leave more SMs idle than their neighbours)
        if (split > p.nkb) break;
        f(Shape{1, 256, split});
        if (!p.keeps) f(Shape{1, 128, split});
    }
}
Shape shape_of(const Product& p) {
    Shape best{2, 256, 1};
    int64_t least = INT64_MAX;
    each_shape(p, [&](const Shape& s) {
        const int64_t time = estimate(p, s);
        if (time < least) {
            least = time;
            best = s;
        }
    });
    return best;
}
std::atomic<long long> g_wait_limit{0};   // SM clocks; 0: by the length of the reduction
int slices(int64_t n) { return (int)ceil_div(n, (int64_t)kSlice); }
Product gated_product(const detox_gated_desc& g, bool keeps) { return Product{g.tokens, 1, 2 * g.hidden, slices(g.in_dim), keeps}; }

// One product: maps, grid, launch.  The matrices of the maps are rows x cols.
struct MapOf {
    Mat m;
    int64_t rows, cols;
};
template <typename T, typename OT, int FORM, int CG, int BN>
detox_status launch_shape(const MapOf& a0, const MapOf& a1, const MapOf& b0, const MapOf& b1, GemmArgs args, int split, int* status,
                          cudaStream_t s) {
    using TL = Tile<CG, BN>;
    constexpr bool kGated = FORM == kForward || FORM == kRecompute;
    // boxes of 64 columns: 128 rows of A and as many of the weights as a tile has columns of g, or 64 steps of the reduction
    const int box_a = FORM == kWgrad ? 64 : 128, box_b = kGated ? BN / 2 : 64;
    CUtensorMap maps[4] = {};
    const MapOf* of[4] = {&a0, &a1, &b0, &b1};
    for (int i = 0; i < 4; ++i) {
        if ((kGated && i == 1) || (FORM == kWgrad && i == 3)) continue;   // not read
        const detox_status st = make_map_16bit(&maps[i], std::is_same<T, __nv_bfloat16>::value, of[i]->m.p, of[i]->m.ld, of[i]->rows,
                                               of[i]->cols, i < 2 ? box_a : box_b);
        if (st != DETOX_OK) return st;
    }
    args.mt = (int)ceil_div(args.rows, (int64_t)TL::M) * (FORM == kWgrad ? 2 : 1);
    args.nt = (int)ceil_div(args.cols, (int64_t)(kGated ? BN / 2 : BN));
    args.split = split;
    // An accumulator takes some 900 clocks a slice at most; the limit is twenty times that, and a tenth of a second more.
    const long long limit = g_wait_limit.load();
    args.wait_limit = limit > 0 ? limit : 200000000LL + 20000LL * (args.kb0 + args.kb1);
    // The operand whose strips the neighbouring tiles share is read once; the other one is read again for every strip, and should
    // be the smaller one, which stays in L2.
    args.n_first = args.rows * (FORM == kWgrad ? 2 : 1) > args.cols * (kGated ? 2 : 1);
    auto* k = gated_gemm_kernel<T, OT, FORM, CG, BN>;
    if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes<CG, BN>) != cudaSuccess) return DETOX_ERR_CUDA;
    const int64_t tiles = (int64_t)args.mt * args.nt;
    const int unit = CG == 2 ? 2 : split;
    // a split's cluster finishes one tile; the others' grids are persistent
    const int64_t units = split > 1 || tiles < kSMs / unit ? tiles : kSMs / unit;
    return launch(CG == 1, k, (unsigned)(units * unit), kThreads, kSmemBytes<CG, BN>, (unsigned)unit, s, maps[0], maps[1], maps[2],
                  maps[3], args, status);
}
template <typename T, typename OT, int FORM>
detox_status launch_gemm(const MapOf& a0, const MapOf& a1, const MapOf& b0, const MapOf& b1, const GemmArgs& args, const Shape& sh,
                         int* status, cudaStream_t s) {
    if (sh.cg == 2) return launch_shape<T, OT, FORM, 2, 256>(a0, a1, b0, b1, args, 1, status, s);
    if (sh.bn == 256) return launch_shape<T, OT, FORM, 1, 256>(a0, a1, b0, b1, args, sh.split, status, s);
    return launch_shape<T, OT, FORM, 1, 128>(a0, a1, b0, b1, args, sh.split, status, s);
}

template <typename T>
detox_status forward(const detox_gated_desc& g, void* H, int64_t ldh, char* ws, cudaStream_t s) {
    const GatedPlan q = gated_plan(g, false);
    int* status = reinterpret_cast<int*>(ws);
    Mat x, wg, wu;
    Copies copies;
    detox_status st = input_matrix(g, q, ws, &copies, &x, s);
    weight_matrices(g, q, ws, &copies, &wg, &wu);
    if (st == DETOX_OK) st = copies.launch(s);
    if (st != DETOX_OK) return st;
    GemmArgs a{};
    a.clear_status = true;
    a.kb0 = slices(g.in_dim);
    a.act = g.act;
    a.rows = g.tokens;
    a.cols = g.hidden;
    a.out0 = H;
    a.ldo = ldh;
    a.out_vec = tma_ok(H, ldh);
    a.gq = g.GQ; a.ge = g.GE; a.uq = g.UQ; a.ue = g.UE;
    a.ldq = g.ldq; a.lde = g.lde;
    a.q_vec = aligned16(g.GQ) && aligned16(g.UQ) && g.ldq % 16 == 0;
    const MapOf mx{x, g.tokens, g.in_dim}, mg{wg, g.hidden, g.in_dim}, mu{wu, g.hidden, g.in_dim};
    return launch_gemm<T, T, kForward>(mx, mx, mg, mu, a, shape_of(gated_product(g, g.GQ != nullptr)), status, s);
}

template <typename T, typename OT>
detox_status weight_gradients(const detox_gated_desc& g, const Mat& dg, const Mat& du, const Mat& x, void* dWg, void* dWu,
                              int64_t lddw, bool clear_status, const Shape& shape, int* status, cudaStream_t s) {
    GemmArgs a{};
    a.clear_status = clear_status;
    a.kb0 = slices(g.tokens);
    a.rows = g.hidden;
    a.cols = g.in_dim;
    a.out0 = dWg;
    a.out1 = dWu;
    a.ldo = lddw;
    a.out_vec = aligned16(dWg) && aligned16(dWu) && lddw % Piece<OT>::N == 0;
    const MapOf mg{dg, g.tokens, g.hidden}, mu{du, g.tokens, g.hidden}, mx{x, g.tokens, g.in_dim};
    return launch_gemm<T, OT, kWgrad>(mg, mu, mx, mx, a, shape, status, s);
}

template <typename T>
detox_status backward(const detox_gated_desc& g, const void* dH, int64_t lddh, void* dX, int64_t lddx, void* dWg, void* dWu,
                      int64_t lddw, int dw_dtype, char* ws, cudaStream_t s) {
    const GatedPlan q = gated_plan(g, true);
    int* status = reinterpret_cast<int*>(ws);
    const bool kept = g.GQ != nullptr;
    const int64_t ldf = padded(g.hidden);
    const Mat dg{ws + q.dg, ldf}, du{ws + q.du, ldf};
    Mat x{nullptr, 0}, wg{nullptr, 0}, wu{nullptr, 0};
    detox_status st = DETOX_OK;
    Copies copies;
    const bool with_x = kept && !g.X && dWg;         // an 8-bit input, laid out in the pass that makes dg and du
    if (with_x) x = Mat{ws + q.x, padded(g.in_dim)};
    else if (dWg || !kept) st = input_matrix(g, q, ws, &copies, &x, s);
    if (dX || !kept) weight_matrices(g, q, ws, &copies, &wg, &wu);
    const Mat dh = copies.add(!kept && !tma_ok(dH, lddh), Mat{dH, lddh}, g.tokens, g.hidden, ws + q.dh);
    if (st == DETOX_OK) st = copies.launch(s);
    if (st != DETOX_OK) return st;
    if (kept) {
        PrepareArgs a{};
        a.dh = dH; a.lddh = lddh; a.dh_span = span_of<T>(dH, lddh, g.tokens, g.hidden);
        a.gq = g.GQ; a.ge = g.GE; a.uq = g.UQ; a.ue = g.UE;
        a.ldq = g.ldq; a.lde = g.lde;
        a.q_vec = aligned16(g.GQ) && aligned16(g.UQ) && g.ldq % 16 == 0;
        a.act = g.act;
        a.rows = g.tokens; a.cols = g.hidden;
        a.dg = const_cast<void*>(dg.p); a.du = const_cast<void*>(du.p); a.ldo = ldf;
        if (with_x) {
            a.xq = g.XQ; a.xe = g.XE; a.ldxq = g.ldxq; a.ldxe = g.ldxe;
            a.xq_vec = aligned16(g.XQ) && g.ldxq % 16 == 0;
            a.x_cols = g.in_dim;
            a.x = const_cast<void*>(x.p); a.ldx = x.ld;
        }
        st = launch_chained(gated_prepare_kernel<T>, items_grid(g.tokens * ceil_div(g.hidden, (int64_t)kWide)), 256, 0, 1, s, a);
    } else {
        GemmArgs a{};
        a.clear_status = true;
        a.kb0 = slices(g.in_dim);
        a.act = g.act;
        a.rows = g.tokens;
        a.cols = g.hidden;
        a.out0 = const_cast<void*>(dg.p);
        a.out1 = const_cast<void*>(du.p);
        a.ldo = ldf;
        a.dh = dh.p;
        a.lddh = dh.ld;
        const MapOf mx{x, g.tokens, g.in_dim}, mg{wg, g.hidden, g.in_dim}, mu{wu, g.hidden, g.in_dim};
        st = launch_gemm<T, T, kRecompute>(mx, mx, mg, mu, a, shape_of(gated_product(g, false)), status, s);
    }
    if (st != DETOX_OK) return st;
    const Product dx_product{g.tokens, 1, g.in_dim, 2 * slices(g.hidden), false};
    const Product dw_product{g.hidden, 2, g.in_dim, slices(g.tokens), false};
    if (dX) {
        GemmArgs a{};
        a.clear_status = kept;
        a.kb0 = a.kb1 = slices(g.hidden);
        a.rows = g.tokens;
        a.cols = g.in_dim;
        a.out0 = dX;
        a.ldo = lddx;
        a.out_vec = tma_ok(dX, lddx);
        const MapOf mdg{dg, g.tokens, g.hidden}, mdu{du, g.tokens, g.hidden};
        const MapOf mg{wg, g.hidden, g.in_dim}, mu{wu, g.hidden, g.in_dim};
        st = launch_gemm<T, T, kDgrad>(mdg, mdu, mg, mu, a, shape_of(dx_product), status, s);
        if (st != DETOX_OK) return st;
    }
    if (!dWg) return DETOX_OK;
    if (dw_dtype == DETOX_DTYPE_FLOAT) return weight_gradients<T, float>(g, dg, du, x, dWg, dWu, lddw, kept && !dX, shape_of(dw_product), status, s);
    return weight_gradients<T, T>(g, dg, du, x, dWg, dWu, lddw, kept && !dX, shape_of(dw_product), status, s);
}

}  // namespace

long long gated_wait_limit(long long clocks) {
    if (clocks != 0 && clocks < DETOX_WAIT_LIMIT_MIN) return g_wait_limit.load();
    return g_wait_limit.exchange(clocks);
}

unsigned long long gated_expired_waits(int32_t* first, bool clear) {
    Expired e;
    if (cudaMemcpyFromSymbol(&e, g_expired, sizeof(e)) != cudaSuccess) return ~0ull;
    for (int i = 0; first && i < DETOX_EXPIRED_WORDS; ++i) first[i] = e.count ? e.first[i] : -1;
    const Expired none{};
    if (clear && cudaMemcpyToSymbol(g_expired, &none, sizeof(none)) != cudaSuccess) return ~0ull;
    return e.count;
}

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
