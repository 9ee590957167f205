// Losses over logits: log-probabilities of chosen tokens, the clipped policy loss with a KL term, the preference loss of paired log ratios.
//
// Per row, with x = scale z log2(e):  lse = ln sum 2^x,  logp = (x_y - log2 sum) ln 2,  d loss / d z_j = c (1[j = y] - 2^x_j / sum).
// A sum leaves out the chosen entry: with q = sum over the others of 2^(x - x_y),  logp = -ln(1 + q)  and  1 - p_y = q / (1 + q)  keep their bits however sure
// of the token the row is (of 1 + q, q = 10^-9 would be lost).
// All of it is bound by HBM: the logits are the largest matrix of a training step, and the least is to read them once and write their
// gradient once.
//
//   policy_kernel    A cluster of 1 to 8 CTAs holds a row in registers.  Entries come in 16-byte pieces, each thread takes 2^(x - base), its base the next whole number
//                    from its largest x on, the pairs (base, sum) of all warps meet once a row (through distributed shared memory where there are several CTAs), and the
//                    gradient is the kept powers times one number a thread.  So the logits are read once, one power is taken of each entry (the
//                    special-function unit would be the bound with two), and a row has one barrier.  The next row's pieces are asked for as this
//                    one's are used up.  8192 x 32000 bf16, a tenth of the rows without a token: 180 to 189 us by machine, 5.3 to 5.5 TB/s (floor of what is read and written 152).  On clusters a full batch is far
//                    from that: 2048 x 128000 464 us (floor 160), 4096 x 64000 264; one CTA an SM, and the CTAs of a row wait for one another.
//   score_kernel     Log-probabilities alone: a warp, a CTA or a cluster goes through a row with a running base and sum.  2048 x 128000 bf16, all
//                    rows read: 93 to 103 us by machine, 5.1 to 5.6 TB/s (floor 80); the special-function unit is at 66 %, issue slots at 59 %.
//   backward_kernel  The gradient where lse is known: entry by entry.  The preference loss needs all of a pair's rows before any gradient, so it takes this
//                    second pass; it goes through the rows backwards, since the last ones that were read still lie in L2.  5510 x 32000 bf16: 102 us.
//   pairs_kernel     Sums over sequences, margins and the rows' gradients, a CTA a pair.
//   total_kernel     Sums of the CTAs' parts, in order.
#include <cmath>

#include "worker.cuh"

namespace detox {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxCluster = 8;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// ex2.approx is off by up to 1.4e-7 of itself, and comes out 5.0e-8 too small on average (2^20 arguments in each of (-24, -23] .. (-2, -1]: 4.9e-8 to 5.1e-8; in (-1, 0] 4.0e-8).
// Over the sums of a sequence's log-probabilities that adds up, so it is put right in the logarithm of a sum.  (As a factor of the sum it would be a unit of its last
// place or nothing.)  Powers are taken relative to whole numbers: the factors between sums are then powers of two, which have no error.
constexpr float kPowerShort = 5.0e-8f;
__device__ __forceinline__ float minus_inf() { return __int_as_float(0xff800000); }

// ---- clusters -------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_meet() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Another CTA's shared memory may be written only once that CTA has started, which being launched together does not say: every CTA tells it first and waits for the others
// before its first store.  (Two steps, so that the loads between them hide it; a CTA that has told waits on every path.)
__device__ __forceinline__ void cluster_tell_started() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait_started() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// two floats to the same place in another CTA's shared memory
__device__ __forceinline__ void store_at(const float2* here, uint32_t rank, float2 v) {
    uint32_t at = (uint32_t)__cvta_generic_to_shared(here), there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(v.x), "f"(v.y) : "memory");
}

// (base, sum of 2^(x - base)) of two sets, the base no less than the largest x; the empty set is (-Inf, 0)
__device__ __forceinline__ float2 joined(float2 a, float2 b) {
    const float m = a.x > b.x ? a.x : b.x;   // (NaN sums stay NaN whatever m is)
    const float m0 = m == minus_inf() ? 0.f : m;
    return make_float2(m, a.y * exp2_fast(a.x - m0) + b.y * exp2_fast(b.x - m0));
}

__device__ __forceinline__ float warp_largest(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float warp_total(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// the pairs of a warp's lanes as one, in all lanes
__device__ __forceinline__ float2 joined_warp(float2 a) {
    const float m = warp_largest(a.x), m0 = m == minus_inf() ? 0.f : m;
    return make_float2(m, warp_total(a.y * exp2_fast(a.x - m0)));
}

// 16 bytes, or what was there before; issued where it is written
__device__ __forceinline__ void load_if(uint4& v, const void* from, bool want) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t@p ld.global.cs.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}"
        : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w)
        : "l"(from), "r"((uint32_t)want)
        : "memory");
}
// the entries of a piece, rounded
template <typename T>
__device__ __forceinline__ void store_entries(T* row, int c, int cols, bool vec, const float (&f)[Piece<T>::N]) {
    constexpr int N = Piece<T>::N;
    if (vec && c + N <= cols) {
        st_stream_u4(row + c, Piece<T>::join(f));
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c + j < cols) row[c + j] = from_f32<T>(f[j]);
    }
}

// hi + lo, for what a row needs more than fp32's bits of: sums over a sequence add its log-probabilities up, and a ratio is formed of their difference to others.
struct Two {
    float hi, lo;
};
// (rounded products and sums by name where their roundings count: the compiler joins a * b + c into one otherwise)
__device__ __forceinline__ Two sum_of(float a, float b) {   // exactly
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return Two{s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two product_of(float a, float b) {   // exactly
    const float p = __fmul_rn(a, b);
    return Two{p, fmaf(a, b, -p)};
}
__device__ __forceinline__ double wide(Two v) { return (double)v.hi + (double)v.lo; }
constexpr float kLn2Rest = -1.9046543e-9f;             // ln 2 - kLn2
// scale log2(e) as hi + lo.  One fp32 number would be off by up to 2^-24 of itself, which is another temperature: the same way for every token of a sequence, and times the
// logits' size in a ratio.
struct Powers {
    float hi, lo;                  // powers of 2^(z hi + z lo - base), or, with lo = 0, of 2^(z hi - base);
    float rest;                    // then what lo would be, over hi, is what the distance from the largest entry to the chosen one lacks
};
// a sum of powers: its exponent and the logarithm of the rest, within 0.6 of 0
__device__ __forceinline__ void split_log2(float sum, float& exponent, float& rest) {
    const int bits = __float_as_int(sum), e = (bits - 0x3f400000) >> 23;
    exponent = (float)e;
    rest = log2f(__int_as_float(bits - (e << 23))) + (sum - sum);   // (NaN stays NaN)
}
// x of an entry.  Below -2^31 it is nothing: entries masked with some number.  From there on a product's rounding, and with it the exponent of a power that should be near 1, may
// be beyond 128 (masks of -10^10 or -10^20 made NaN of rows where a thread has no other entries), and the lowest numbers of bf16 and fp32 leave fp32's range.
constexpr float kFar = 2147483648.f;
__device__ __forceinline__ bool is_nothing(float x) { return x < -kFar; }

// The chosen token's log-probability, from its logit zy (NaN where there is no such token) and the sum of the others' powers of 2^(x - base).  What is below 2^-126 of the
// largest is nothing.
constexpr float kLeast = 1.17549435e-38f;
__device__ __forceinline__ Two logp_of(float base, float sum, float zy, Powers k2) {
    const Two x = product_of(zy, k2.hi);
    if (is_nothing(x.hi)) return Two{minus_inf() + (sum - sum), 0.f};   // (NaN stays NaN)
    if (sum < kLeast) return Two{x.hi - x.hi, 0.f};
    // log2 q = hi + lo
    const float low = x.lo + zy * k2.lo;
    float exponent, mantissa;
    split_log2(sum, exponent, mantissa);
    const Two d = sum_of(base, -x.hi), t = sum_of(d.hi, exponent);
    const float hi = t.hi, lo = d.lo + t.lo + (mantissa - low) + fmaf(d.hi, k2.rest, kPowerShort * kLog2e);
    const bool less = hi + lo <= 0.f;
    // of q, or of 1 / q: at most 1.  (Of distances that leave nothing of it, as to entries masked with -10^9, lo is not small either.)
    const float whole = exp2_fast(less ? hi : -hi), u = whole > 0.f ? whole * exp2_fast(less ? lo : -lo) : whole, l = log1pf(fmaf(u, 2.f * kPowerShort, u));
    const Two a = product_of(hi, kLn2);
    return less ? Two{-l, 0.f} : sum_of(-a.hi, -(a.lo + fmaf(hi, kLn2Rest, lo * kLn2) + l));
}

// 1 / x of a normal number, to a unit
__device__ __forceinline__ float inverse_of(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return fmaf(fmaf(-x, y, 1.f), y, y);
}
// 2^(hi + lo), lo what a rounding of hi's size has left: its square is left out (10^-6 of the power where logits have some 10^4).  Infinities of hi or of the result stay
__device__ __forceinline__ float power_of(float hi, float lo) {
    const float y = exp2_fast(hi);
    return fabsf(hi) < -minus_inf() ? fmaf(y < -minus_inf() ? y : 0.f, lo * kLn2, y) : y;
}
// v log2(e)
__device__ __forceinline__ Two in_powers(float v) {
    const Two p = product_of(v, kLog2e);
    return Two{p.hi, p.lo + v * 1.92596299e-8f};               // log2 e - kLog2e
}

// What all threads need of a row for its gradient, from (base, sum of the others' powers of 2^(x - base)).  With q = sum 2^(base - x_y) the token has p = 1 / (1 + q).
// The ratio p e^-old and e^ref / p are a power of two each, whose exponent is formed as hi + lo, without the logarithm of p: they are off by what the sum is off, a few
// units of 2^-23, and by nothing of the size of the logarithms.  (The same in 64 bits would cost 16 warps' worth of them a row.)
struct Chosen {
    float p;                       // p is this times 2^(at.hi + at.lo), which may lie outside of fp32's range
    float p_inverse;
    Two at;
    float rest;                    // 1 - p
    float share;                   // times 2^(x_j - base): p_j
    bool empty;                    // nothing but -Inf
};
__device__ __forceinline__ Chosen chosen_of(float2 all, float zy, Powers k2) {
    const Two product = product_of(zy, k2.hi);
    const bool nothing = is_nothing(product.hi), none = all.y < kLeast;
    const float x = nothing ? -2.f * kFar : product.hi, low = nothing ? 0.f : product.lo, sum = none ? 1.f : all.y;
    const int bits = __float_as_int(sum), e = (bits - 0x3f400000) >> 23;
    const float m = __int_as_float(bits - (e << 23)) + (sum - sum), m_inverse = inverse_of(m);   // within 0.75 .. 1.5; NaN stays NaN
    // q = m 2^(hi + lo)
    const Two d = sum_of(all.x == minus_inf() ? 0.f : all.x, -x), t = sum_of(none ? -2.f * kFar : d.hi, (float)e);
    const float hi = t.hi, lo = fmaf(nothing ? 0.f : d.hi, k2.rest, d.lo + t.lo - low + kPowerShort * kLog2e);
    const bool less = hi <= 0.f;
    const float power = exp2_fast(less ? hi : -hi);
    const float u = fmaf(power, fmaf(less ? lo : -lo, kLn2, kPowerShort), power) * (less ? m : m_inverse);   // q, or 1 / q
    const float inverse = inverse_of(1.f + u);
    Chosen c;
    c.p = less ? inverse : inverse * m_inverse;
    c.p_inverse = less ? 1.f + u : (1.f + u) * m;
    c.at = less ? Two{0.f, 0.f} : Two{-hi, -lo};
    c.rest = less ? u * inverse : inverse;
    c.share = c.rest * m_inverse * __int_as_float((127 - e) << 23);
    c.empty = nothing && none;
    return c;
}

// e^d - 1 - d, from e^d: near 0 by the series (the next term is 10^-7 of it at 1/2), where the difference would lose its bits
__device__ __forceinline__ float above_line(float d, float power) {
    float s = fmaf(d, 1.f / 40320.f, 1.f / 5040.f);
    s = fmaf(d, s, 1.f / 720.f);
    s = fmaf(d, s, 1.f / 120.f);
    s = fmaf(d, s, 1.f / 24.f);
    s = fmaf(d, s, 1.f / 6.f);
    s = d * d * fmaf(d, s, 0.5f);
    if (fabsf(d) < 0.5f) return s;
    return d == -minus_inf() ? d : (power - 1.f) - d;
}

// ---- the policy loss -------------------------------------------------------------------------------
struct RowsArgs {
    const void* Z;
    int64_t ldz;
    Span span;
    int64_t rows;
    int vocab, pieces, cluster;    // columns of a row; its pieces, which the CTAs of a cluster share
    const void* y;
    bool wide;                     // y in 64 bits
    Powers k2;                     // scale log2(e)
    int32_t zero;                  // 0, which the compiler does not know
    float* logp;
    const float *old_logp, *advantage, *ref_logp, *weight;
    float low, high, kl_coef, even_weight, grad_scale;   // grad_scale: times scale
    void* dZ;
    int64_t lddz;
    bool dz_vec;
    double* parts;                 // 4 for each cluster
};

__device__ __forceinline__ int64_t chosen(const void* y, bool wide, int64_t row) {
    return wide ? static_cast<const int64_t*>(y)[row] : (int64_t)static_cast<const int32_t*>(y)[row];
}

// The largest entry of pieces, two at a time where they are 16 bits wide (NaN is passed over).
template <typename T> struct Largest;
template <> struct Largest<float> {
    float m;
    __device__ __forceinline__ Largest() : m(minus_inf()) {}
    __device__ __forceinline__ void take(uint4 v) {
        m = fmaxf(fmaxf(m, fmaxf(__uint_as_float(v.x), __uint_as_float(v.y))), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    }
    __device__ __forceinline__ float value() const { return m; }
    static constexpr uint32_t kNone = 0xff800000u;             // -Inf
};
template <> struct Largest<__half> {
    uint32_t m = 0xfc00fc00u;
    __device__ __forceinline__ void take(uint4 v) { two(v.x); two(v.y); two(v.z); two(v.w); }
    __device__ __forceinline__ void two(uint32_t w) {
        const __half2 r = __hmax2(*reinterpret_cast<const __half2*>(&m), *reinterpret_cast<const __half2*>(&w));
        m = *reinterpret_cast<const uint32_t*>(&r);
    }
    __device__ __forceinline__ float value() const { const float2 f = unpack2<__half>(m); return fmaxf(f.x, f.y); }
    static constexpr uint32_t kNone = 0xfc00fc00u;
};
template <> struct Largest<__nv_bfloat16> {
    uint32_t m = 0xff80ff80u;
    __device__ __forceinline__ void take(uint4 v) { two(v.x); two(v.y); two(v.z); two(v.w); }
    __device__ __forceinline__ void two(uint32_t w) {
        const __nv_bfloat162 r = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&m), *reinterpret_cast<const __nv_bfloat162*>(&w));
        m = *reinterpret_cast<const uint32_t*>(&r);
    }
    __device__ __forceinline__ float value() const { const float2 f = unpack2<__nv_bfloat16>(m); return fmaxf(f.x, f.y); }
    static constexpr uint32_t kNone = 0xff80ff80u;
};
// what powers of entries up to z are taken relative to: the whole number from z's x on
__device__ __forceinline__ float base_of(float z, float k2) {
    const float x = z * k2;
    return is_nothing(x) ? minus_inf() : ceilf(x);
}
// a piece of which only the first `n` entries are in the row: -Inf for the others
template <typename T>
__device__ __forceinline__ uint4 only_first(uint4 v, int n) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            if (i >= n) w[i] = Largest<T>::kNone;
        } else {
            if (2 * i >= n) w[i] = Largest<T>::kNone;
            else if (2 * i + 1 >= n) w[i] = (w[i] & 0xffffu) | (Largest<T>::kNone & 0xffff0000u);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// the bits of entry j of a piece, and a piece with -Inf in the place of such bits
template <typename T>
__device__ __forceinline__ uint4 entry_mask(int j) {
    constexpr int A = 4 / (int)sizeof(T);                      // entries of a word
    const uint32_t bits = sizeof(T) == 4 ? 0xffffffffu : 0xffffu << (16 * (j & 1));
    return make_uint4(j / A == 0 ? bits : 0u, j / A == 1 ? bits : 0u, j / A == 2 ? bits : 0u, j / A == 3 ? bits : 0u);
}
template <typename T>
__device__ __forceinline__ uint4 hidden(uint4 v, uint4 m) {
    constexpr uint32_t none = sizeof(T) == 4 ? Largest<T>::kNone : (Largest<T>::kNone & 0xffffu) * 0x10001u;
    return make_uint4((v.x & ~m.x) | (none & m.x), (v.y & ~m.y) | (none & m.y), (v.z & ~m.z) | (none & m.z), (v.w & ~m.w) | (none & m.w));
}
// Registers: a thread holds P pieces of the next row (not AHEAD: of this one, and is done with them when it has the powers) and this row's
// powers in fp32.  16 pieces of fp32 leave no room for both.  Beside them a row's numbers: with one or two pieces these decide (9000 x 300 bf16, one piece: 41.6 us with 32 for them, 37.5 with
// 40; 20000 x 2050 at odd offsets, three: 140 and 157).
template <typename T, int P> constexpr bool kAhead = P * Piece<T>::N + 4 * P <= 96;
template <typename T, int P> constexpr int kRegisters = P * Piece<T>::N + (kAhead<T, P> ? 4 * P : 0) + (sizeof(T) == 4 ? 48 : 32) + (P <= 2 ? 8 : 0);
constexpr int between(int least, int most, int v) { return v < least ? least : (v > most ? most : v); }
template <typename T, int THREADS, int P> constexpr int kCtas = between(1, 2048 / THREADS, 65536 / (THREADS * kRegisters<T, P>));

// P pieces a thread; but for ANY the CTAs of a cluster have more than (P - 1) * THREADS each, so that only a thread's last one may be missing (a comparison and a
// branch for each piece took a third of the instructions).
template <typename T, int THREADS, int P, bool ANY>
__global__ void __launch_bounds__(THREADS, (kCtas<T, THREADS, P>)) policy_kernel(const __grid_constant__ RowsArgs g) {
    constexpr int N = Piece<T>::N, WARPS = THREADS / 32;
    constexpr bool AHEAD = kAhead<T, P>;
    constexpr int kTeller = THREADS - 32;      // who keeps the sums: in the warp that has the fewest pieces
    __shared__ float2 met[2][kMaxCluster * WARPS];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int cluster = g.cluster;
    const int rank = cluster > 1 ? (int)cluster_rank() : 0;
    const int64_t stride = gridDim.x / cluster;
    const int first = rank * g.pieces / cluster, pieces = (rank + 1) * g.pieces / cluster - first;
    const int begin = first * N;                              // this CTA's columns of a row
    const int cols = g.vocab - begin < pieces * N ? g.vocab - begin : pieces * N;
    if (cluster == 1) pdl_trigger();
    else cluster_tell_started();
    pdl_wait();
    int64_t row = blockIdx.x / cluster;
    const T* Z = static_cast<const T*>(g.Z);
    uint4 raw[P] = {};
    // whether thread's piece i is there
    auto there = [&](int i) { return (!ANY && i < P - 1) || (int)threadIdx.x + i * THREADS < pieces; };
    // a row's chosen token, -1 where the row does not count, and its weight
    auto look = [&](int64_t r, int64_t& token, float& weight) {
        token = -1;
        weight = 0.f;
        if (r >= g.rows) return;
        token = chosen(g.y, g.wide, r);
        weight = g.weight ? g.weight[r] : g.even_weight;
        if (weight == 0.f) token = -1;
    };
    auto fetch = [&](int i, const T* from, bool want, int behind = 0) {
        if constexpr (ANY) raw[i] = load_piece<true>(from, (int)(threadIdx.x + i * THREADS) * N + behind, want ? cols : 0, g.span);
        else load_if(raw[i], from + ((int)(threadIdx.x + i * THREADS) * N + behind), want && there(i));
    };
    int64_t y, next_y;
    float w, next_w;
    look(row, y, w);
    look(row + stride, next_y, next_w);
    if (AHEAD) {
#pragma unroll
        for (int i = 0; i < P; ++i) fetch(i, Z + row * g.ldz + begin, y >= 0);
    }
    double sum_loss = 0., sum_pg = 0., sum_kl = 0., sum_clip = 0.;
    int turn = 0;
    if (cluster > 1) cluster_wait_started();
    for (; row < g.rows; row += stride) {
        const int64_t next = row + stride;
        const T *here = Z + row * g.ldz + begin, *there_next = Z + next * g.ldz + begin;
        T* to = static_cast<T*>(g.dZ) + (g.dZ ? row * g.lddz + begin : 0);
        if (y < 0) {                                           // (the same in all CTAs of the cluster)
            if (AHEAD) {
#pragma unroll
                for (int i = 0; i < P; ++i) fetch(i, there_next, next_y >= 0);
            }
            if (g.logp && rank == 0 && threadIdx.x == 0) g.logp[row] = 0.f;
            if (g.dZ) {
                const float none[N] = {};
                for (int c = (int)threadIdx.x * N; c < cols; c += THREADS * N) store_entries(to, c, cols, !ANY || g.dz_vec, none);
            }
        } else {
            if (!AHEAD) {
#pragma unroll
                for (int i = 0; i < P; ++i) fetch(i, here, true);
            }
            const float zy = y < g.vocab ? to_f32(Z[row * g.ldz + y]) : __int_as_float(0x7fc00000);
            const float old = g.old_logp[row], adv = g.advantage[row], ref = g.ref_logp ? g.ref_logp[row] : 0.f;
            // The chosen entry, where one of this thread's pieces has it, becomes -Inf.  (8192 x 32000 bf16: 182 us, 179 with the entry left in, as it was then.  Its power taken out of the sum
            // again afterwards, in a branch that one warp enters, held the others up at the barrier: 185 to 190.)
            const int at = y < g.vocab ? (int)y - begin : -1;
            const bool mine = at >= 0 && at < cols && at / N % THREADS == (int)threadIdx.x;
            const int own = mine ? at / (N * THREADS) : -1;
            const uint4 hide = entry_mask<T>(at % N);
            Largest<T> most;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if (own == i) raw[i] = hidden<T>(raw[i], hide);
                if constexpr (ANY) {
                    const int c = (int)(threadIdx.x + i * THREADS) * N;
                    if (c + N > cols) raw[i] = only_first<T>(raw[i], cols - c);
                } else {
                    if (!there(i)) raw[i] = make_uint4(Largest<T>::kNone, Largest<T>::kNone, Largest<T>::kNone, Largest<T>::kNone);
                }
                most.take(raw[i]);
            }
            const float top = base_of(most.value(), g.k2.hi), base = top == minus_inf() ? 0.f : top;
            const uint64_t k22 = pair_of(g.k2.hi, g.k2.hi), base2 = pair_of(-base, -base);
            uint64_t e[P * N / 2], sum2[2] = {0ull, 0ull};
            // A piece's registers take the next row's as soon as its powers are formed.  The address depends on one of these, so that the loads go out one by one: left free, the
            // compiler unpacked all pieces first and asked for all of the next row at once in some builds, which holds up the load unit (8192 x 32000 bf16: 198 us, so 184).
#pragma unroll
            for (int i = 0; i < P; ++i) {
                uint64_t f[N / 2];
                Piece<T>::split(raw[i], f);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) {
                    const uint64_t x = fma2(f[j], k22, base2);
                    const uint64_t v = pair_of(exp2_fast(pair_lo(x)), exp2_fast(pair_hi(x)));
                    sum2[j & 1] = add2(sum2[j & 1], v);
                    e[i * (N / 2) + j] = v;
                }
                if (AHEAD) fetch(i, there_next, next_y >= 0, (int)e[i * (N / 2)] & g.zero);
            }
            sum2[0] = add2(sum2[0], sum2[1]);
            float2 all = joined_warp(make_float2(top, pair_lo(sum2[0]) + pair_hi(sum2[0])));
            // (slots are written again two rows on, and every thread has passed the barrier between)
            float2* slots = met[turn & 1];
            ++turn;
            if (cluster == 1) {
                if (lane == 0) slots[warp] = all;
                __syncthreads();
                all = lane < WARPS ? slots[lane] : make_float2(minus_inf(), 0.f);
            } else {
                if (lane < cluster) store_at(&slots[rank * WARPS + warp], (uint32_t)lane, all);
                cluster_meet();
                all = make_float2(minus_inf(), 0.f);
                for (int i = lane; i < cluster * WARPS; i += 32) all = joined(all, slots[i]);
            }
            all = joined_warp(all);
            const Chosen token = chosen_of(all, zy, g.k2);
            const Two o = in_powers(old), gap = sum_of(token.at.hi, -o.hi);
            const float r = token.empty ? 0.f : token.p * power_of(gap.hi, gap.lo + token.at.lo - o.lo);
            // (a ratio beyond fp32's range is no infinity that an advantage of 0 could not take away)
            const bool away = adv == 0.f && r == -minus_inf() && gap.hi < -minus_inf();
            const float free = away ? 0.f : r * adv, held = fminf(fmaxf(r, g.low), g.high) * adv;
            const bool clipped = free > held;
            float up = 0.f, slope = clipped ? 0.f : -free;     // up: e^(ref - logp)
            if (g.ref_logp) {
                const Two f = in_powers(ref), d = sum_of(f.hi, -token.at.hi);
                up = token.empty ? -minus_inf() : token.p_inverse * power_of(d.hi, d.lo + f.lo - token.at.lo);
                if (g.kl_coef != 0.f) slope = fmaf(-g.kl_coef, up - 1.f, slope);   // (a term without weight may be infinite)
            }
            const float coef = token.empty ? 0.f : g.grad_scale * w * slope;
            const float share = exp2_fast(top - (all.x == minus_inf() ? 0.f : all.x)) * token.share, factor = share == 0.f ? 0.f : -coef * share;
            if (g.dZ) {
                const uint64_t factor2 = pair_of(factor, factor);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    uint64_t out[N / 2];
#pragma unroll
                    for (int j = 0; j < N / 2; ++j) out[j] = mul2(e[i * (N / 2) + j], factor2);
                    const int c = (int)(threadIdx.x + i * THREADS) * N;
                    if constexpr (ANY) store_piece(to, c, cols, g.dz_vec, out);
                    else if (there(i)) st_stream_u4(to + c, Piece<T>::join(out));
                }
                // the chosen entry, by the thread that stored its piece
                if (mine && !token.empty) to[at] = from_f32<T>(coef * token.rest);
            }
            if (rank == 0 && threadIdx.x == kTeller) {
                const Two logp = logp_of(all.x, all.y, zy, g.k2);
                float kl = 0.f;
                if (g.ref_logp) {
                    const Two d = sum_of(ref, -logp.hi);
                    kl = above_line(fabsf(d.hi) < -minus_inf() ? d.hi + (d.lo - logp.lo) : d.hi, up);
                }
                const double pg = -(double)(clipped ? held : free);
                if (g.logp) g.logp[row] = logp.hi + logp.lo;
                sum_loss += (double)w * (g.kl_coef != 0.f ? (double)g.kl_coef * (double)kl + pg : pg);
                sum_pg += (double)w * pg;
                sum_kl += (double)w * (double)kl;
                if (clipped) sum_clip += (double)w;
            }
        }
        y = next_y;
        w = next_w;
        look(next + stride, next_y, next_w);
    }
    if (rank == 0 && threadIdx.x == kTeller) {
        double* to = g.parts + 4 * (blockIdx.x / cluster);
        to[0] = sum_loss; to[1] = sum_pg; to[2] = sum_kl; to[3] = sum_clip;
    }
    if (cluster > 1) cluster_meet();   // no CTA leaves while another may still write to its shared memory
}

// ---- log-probabilities alone -------------------------------------------------------------------------
// Nothing of a row has to stay: its threads go through it piece by piece with a running base and sum, and rows need no common
// pace.  GROUP threads have a row, or a CTA of a cluster its part of one.
constexpr int kScoreThreads = 256, kScorePieces = 4;

struct ScoreArgs {
    const void* Z;
    int64_t ldz;
    Span span;
    int64_t rows;
    int vocab, chunk;
    int cluster;
    const void* y;
    bool wide;
    Powers k2;
    float scale;
    bool all_rows;                 // those without a chosen token too, for their lse
    float *logp, *lse;             // either may be NULL
    double* logp64;                // the same before its rounding, for sums over sequences; or NULL
    Two* base;                     // what the backward pass takes its powers relative to, see base_from; or NULL
    Two per_lse;
    float* zeros;                  // a vector of `rows` zeros to write (the preference loss's gradients of logp), or NULL
};

// Powers of 2^(z hi - base) are probabilities times 2^(base's rest), with hi the temperature's first part and base = lse hi / scale (`per`: hi / scale): then what lo would add is in the
// base as far as entries near lse have it, and an entry lacks lo times its distance from there.  Infinities and NaN have no rest.
__device__ __forceinline__ Two base_from(Two lse, Two per) {
    const Two p = product_of(lse.hi, per.hi);
    return Two{p.hi, fabsf(p.hi) < -minus_inf() ? p.lo + fmaf(lse.hi, per.lo, lse.lo * per.hi) : 0.f};
}

template <typename T, int GROUP, bool ANY>
__global__ void __launch_bounds__(kScoreThreads, 5) score_kernel(const __grid_constant__ ScoreArgs g) {
    constexpr int N = Piece<T>::N, WARPS = kScoreThreads / 32;
    __shared__ float2 met[kMaxCluster * WARPS];
    if (g.cluster == 1) pdl_trigger();
    else cluster_tell_started();
    pdl_wait();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, member = threadIdx.x % GROUP;
    const uint32_t rank = GROUP > 32 && g.cluster > 1 ? cluster_rank() : 0u;
    const int64_t row = GROUP == 32 ? (int64_t)blockIdx.x * WARPS + warp : (int64_t)(blockIdx.x / g.cluster);
    if (row >= g.rows) return;                                 // (whole warps, and only with GROUP = 32, where there are no clusters)
    const int begin = (int)rank * g.chunk, cols = g.vocab - begin < g.chunk ? g.vocab - begin : g.chunk;
    const T* Z = static_cast<const T*>(g.Z) + row * g.ldz;
    const int64_t y = chosen(g.y, g.wide, row);
    const bool first = rank == 0 && member == 0;
    if (first && g.zeros) g.zeros[row] = 0.f;
    if (y < 0 && !g.all_rows) {                                // (the same in all threads of the row)
        if (first && g.logp) g.logp[row] = 0.f;
        if (first && g.logp64) g.logp64[row] = 0.;
        if (g.cluster > 1) cluster_wait_started();
        return;
    }
    const bool there = y >= 0 && y < g.vocab;
    const float zy = first && there ? to_f32(Z[y]) : __int_as_float(0x7fc00000);
    // the chosen entry, where one of this thread's pieces has it: left out of the sum
    const int at = there ? (int)y - begin : -1;
    const int chosen_piece = at >= 0 && at < cols && at / N % GROUP == member ? at / N * N : -1;
    float top = minus_inf();
    uint64_t sum2[2] = {0ull, 0ull};
    const uint64_t k22 = pair_of(g.k2.hi, g.k2.hi), low2 = pair_of(g.k2.lo, g.k2.lo);
    for (int c0 = member * N; c0 < cols; c0 += GROUP * kScorePieces * N) {
        uint4 raw[kScorePieces];
#pragma unroll
        for (int i = 0; i < kScorePieces; ++i) raw[i] = load_piece<ANY>(Z + begin, c0 + i * GROUP * N, cols, g.span);
        Largest<T> most;
        if (c0 + ((kScorePieces - 1) * GROUP + 1) * N > cols) {
#pragma unroll
            for (int i = 0; i < kScorePieces; ++i) raw[i] = only_first<T>(raw[i], cols - c0 - i * GROUP * N);
        }
        if ((unsigned)(chosen_piece - c0) < (unsigned)(GROUP * kScorePieces * N)) {
#pragma unroll
            for (int i = 0; i < kScorePieces; ++i)
                if (chosen_piece == c0 + i * GROUP * N) raw[i] = hidden<T>(raw[i], entry_mask<T>(at % N));
        }
#pragma unroll
        for (int i = 0; i < kScorePieces; ++i) most.take(raw[i]);
        const float here = base_of(most.value(), g.k2.hi);
        if (here > top) {
            const float less = exp2_fast(top - here);
            const uint64_t less2 = pair_of(less, less);
            sum2[0] = mul2(sum2[0], less2);
            sum2[1] = mul2(sum2[1], less2);
            top = here;
        }
        const float base = top == minus_inf() ? 0.f : top;
        const uint64_t base2 = pair_of(-base, -base);
#pragma unroll
        for (int i = 0; i < kScorePieces; ++i) {
            uint64_t f[N / 2];
            Piece<T>::split(raw[i], f);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) {
                const uint64_t x = fma2(f[j], low2, fma2(f[j], k22, base2));
                sum2[j & 1] = add2(sum2[j & 1], pair_of(exp2_fast(pair_lo(x)), exp2_fast(pair_hi(x))));
            }
        }
    }
    sum2[0] = add2(sum2[0], sum2[1]);
    float2 all = make_float2(top, pair_lo(sum2[0]) + pair_hi(sum2[0]));
    all = joined_warp(all);
    if constexpr (GROUP > 32) {
        if (g.cluster == 1) {
            if (lane == 0) met[warp] = all;
            __syncthreads();
        } else {
            cluster_wait_started();
            if (lane == 0) store_at(&met[(int)rank * WARPS + warp], 0u, all);
            cluster_meet();
        }
        if (rank != 0 || warp != 0) return;
        all = make_float2(minus_inf(), 0.f);
        for (int i = lane; i < g.cluster * WARPS; i += 32) all = joined(all, met[i]);
        all = joined_warp(all);
    }
    if (first) {
        const Two lp = y < 0 ? Two{0.f, 0.f} : logp_of(all.x, all.y, zy, g.k2);
        if (g.logp) g.logp[row] = lp.hi + lp.lo;
        if (g.logp64) g.logp64[row] = wide(lp);
        if (g.lse || g.base) {
            const Two own = product_of(zy, g.scale);
            Two lse = sum_of(own.hi, -lp.hi);
            lse.lo += own.lo - lp.lo;
            if (!there || is_nothing(zy * g.k2.hi)) {              // the others' alone
                float exponent, rest;
                split_log2(all.y, exponent, rest);
                const Two t = sum_of(all.x, exponent), a = product_of(t.hi, kLn2);
                const bool empty = all.x == minus_inf() && all.y == 0.f;
                lse = empty ? Two{minus_inf(), 0.f} : Two{a.hi, a.lo + fmaf(t.hi, kLn2Rest, (t.lo + rest + kPowerShort * kLog2e) * kLn2)};
            }
            if (g.lse) g.lse[row] = lse.hi + lse.lo;
            if (g.base) g.base[row] = base_from(lse, g.per_lse);
        }
    }
}

// out[i] = factor * sum over k of parts[k][i], i < WIDTH, by one warp; fixed order
template <int WIDTH>
__device__ __forceinline__ void total_of(const double* __restrict__ parts, int64_t count, double factor, float* __restrict__ out) {
    const int lane = threadIdx.x % 32;
    double sum[WIDTH] = {};
#pragma unroll 4
    for (int64_t k = lane; k < count; k += 32)
#pragma unroll
        for (int i = 0; i < WIDTH; ++i) sum[i] += parts[k * WIDTH + i];
#pragma unroll
    for (int i = 0; i < WIDTH; ++i) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
        if (lane == 0) out[i] = (float)(factor * sum[i]);
    }
}
template <int WIDTH>
__global__ void total_kernel(const double* __restrict__ parts, int64_t count, double factor, float* __restrict__ out) {
    pdl_trigger();
    pdl_wait();
    total_of<WIDTH>(parts, count, factor, out);
}

// ---- the gradient from lse -------------------------------------------------------------------------
constexpr int kBackThreads = 256, kBackPieces = 4;

struct BackArgs {
    const void* Z;
    int64_t ldz;
    Span span;
    int64_t rows;
    int vocab, slices;
    const void* y;
    bool wide;
    float k2, scale;               // scale: of the logits and of the gradient
    const float *lse, *dlogp;
    Two per_lse;
    const Two* base;               // instead of lse: what a forward pass left, and
    const double* logp;            // the chosen token's log-probability beside it
    void* dZ;
    int64_t lddz;
    bool dz_vec;
    const double* parts;           // of the preference loss, which the first warp adds up on the way (a launch less); or NULL
    int64_t pairs;
    float* loss;
};

// a warp for each slice of 32 * kBackPieces pieces, from the last one back
template <typename T, bool ANY>
__global__ void __launch_bounds__(kBackThreads) backward_kernel(const __grid_constant__ BackArgs g) {
    constexpr int N = Piece<T>::N, kSlice = 32 * kBackPieces * N;
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x % 32;
    if (g.loss && blockIdx.x == 0 && threadIdx.x < 32) total_of<1>(g.parts, g.pairs, 1.0 / (double)g.pairs, g.loss);
    const int64_t items = g.rows * g.slices, stride = (int64_t)gridDim.x * (kBackThreads / 32);
    for (int64_t k = (int64_t)blockIdx.x * (kBackThreads / 32) + threadIdx.x / 32; k < items; k += stride) {
        const int64_t item = items - 1 - k, row = item / g.slices;
        const int c0 = (int)(item - row * g.slices) * kSlice + lane * N;
        const int64_t y = chosen(g.y, g.wide, row);
        const float d = g.dlogp[row];
        const Two base = g.base ? g.base[row] : base_from(Two{g.lse[row], 0.f}, g.per_lse);
        const bool live = y >= 0 && d != 0.f && base.hi != minus_inf();
        const T* from = static_cast<const T*>(g.Z) + row * g.ldz;
        uint4 raw[kBackPieces];
#pragma unroll
        for (int i = 0; i < kBackPieces; ++i) raw[i] = load_piece<ANY>(from, c0 + i * 32 * N, live ? g.vocab : 0, g.span);
        const float coef = y < g.vocab ? d * g.scale : __int_as_float(0x7fc00000);
        const float factor = -coef * exp2_fast(-base.lo);
        const int at = y < g.vocab ? (int)y : -1;
        T* to = static_cast<T*>(g.dZ) + row * g.lddz;
#pragma unroll
        for (int i = 0; i < kBackPieces; ++i) {
            const int c = c0 + i * 32 * N;
            if (c >= g.vocab) continue;
            float f[N];
            Piece<T>::split(raw[i], f);
            if (live) {
#pragma unroll
                for (int j = 0; j < N; ++j) f[j] = exp2_fast(fmaf(f[j], g.k2, -base.hi)) * factor;
                if (at >= c && at < c + N) {
                    // 1 - p from log p, where that is known: the difference has few bits left for a token that the row is sure of
                    const float rest = g.logp ? -expm1f((float)g.logp[row]) : 0.f;
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (at == c + j) f[j] = g.logp ? coef * rest : f[j] + coef;
                }
            }
            store_entries(to, c, g.vocab, !ANY || g.dz_vec, f);
        }
    }
}

// ---- pairs of sequences ----------------------------------------------------------------------------
constexpr int kPairThreads = 256;

__global__ void __launch_bounds__(kPairThreads) pairs_kernel(const double* __restrict__ logp, int64_t rows, const int32_t* __restrict__ offsets,
                                                             const float* __restrict__ ref, int64_t pairs, float beta, float smoothing,
                                                             float grad, float* __restrict__ margin, float* __restrict__ sums,
                                                             float* __restrict__ dlogp, double* __restrict__ parts) {
    __shared__ double sm[2][kPairThreads / 32];
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int64_t p = blockIdx.x; p < pairs; p += gridDim.x) {
        int64_t at[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int64_t least = i ? at[i - 1] : 0, o = offsets[2 * p + i];
            at[i] = o < least ? least : (o > rows ? rows : o);
        }
        double s[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            double x = 0.;
            for (int64_t t = at[i] + threadIdx.x; t < at[i + 1]; t += kPairThreads) x += logp[t];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
            if (lane == 0) sm[i][warp] = x;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i] = 0.;
#pragma unroll
            for (int k = 0; k < kPairThreads / 32; ++k) s[i] += sm[i][k];
        }
        const double h = (double)beta * ((s[0] - (double)ref[2 * p]) - (s[1] - (double)ref[2 * p + 1]));
        const float x = (float)h;
        // -log sigmoid(x) = max(-x, 0) + log(1 + e^-|x|), and the sigmoids, from one exponential
        const float u = expf(-fabsf(x)), l = log1pf(u), up = 1.f / (1.f + u), down = u / (1.f + u);
        const float plus = x >= 0.f ? up : (x < 0.f ? down : x), minus = x >= 0.f ? down : (x < 0.f ? up : x);   // sigmoid(x), sigmoid(-x)
        if (threadIdx.x == 0) {
            const float rise = x < 0.f ? -x : 0.f, fall = x > 0.f ? x : 0.f;
            // (a term without weight may be infinite)
            parts[p] = (double)((smoothing < 1.f ? (1.f - smoothing) * (rise + l) : 0.f) + (smoothing > 0.f ? smoothing * (fall + l) : 0.f));
            margin[p] = x;
            sums[2 * p] = (float)s[0];
            sums[2 * p + 1] = (float)s[1];
        }
        if (dlogp) {
            const float d = grad * (smoothing * plus - (1.f - smoothing) * minus);
            for (int64_t t = at[0] + threadIdx.x; t < at[1]; t += kPairThreads) dlogp[t] = d;
            for (int64_t t = at[1] + threadIdx.x; t < at[2]; t += kPairThreads) dlogp[t] = -d;
        }
        __syncthreads();
    }
}

// ---- shapes ----------------------------------------------------------------------------------------
// How many CTAs share a row: as many as its entries need registers of; then, while rows are so few that SMs are left over, more, down to
// kLeastChunk entries each.
constexpr int kLeastChunk = 2048;
// pieces of a thread with the next row's beside them: eight of 16 bits, twelve of fp32
template <typename T> constexpr int kMostPieces = 96 / (Piece<T>::N + 4);
template <typename T>
int cluster_of(int64_t rows, int64_t vocab, bool aligned) {
    int64_t cluster = 1;                                       // 1, 2, 4 or 8
    while (cluster < kMaxCluster && vocab > cluster * 512 * kMostPieces<T> * Piece<T>::N) cluster *= 2;   // (fp32 beyond eight: sixteen pieces a thread)
    while (cluster * 2 <= kMaxCluster && rows * cluster * 2 <= kSMs && vocab >= cluster * 2 * kLeastChunk) cluster *= 2;
    // Where a few rows would need a second turn of large CTAs, smaller ones, several to an SM, wait less.  Eight instead of four CTAs, 38 to 73 rows of bf16: 65544 columns
    // 14.3 -> 12.4 us (73: 18.5 -> 17.8), 100000 16.2 -> 14.5 (22.7 -> 21.2), 131072 16.5 -> 16.0 (24.5 -> 21.7).  Four instead of two pay only for rows that no vector load
    // fits, and for few: 75 and 90 of 50257 36.3 -> 33.3 and 39.0 -> 37.3, 110 40.8 -> 40.6, 147 44.1 -> 59.7; aligned 75 of 40000 and 50264 12.4 -> 12.9 and 14.4 -> 14.4, 147 13.5 ->
    // 18.5 and 14.4 -> 20.5.  (Rows of one CTA each stay: 150 of 32000 take 10.6 us, with clusters of four 13.3.)
    const int64_t ctas = rows * cluster;
    if (ctas > kSMs && ((cluster == 4 && ctas < 2 * kSMs) || (cluster == 2 && !aligned && 4 * ctas <= 5 * kSMs))) cluster *= 2;
    return (int)cluster;
}
// Calls f<THREADS, P>() for CTAs of `pieces` pieces: P is what a thread has, and the CTA the smallest of which that is at most eight (of 512 threads: kMostPieces), four in
// CTAs of 128 (they wait less for one another).
template <typename T, bool ANY, typename F>
detox_status by_pieces(int pieces, F f) {
    switch (ceil_div(pieces, 128)) {
        case 1: return f.template operator()<128, 1>();
        case 2: return f.template operator()<128, 2>();
        case 3: return f.template operator()<128, 3>();
        case 4: return f.template operator()<128, 4>();
    }
    switch (ceil_div(pieces, 256)) {
        case 3: return f.template operator()<256, 3>();
        case 4: return f.template operator()<256, 4>();
        case 5: return f.template operator()<256, 5>();
        case 6: return f.template operator()<256, 6>();
        case 7: return f.template operator()<256, 7>();
        case 8: return f.template operator()<256, 8>();
    }
    switch (ceil_div(pieces, 512)) {
        case 5: return f.template operator()<512, 5>();
        case 6: return f.template operator()<512, 6>();
        case 7: return f.template operator()<512, 7>();
        case 8: return f.template operator()<512, 8>();
    }
    if constexpr (sizeof(T) == 4) {
        switch (ceil_div(pieces, 512)) {
            case 9: return f.template operator()<512, 9>();
            case 10: return f.template operator()<512, 10>();
            case 11: return f.template operator()<512, 11>();
            case 12: return f.template operator()<512, 12>();
        }
    }
    if constexpr (ANY && sizeof(T) == 4) {
        if (pieces <= 512 * 16) return f.template operator()<512, 16>();
    }
    return DETOX_ERR_UNSUPPORTED;
}

template <typename T, bool ANY>
struct Policy {
    const RowsArgs& g;
    int64_t* clusters;
    cudaStream_t s;
    template <int THREADS, int P>
    detox_status operator()() const {
        const int64_t most = (int64_t)kSMs * kCtas<T, THREADS, P> / g.cluster;
        *clusters = g.rows < most ? g.rows : most;
        // Clusters that fill the SMs' registers do not overlap with the stream's other kernels, as the gated products' pairs do not.
        return launch(g.cluster == 1, policy_kernel<T, THREADS, P, ANY>, (unsigned)(*clusters * g.cluster), THREADS, 0, (unsigned)g.cluster, s, g);
    }
};
template <typename T>
bool pieces(const void* p, int64_t ld) {
    return aligned16(p) && ld % Piece<T>::N == 0;
}
// clusters: how many parts the loss has
template <typename T>
detox_status policy_of(RowsArgs g, int64_t* clusters, cudaStream_t s) {
    g.pieces = (int)ceil_div((int64_t)g.vocab, (int64_t)Piece<T>::N);
    g.span = span_of<T>(g.Z, g.ldz, g.rows, g.vocab);
    g.dz_vec = pieces<T>(g.dZ, g.lddz);
    const bool aligned = g.vocab % Piece<T>::N == 0 && g.span.vec && (!g.dZ || g.dz_vec);
    g.cluster = cluster_of<T>(g.rows, g.vocab, aligned);
    const int most = (int)ceil_div((int64_t)g.pieces, (int64_t)g.cluster);
    if (aligned && most <= 512 * kMostPieces<T>) return by_pieces<T, false>(most, Policy<T, false>{g, clusters, s});
    return by_pieces<T, true>(most, Policy<T, true>{g, clusters, s});
}

// A warp for a row of up to 8 pieces a lane; else a CTA, or where rows are few a cluster, as long as its threads have pieces for a turn each.
template <typename T>
detox_status score_of(ScoreArgs g, cudaStream_t s) {
    constexpr int N = Piece<T>::N;
    g.span = span_of<T>(g.Z, g.ldz, g.rows, g.vocab);
    const bool any = !(g.vocab % N == 0 && g.span.vec);
    g.cluster = 1;
    g.chunk = g.vocab;
    if (g.vocab <= 32 * 8 * N)
        return launch_chained(any ? score_kernel<T, 32, true> : score_kernel<T, 32, false>, (unsigned)ceil_div(g.rows, (int64_t)(kScoreThreads / 32)),
                              kScoreThreads, 0, 1, s, g);
    while (g.cluster < kMaxCluster && g.rows * g.cluster <= kSMs * 2 && g.vocab >= g.cluster * 2 * kScoreThreads * kScorePieces * N) g.cluster *= 2;
    g.chunk = (int)(ceil_div(ceil_div((int64_t)g.vocab, (int64_t)g.cluster), (int64_t)N) * N);
    return launch(g.cluster == 1, any ? score_kernel<T, kScoreThreads, true> : score_kernel<T, kScoreThreads, false>, (unsigned)(g.rows * g.cluster),
                  kScoreThreads, 0, (unsigned)g.cluster, s, g);
}

template <typename T>
detox_status backward_of(BackArgs g, cudaStream_t s) {
    g.slices = (int)ceil_div((int64_t)g.vocab, (int64_t)32 * kBackPieces * Piece<T>::N);
    g.span = span_of<T>(g.Z, g.ldz, g.rows, g.vocab);
    g.dz_vec = pieces<T>(g.dZ, g.lddz);
    const bool any = !(g.vocab % Piece<T>::N == 0 && g.span.vec && g.dz_vec);
    const int64_t need = ceil_div(g.rows * g.slices, (int64_t)(kBackThreads / 32)), most = (int64_t)kSMs * 16;
    return launch_chained(any ? backward_kernel<T, true> : backward_kernel<T, false>, (unsigned)(need < most ? need : most), kBackThreads, 0, 1, s, g);
}

}  // namespace

namespace {
// For powers that have both parts, lo is above 0, so that -Inf stays -Inf through both products.  (8192 x 32000 bf16, policy loss: a second product for each entry takes 202 us
// instead of 182.  There the entries have hi alone, and only their common base both: what is left is lo times their distance from the largest, at most 10^-7 of the sum.)
Powers powers_of(float scale, bool both) {
    const double k = (double)scale * 1.4426950408889634;
    float hi = (float)k;
    if (both && (double)hi >= k) hi = nextafterf(hi, 0.f);
    const float lo = (float)(k - (double)hi), least = 1.4e-45f;
    if (!both) return Powers{hi, 0.f, lo / hi};
    return Powers{hi > least ? hi : least, lo > least ? lo : least, 0.f};
}
Two per_lse_of(float scale) {
    const double per = (double)powers_of(scale, false).hi / (double)scale;
    return Two{(float)per, (float)(per - (double)(float)per)};
}
detox_status launch_scores(int dtype, const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y, float scale, bool all_rows,
                           float* logp, float* lse, double* logp64, Two* base, float* zeros, cudaStream_t s) {
    if (rows == 0) return DETOX_OK;
    ScoreArgs g = {};
    g.Z = Z; g.ldz = ldz; g.rows = rows; g.vocab = (int)vocab;
    g.y = y; g.wide = index == DETOX_INDEX_INT64;
    g.k2 = powers_of(scale, true);
    g.scale = scale;
    g.all_rows = all_rows;
    g.logp = logp; g.lse = lse; g.logp64 = logp64; g.base = base; g.zeros = zeros;
    g.per_lse = per_lse_of(scale);
    if (dtype == DETOX_DTYPE_FLOAT) return score_of<float>(g, s);
    if (dtype == DETOX_DTYPE_HALF) return score_of<__half>(g, s);
    return score_of<__nv_bfloat16>(g, s);
}
detox_status backward_of(int dtype, const BackArgs& g, cudaStream_t s) {
    if (dtype == DETOX_DTYPE_FLOAT) return backward_of<float>(g, s);
    if (dtype == DETOX_DTYPE_HALF) return backward_of<__half>(g, s);
    return backward_of<__nv_bfloat16>(g, s);
}
BackArgs back_args(const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y, float scale, const float* dlogp, void* dZ,
                   int64_t lddz) {
    BackArgs g = {};
    g.Z = Z; g.ldz = ldz; g.rows = rows; g.vocab = (int)vocab;
    g.y = y; g.wide = index == DETOX_INDEX_INT64;
    g.k2 = powers_of(scale, false).hi;
    g.scale = scale;
    g.per_lse = per_lse_of(scale);
    g.dlogp = dlogp;
    g.dZ = dZ; g.lddz = lddz;
    return g;
}
}  // namespace

detox_status launch_token_logp(int dtype, const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y, float scale,
                               float* logp, float* lse, cudaStream_t s) {
    return launch_scores(dtype, Z, ldz, rows, vocab, index, y, scale, lse != nullptr, logp, lse, nullptr, nullptr, nullptr, s);
}

detox_status launch_token_logp_backward(int dtype, const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y,
                                        float scale, const float* lse, const float* dlogp, void* dZ, int64_t lddz, cudaStream_t s) {
    if (rows == 0) return DETOX_OK;
    BackArgs g = back_args(Z, ldz, rows, vocab, index, y, scale, dlogp, dZ, lddz);
    g.lse = lse;
    return backward_of(dtype, g, s);
}

size_t policy_loss_ws_bytes(int64_t rows) {
    const int64_t most = (int64_t)kSMs * 16;   // CTAs of 128 threads on an SM
    return align_up((size_t)(rows < most ? rows : most) * 4 * sizeof(double));
}

detox_status launch_policy_loss(const detox_policy_desc& d, float* stats, float* logp, void* dZ, int64_t lddz, void* ws, cudaStream_t s) {
    int64_t clusters = 0;
    double* parts = static_cast<double*>(ws);
    if (d.rows > 0) {
        RowsArgs g = {};
        g.Z = d.Z; g.ldz = d.ldz; g.rows = d.rows; g.vocab = (int)d.vocab;
        g.y = d.y; g.wide = d.index == DETOX_INDEX_INT64;
        g.k2 = powers_of(d.scale, false);
        g.logp = logp;
        g.old_logp = d.old_logp; g.advantage = d.advantage; g.ref_logp = d.ref_logp; g.weight = d.weight;
        g.low = 1.f - d.clip_low; g.high = 1.f + d.clip_high;
        g.kl_coef = d.kl_coef;
        g.even_weight = (float)(1.0 / (double)d.rows);
        g.grad_scale = d.grad_scale * d.scale;
        g.dZ = dZ; g.lddz = lddz;
        g.parts = parts;
        detox_status st;
        if (d.dtype == DETOX_DTYPE_FLOAT) st = policy_of<float>(g, &clusters, s);
        else if (d.dtype == DETOX_DTYPE_HALF) st = policy_of<__half>(g, &clusters, s);
        else st = policy_of<__nv_bfloat16>(g, &clusters, s);
        if (st != DETOX_OK) return st;
    }
    return launch_chained(total_kernel<4>, 1, 32, 0, 1, s, parts, clusters, 1.0, stats);
}

// logp in 64 bits, the backward pass's base in two parts and logp's gradient for each row, then a part of the loss for each pair
size_t preference_loss_ws_bytes(int64_t rows, int64_t pairs) {
    return 2 * align_up((size_t)rows * 8) + align_up((size_t)rows * sizeof(float)) + align_up((size_t)pairs * sizeof(double));
}

detox_status launch_preference_loss(const detox_preference_desc& d, float* loss, float* margin, float* sums, void* dZ, int64_t lddz, void* ws,
                                    cudaStream_t s) {
    const size_t wide = align_up((size_t)d.rows * 8), vector = align_up((size_t)d.rows * sizeof(float));
    char* at = static_cast<char*>(ws);
    double *logp = reinterpret_cast<double*>(at), *parts = reinterpret_cast<double*>(at + 2 * wide + vector);
    Two* base = reinterpret_cast<Two*>(at + wide);
    float* dlogp = reinterpret_cast<float*>(at + 2 * wide);
    detox_status st = launch_scores(d.dtype, d.Z, d.ldz, d.rows, d.vocab, d.index, d.y, d.scale, false, nullptr, nullptr, logp, dZ ? base : nullptr, dZ ? dlogp : nullptr, s);
    if (st != DETOX_OK) return st;
    if (d.pairs > 0) {
        const int64_t most = (int64_t)kSMs * 8;
        const float grad = (float)((double)d.grad_scale * (double)d.beta / (double)d.pairs);
        st = launch_chained(pairs_kernel, (unsigned)(d.pairs < most ? d.pairs : most), kPairThreads, 0, 1, s, logp, d.rows, d.offsets, d.ref,
                            d.pairs, d.beta, d.smoothing, grad, margin, sums, dZ && d.rows ? dlogp : nullptr, parts);
        if (st != DETOX_OK) return st;
    }
    if (dZ && d.rows > 0) {
        BackArgs g = back_args(d.Z, d.ldz, d.rows, d.vocab, d.index, d.y, d.scale, dlogp, dZ, lddz);
        g.base = base; g.logp = logp;
        if (d.pairs > 0) {
            g.parts = parts; g.pairs = d.pairs; g.loss = loss;
        }
        st = backward_of(d.dtype, g, s);
        if (st != DETOX_OK || d.pairs > 0) return st;
    }
    return launch_chained(total_kernel<1>, 1, 32, 0, 1, s, parts, d.pairs, d.pairs > 0 ? 1.0 / (double)d.pairs : 0.0, loss);
}

}  // namespace detox
