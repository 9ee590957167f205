// One AdamW step over many tensors, with states in 32 bits or in 8.
//
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p - lr (wd p + (m / c1) / (sqrt(v / c2) + eps)),  c_i = 1 - b_i^step
//
// Bound by HBM: every buffer is read once and written once (fp32 weights and states: 28 bytes an entry; bf16 weights, fp32 masters and
// gradients, 8-bit states: 18).  The tensors' pointers travel as kernel parameters, so a step is one launch for each few hundred of them,
// with nothing to copy and nothing to set up, and a captured one keeps them; tensors of different types take a launch for each kind.  A warp
// takes blocks of 128 entries, 4 a lane, so that a block's scale is one warp-wide reduction and every access of a warp is contiguous: 16 bytes a
// lane in fp32, and where a buffer is not aligned for that, single entries dealt round the lanes.  Tensors whose buffers are all out of alignment by
// the same number of entries (slices of vectors of one layout) are taken from the boundary before their first one on.
// 21.7 M fp32 entries in 161 tensors at odd offsets: 100 us, 6.1 TB/s (floor 94).
//
// 8 bits: m and sqrt(v) as e4m3 numbers with a power-of-two scale for each block.  Of v the root is kept, since its range is half as
// wide (v's would leave the form's 18 binary orders).  Rounding is random: added to the bits that the form drops, 16 random ones round up or down with
// the right mean; a sum of thousands of steps that each change an entry by less than its spacing keeps its mean that way.
// 169 M entries in 13 tensors: 597 to 645 us by machine, 4.7 to 5.1 TB/s (floor 467); the rounding's instructions are what it spends beside it (484 without them).  Slices that start off a
// boundary go byte by byte: 48 M entries in 12 tensors 180 us aligned, 305 otherwise.
#include <cmath>
#include <cstring>

#include "worker.cuh"

namespace detox {

namespace {

constexpr int kThreads = 256;
constexpr int kCtas = 4;                         // on an SM
// Blocks of 128 entries that a warp has in flight.  32 bits: two take 112 us for 21.7 M entries, one 100.  8 bits: 169 M entries take 600 us with one, 575 with two.
template <bool EIGHT> constexpr int kBlocks = EIGHT ? 2 : 1;
template <bool EIGHT> constexpr int kPart = kBlocks<EIGHT> * kKeepBlock * (kThreads / 32);   // entries that a CTA has in flight
// Entries that a CTA takes at a time.  8 bits: two parts, so that the scales that it writes fill sectors of 32 bytes, by one store.  As single bytes, from several SMs into
// one sector, they took a fifth of the time (618 us without any rounding, 498 without the scales' stores).
template <bool EIGHT> constexpr int kUnit = EIGHT ? 2 * kPart<EIGHT> : kPart<EIGHT>;
static_assert(kUnit<true> / kKeepBlock == 32 && 4 * (kThreads / 32) == 32, "a scale for each lane, four for each warp");
constexpr int kKinds = 3 * 3 * 2;                // types of weights and gradients, with a master copy or without

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
    bool vec;                                    // every buffer is aligned for a lane's 4 entries
    int32_t skip;                                // the first entries are not the tensor's (the pointers are that far before it)
};
struct Numbers {
    uint64_t beta1, beta2, rest1, rest2, eps, grad_scale;   // twice each, as the packed arithmetic takes them; rest: 1 - beta
    float lr;
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

__device__ __forceinline__ uint32_t mix_rest(uint32_t x) {
    x *= 0x85ebca6bu;
    x ^= x >> 13;
    x *= 0xc2b2ae35u;
    return x ^ (x >> 16);
}
__device__ __forceinline__ uint32_t mix(uint32_t x) {
    return mix_rest(x ^ (x >> 16));
}

// The root and the inverse to a unit or so, an instruction each (sqrtf and a division cost some eight an entry).  In 32 bits the root of v below 2^-126 is taken, too, since beside the
// least eps it counts.  In 8 bits such v count as 0: the three instructions that it takes would cost a tenth (169 M entries 597 -> 653 us), and the least eps is larger for it.  What
// the inverse is taken of is no less than eps.
template <bool SMALL>
__device__ __forceinline__ float root_of(float x) {
    float y;
    if constexpr (SMALL) asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    else asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float inverse_of(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 4 entries of a lane: contiguous ones from entry `at` on (VEC), or at, at + 32, ... of the block, where there are so many.  Offsets in 32 bits from a pointer that is the same
// for all threads take no registers for addresses.
template <bool VEC, typename T>
__device__ __forceinline__ void load4(const T* from, unsigned at, int low, int left, float (&f)[4]) {
    if constexpr (!VEC) {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = 32 * j + lane >= low && 32 * j + lane < left ? to_f32(from[at + 32u * j]) : 0.f;
    } else if constexpr (sizeof(T) == 4) {
        const float4 x = ld_stream_f4(reinterpret_cast<const float*>(from) + at);
        f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
    } else {
        const uint2 x = __ldcs(reinterpret_cast<const uint2*>(from + at));
        const float2 a = unpack2<T>(x.x), b = unpack2<T>(x.y);
        f[0] = a.x; f[1] = a.y; f[2] = b.x; f[3] = b.y;
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store4(T* to, unsigned at, int low, int left, const float (&f)[4]) {
    if constexpr (!VEC) {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (32 * j + lane >= low && 32 * j + lane < left) to[at + 32u * j] = from_f32<T>(f[j]);
    } else if constexpr (sizeof(T) == 4) {
        st_stream_f4(reinterpret_cast<float*>(to) + at, make_float4(f[0], f[1], f[2], f[3]));
    } else {
        __stcs(reinterpret_cast<uint2*>(to + at), make_uint2(pack2<T>(f[0], f[1]), pack2<T>(f[2], f[3])));
    }
}
// 4 bytes of a lane, as one word
template <bool VEC>
__device__ __forceinline__ uint32_t load_bytes(const uint8_t* from, unsigned at, int left) {
    uint32_t q = 0u;
    if constexpr (VEC) {
        q = __ldcs(reinterpret_cast<const unsigned int*>(from + at));
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (32 * j + (int)(threadIdx.x % 32) < left) q |= (uint32_t)from[at + 32u * j] << (8 * j);
    }
    return q;
}
template <bool VEC>
__device__ __forceinline__ void store_bytes(uint8_t* to, unsigned at, int left, uint32_t q) {
    if constexpr (VEC) {
        __stcs(reinterpret_cast<unsigned int*>(to + at), q);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (32 * j + (int)(threadIdx.x % 32) < left) to[at + 32u * j] = (uint8_t)(q >> (8 * j));
    }
}

__device__ __forceinline__ float largest(float a, float b) {   // NaN where one is NaN
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// The 8-bit form of entries, rounded at random
//
// e4m3 keeps 3 of the 23 bits behind an fp32 number's first one, so a random number of 20 bits (16 random ones and zeros) is added to the number's own bits and the lowest 20 are
// cut off.  Divided by the scale and by 2^120 an entry is an fp32 number whose bits 26 .. 20 are the e4m3 number's, below 2^-6, where e4m3's steps stay 2^-9
// wide, too: fp32's own numbers without a first bit begin at 2^-126.  So entries of any size take the same path, without a conversion: added, shifted, a byte taken out.
//
// Four of a lane, finite, the block's largest at most 448 after the scale (a root that is a unit too large there does no harm: the random numbers are at least 16 short of a
// carry).  ROOTS: of the hash h's upper half, and entries > 0 stay so; else of its lower half, and with signs.
template <bool ROOTS>
__device__ __forceinline__ uint32_t rounded4(const uint64_t (&p)[2], float inverse, const uint32_t (&h)[4]) {
    const uint64_t inverse2 = pair_of(inverse, inverse), down2 = pair_of(7.52316385e-37f, 7.52316385e-37f);   // 2^-120
    const uint64_t a = mul2(mul2(p[0], inverse2), down2), b = mul2(mul2(p[1], inverse2), down2);
    const uint32_t w[4] = {(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = (w[j] << 4) + __byte_perm(h[j], 0u, ROOTS ? 0x4324 : 0x4104);   // the byte on top is the number
    auto tops = [](uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) { return __byte_perm(__byte_perm(x0, x1, 0x0073), __byte_perm(x2, x3, 0x0073), 0x5410); };
    uint32_t q = tops(r[0], r[1], r[2], r[3]);
    if (!ROOTS) return q | (tops(w[0], w[1], w[2], w[3]) & 0x80808080u);
    if ((q - 0x01010101u) & ~q & 0x80808080u) {   // a byte is 0
        const float x[4] = {pair_lo(p[0]), pair_hi(p[0]), pair_lo(p[1]), pair_hi(p[1])};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (((q >> (8 * j)) & 0xffu) == 0u && x[j] > 0.f) q |= 1u << (8 * j);
    }
    return q;
}
// The same, and NaN for what is not finite: a function of its own, since it is hardly ever needed and its registers would be missed
template <bool ROOTS>
__device__ __noinline__ uint32_t rounded4_any(uint64_t p0, uint64_t p1, float inverse, uint32_t h0, uint32_t h1, uint32_t h2, uint32_t h3) {
    const uint64_t p[2] = {p0, p1};
    const uint32_t h[4] = {h0, h1, h2, h3}, x[4] = {(uint32_t)p0, (uint32_t)(p0 >> 32), (uint32_t)p1, (uint32_t)(p1 >> 32)};
    uint32_t q = rounded4<ROOTS>(p, inverse, h);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if ((x[j] & 0x7fffffffu) >= 0x7f800000u) q |= 0x7fu << (8 * j);
    return q;
}

// The largest entry of a block, 4 entries a lane (two packed pairs), as an integer (positive numbers, Inf and NaN are in that order).
__device__ __forceinline__ uint32_t largest_of(const uint64_t (&p)[2]) {
    const float lane = largest(largest(fabsf(pair_lo(p[0])), fabsf(pair_hi(p[0]))), largest(fabsf(pair_lo(p[1])), fabsf(pair_hi(p[1]))));
    return __reduce_max_sync(0xffffffffu, __float_as_uint(lane) & 0x7fffffffu);
}
// ... and of its finite entries alone
__device__ __noinline__ uint32_t largest_finite(uint64_t p0, uint64_t p1) {
    const uint32_t a[4] = {(uint32_t)p0, (uint32_t)(p0 >> 32), (uint32_t)p1, (uint32_t)(p1 >> 32)};
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if ((a[j] & 0x7fffffffu) < 0x7f800000u) top = max(top, a[j] & 0x7fffffffu);
    return __reduce_max_sync(0xffffffffu, top);
}

// The 8-bit form of a block, rounded at random.  Returns the scale's biased exponent.  Inf and NaN become NaN and do not count for it.
//
// of: the entries (ROOTS: their squares), and top their largest, from which the scale is taken.  It decides over a whole block's scale, so its root is rounded properly
// here; the entries' own are approximate.
template <bool ROOTS>
__device__ __forceinline__ uint32_t keep_at_random(const uint64_t (&p)[2], const uint64_t (&of)[2], uint32_t top, const uint32_t (&h)[4], uint32_t* q) {
    const bool finite = top < 0x7f800000u;
    if (!finite) top = largest_finite(of[0], of[1]);
    const uint32_t e = keep_exponent(ROOTS ? sqrtf(__uint_as_float(top)) : __uint_as_float(top));
    const float inverse = keep_inverse(e);
    if (finite) *q = rounded4<ROOTS>(p, inverse, h);
    else *q = rounded4_any<ROOTS>(p[0], p[1], inverse, h[0], h[1], h[2], h[3]);
    return e;
}

struct Now {
    float lr, c1, root_c2;
    uint32_t seed;                               // of the tensor's random bits
};
__device__ __forceinline__ uint64_t both(float v) { return pair_of(v, v); }
__device__ __forceinline__ uint64_t pairs_at(const float (&f)[4], int k) { return pair_of(f[2 * k], f[2 * k + 1]); }

// A part of tensor t from entry `at` on.  PT, GT: of the weights and the gradient.  The arithmetic goes two entries at a time.  EIGHT and VEC:
// `part` of a unit; scales_m and scales_v hold the unit's scales, one a lane, and the new ones are left in keep_m and keep_v, a byte for each of this warp's blocks.
template <bool EIGHT, bool VEC, typename PT, typename GT, bool MASTER>
__device__ __forceinline__ void step_part(const Tensor& t, int64_t at, const Numbers& number, const Now& now, int part, float scales_m, float scales_v, uint32_t& keep_m,
                                          uint32_t& keep_v) {
    constexpr int B = kBlocks<EIGHT>, kStep = kKeepBlock * (kThreads / 32);
    const int lane = threadIdx.x % 32, first = threadIdx.x / 32 * kKeepBlock;   // this warp's blocks start at at + first + b kStep
    const unsigned own = VEC ? 4 * threadIdx.x : first + lane;                  // and this lane's entries of them
    const GT* G = static_cast<const GT*>(t.G) + at;
    PT* P = static_cast<PT*>(t.P) + at;
    float* master = t.master + at;
    uint8_t *M8 = static_cast<uint8_t*>(t.M) + at, *V8 = static_cast<uint8_t*>(t.V) + at;
    float *M = static_cast<float*>(t.M) + at, *V = static_cast<float*>(t.V) + at;
    const uint8_t *ME = t.ME + at / kKeepBlock, *VE = t.VE + at / kKeepBlock;
    const int rest = t.n - at < kPart<EIGHT> ? (int)(t.n - at) : kPart<EIGHT>;
    float g[B][4], p[B][4];
    float m32[EIGHT ? 1 : B][4], v32[EIGHT ? 1 : B][4];
    uint32_t mq[B], vq[B];
    float ms[B], vs[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const int i = first + b * kStep, left = rest - i, low = at == 0 ? t.skip - i : 0;
        if (!VEC && left <= 0) continue;
        load4<VEC>(G, own + b * kStep, low, left, g[b]);
        if constexpr (MASTER) load4<VEC>(master, own + b * kStep, low, left, p[b]);
        else load4<VEC>(P, own + b * kStep, low, left, p[b]);
        if constexpr (EIGHT) {
            mq[b] = load_bytes<VEC>(M8, own + b * kStep, left);
            vq[b] = load_bytes<VEC>(V8, own + b * kStep, left);
            if constexpr (VEC) {
                const int block = (part * kPart<true> + i) / kKeepBlock;
                ms[b] = __shfl_sync(0xffffffffu, scales_m, block);
                vs[b] = __shfl_sync(0xffffffffu, scales_v, block);
            } else {
                ms[b] = keep_scale_of_byte(ME[(unsigned)i / kKeepBlock]);
                vs[b] = keep_scale_of_byte(VE[(unsigned)i / kKeepBlock]);
            }
        } else {
            load4<VEC>(M, own + b * kStep, low, left, m32[b]);
            load4<VEC>(V, own + b * kStep, low, left, v32[b]);
        }
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const int i = first + b * kStep, left = rest - i, low = at == 0 ? t.skip - i : 0;
        if (!VEC && left <= 0) continue;
        uint64_t m[2], v[2], root[2];
        if constexpr (EIGHT) {
            float f[4];
            taken4(mq[b], f);
#pragma unroll
            for (int k = 0; k < 2; ++k) m[k] = mul2(pairs_at(f, k), both(ms[b]));
            taken4(vq[b], f);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                v[k] = mul2(pairs_at(f, k), both(vs[b]));
                v[k] = mul2(v[k], v[k]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                m[k] = pairs_at(m32[b], k);
                v[k] = pairs_at(v32[b], k);
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint64_t x = mul2(pairs_at(g[b], k), number.grad_scale);
            m[k] = fma2(number.beta1, m[k], mul2(number.rest1, x));
            v[k] = fma2(number.beta2, v[k], mul2(number.rest2, mul2(x, x)));
            root[k] = pair_of(root_of<!EIGHT>(pair_lo(v[k])), root_of<!EIGHT>(pair_hi(v[k])));
            const uint64_t below = fma2(root[k], both(now.root_c2), number.eps);
            const uint64_t way = mul2(mul2(m[k], both(now.c1)), pair_of(inverse_of(pair_lo(below)), inverse_of(pair_hi(below))));
            const uint64_t was = pairs_at(p[b], k), is = fma2(both(-now.lr), fma2(both(t.weight_decay), was, way), was);
            p[b][2 * k] = pair_lo(is);
            p[b][2 * k + 1] = pair_hi(is);
        }
        if constexpr (MASTER) store4<VEC>(master, own + b * kStep, low, left, p[b]);
        store4<VEC>(P, own + b * kStep, low, left, p[b]);
        if constexpr (EIGHT) {
            const uint32_t top_m = largest_of(m), top_v = largest_of(v);
            uint32_t h[4];
            const uint32_t entry = (uint32_t)at + own + b * kStep;
#pragma unroll
            for (int j = 0; j < 4; ++j)   // (four entries from a multiple of four on differ in the lowest bits alone, which the first shift drops)
                h[j] = VEC ? mix_rest((now.seed ^ entry) ^ ((now.seed ^ entry) >> 16) ^ (uint32_t)j) : mix(now.seed ^ (entry + 32u * j));
            uint32_t q;
            const uint32_t me = keep_at_random<false>(m, m, top_m, h, &q);
            store_bytes<VEC>(M8, own + b * kStep, left, q);
            const uint32_t ve = keep_at_random<true>(root, v, top_v, h, &q);
            store_bytes<VEC>(V8, own + b * kStep, left, q);
            if constexpr (VEC) {
                keep_m |= me << (8 * (part * B + b));
                keep_v |= ve << (8 * (part * B + b));
            } else if (lane == 0) {
                t.ME[(at + i) / kKeepBlock] = (uint8_t)me;
                t.VE[(at + i) / kKeepBlock] = (uint8_t)ve;
            }
        } else {
            const float fm[4] = {pair_lo(m[0]), pair_hi(m[0]), pair_lo(m[1]), pair_hi(m[1])};
            const float fv[4] = {pair_lo(v[0]), pair_hi(v[0]), pair_lo(v[1]), pair_hi(v[1])};
            store4<VEC>(M, own + b * kStep, low, left, fm);
            store4<VEC>(V, own + b * kStep, low, left, fv);
        }
    }
}

// Tensors of any alignment, and the ends of all: a function of its own, since beside the other's its registers do not fit (5 to 80 words spilled)
template <bool EIGHT, typename PT, typename GT, bool MASTER>
__device__ __noinline__ void step_any(const Tensor& t, int64_t at, const Numbers& number, Now now) {
    for (int64_t end = at + kUnit<EIGHT>; at < end && at < t.n; at += kPart<EIGHT>) {
        uint32_t none = 0u;
        step_part<EIGHT, false, PT, GT, MASTER>(t, at, number, now, 0, 0.f, 0.f, none, none);
    }
}

template <bool EIGHT, typename PT, typename GT, bool MASTER, int CAP>
__global__ void __launch_bounds__(kThreads, kCtas) adamw_kernel(const __grid_constant__ Table<CAP> table, const __grid_constant__ Numbers number) {
    pdl_trigger();
    pdl_wait();
    float lr = number.lr, c1 = number.c1, root_c2 = number.root_c2;
    uint32_t step = number.step;
    if (number.lr_dev) lr = *number.lr_dev;
    if (number.step_dev) {
        const int64_t there = *number.step_dev, t = there < 1 ? 1 : there;
        step = (uint32_t)t;
        const float count = (float)t;
        // 1 - b^t = -(e^(t log b) - 1), without the difference's loss of bits (b = 0: log b = -Inf)
        c1 = 1.f / -expm1f(count * number.log_beta1);
        root_c2 = sqrtf(1.f / -expm1f(count * number.log_beta2));
    }
    Now now{lr, c1, root_c2, 0u};
    const uint32_t start = EIGHT ? mix(number.seed + 0x9e3779b9u * step) : 0u;
    const int64_t units = table.end[table.count - 1];
    int which = 0, turn = 0;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
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
        const int64_t at = (unit - (which ? table.end[which - 1] : 0)) * kUnit<EIGHT>;
        if (EIGHT) now.seed = mix(start + t.key);
        if (!t.vec || t.n - at < kUnit<EIGHT> || at < t.skip) {
            step_any<EIGHT, PT, GT, MASTER>(t, at, number, now);
        } else if constexpr (!EIGHT) {
            uint32_t none = 0u;
            step_part<false, true, PT, GT, MASTER>(t, at, number, now, 0, 0.f, 0.f, none, none);
        } else {
            // (written again two units on, and every thread has passed the barrier between)
            __shared__ uint32_t scales[2][2][kThreads / 32];
            uint32_t(*here)[kThreads / 32] = scales[turn & 1];
            ++turn;
            const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
            const int64_t block = at / kKeepBlock;
            const float scales_m = keep_scale_of_byte(t.ME[block + lane]), scales_v = keep_scale_of_byte(t.VE[block + lane]);
            uint32_t keep_m = 0u, keep_v = 0u;
#pragma unroll 1
            for (int part = 0; part < 2; ++part)
                step_part<true, true, PT, GT, MASTER>(t, at + part * kPart<true>, number, now, part, scales_m, scales_v, keep_m, keep_v);
            if (lane == 0) {
                here[0][warp] = keep_m;
                here[1][warp] = keep_v;
            }
            __syncthreads();
            // (byte i of a warp's word is that of block warp + i * warps)
            if (warp < 2) (warp == 0 ? t.ME : t.VE)[block + lane] = (uint8_t)(here[warp][lane % (kThreads / 32)] >> (8 * (lane / (kThreads / 32))));
        }
    }
}

uint64_t twice(double v) {
    const float f = (float)v;
    uint32_t w;
    memcpy(&w, &f, sizeof w);
    return ((uint64_t)w << 32) | w;
}

// how many entries of `size` bytes p lies behind the last place that is aligned for four of them
int behind(const void* p, int size) { return (int)(reinterpret_cast<uintptr_t>(p) / (uintptr_t)size % 4); }

// The tensors of one kind among those from *from on, as many as the table holds.
struct Kind {
    int p_dtype, g_dtype;
    bool master;
    bool operator==(const Kind& k) const { return p_dtype == k.p_dtype && g_dtype == k.g_dtype && master == k.master; }
};
Kind kind_of(const detox_adamw_tensor& t) { return Kind{t.p_dtype, t.g_dtype, t.master != nullptr}; }

template <bool EIGHT, typename PT, typename GT, bool MASTER, int CAP>
detox_status step_table(const Numbers& number, const Kind& kind, const detox_adamw_tensor* from, const detox_adamw_tensor* end, cudaStream_t s) {
    Table<CAP> table;
    while (from != end) {
        int64_t units = 0;
        int n = 0;
        for (; from != end && n < CAP; ++from) {
            if (from->n == 0 || !(kind_of(*from) == kind)) continue;
            const int ss = EIGHT ? 1 : 4, off = behind(from->P, sizeof(PT));
            const bool even = behind(from->G, sizeof(GT)) == off && (!MASTER || behind(from->master, 4) == off) && behind(from->M, ss) == off && behind(from->V, ss) == off;
            Tensor& t = table.of[n];
            // blocks of 8-bit states start with the tensor
            t.vec = even && (off == 0 || !EIGHT);
            t.skip = t.vec ? off : 0;
            t.P = static_cast<PT*>(from->P) - t.skip;
            t.G = static_cast<const GT*>(from->G) - t.skip;
            t.master = MASTER ? from->master - t.skip : nullptr;
            t.M = static_cast<char*>(from->M) - t.skip * ss;
            t.V = static_cast<char*>(from->V) - t.skip * ss;
            t.ME = from->ME; t.VE = from->VE;
            t.n = from->n + t.skip;
            t.weight_decay = from->weight_decay;
            t.key = from->key;
            units += ceil_div(t.n, (int64_t)kUnit<EIGHT>);
            table.end[n++] = units;
        }
        if (n == 0) break;
        table.count = n;
        const int64_t most = (int64_t)kSMs * kCtas;
        const detox_status st = launch_chained(adamw_kernel<EIGHT, PT, GT, MASTER, CAP>, (unsigned)(units < most ? units : most), kThreads, 0, 1, s, table, number);
        if (st != DETOX_OK) return st;
    }
    return DETOX_OK;
}
template <bool EIGHT, typename PT, typename GT, bool MASTER>
detox_status step_kind(const Numbers& number, const Kind& kind, const detox_adamw_tensor* from, const detox_adamw_tensor* end, cudaStream_t s) {
    return end - from <= kFew ? step_table<EIGHT, PT, GT, MASTER, kFew>(number, kind, from, end, s)
                              : step_table<EIGHT, PT, GT, MASTER, kMany>(number, kind, from, end, s);
}
template <bool EIGHT, typename PT>
detox_status step_types(const Numbers& number, const Kind& kind, const detox_adamw_tensor* from, const detox_adamw_tensor* end, cudaStream_t s) {
    if constexpr (sizeof(PT) == 4) {
        if (kind.master) return DETOX_ERR_UNSUPPORTED;
        if (kind.g_dtype == DETOX_DTYPE_FLOAT) return step_kind<EIGHT, PT, float, false>(number, kind, from, end, s);
        if (kind.g_dtype == DETOX_DTYPE_HALF) return step_kind<EIGHT, PT, __half, false>(number, kind, from, end, s);
        return step_kind<EIGHT, PT, __nv_bfloat16, false>(number, kind, from, end, s);
    } else {
        if (kind.g_dtype == DETOX_DTYPE_FLOAT)
            return kind.master ? step_kind<EIGHT, PT, float, true>(number, kind, from, end, s) : step_kind<EIGHT, PT, float, false>(number, kind, from, end, s);
        if (kind.g_dtype != kind.p_dtype) return DETOX_ERR_UNSUPPORTED;
        return kind.master ? step_kind<EIGHT, PT, PT, true>(number, kind, from, end, s) : step_kind<EIGHT, PT, PT, false>(number, kind, from, end, s);
    }
}
template <bool EIGHT>
detox_status step_types(const Numbers& number, const Kind& kind, const detox_adamw_tensor* from, const detox_adamw_tensor* end, cudaStream_t s) {
    if (kind.p_dtype == DETOX_DTYPE_FLOAT) return step_types<EIGHT, float>(number, kind, from, end, s);
    if (kind.p_dtype == DETOX_DTYPE_HALF) return step_types<EIGHT, __half>(number, kind, from, end, s);
    return step_types<EIGHT, __nv_bfloat16>(number, kind, from, end, s);
}

}  // namespace

detox_status launch_adamw(const detox_adamw_desc& d, const detox_adamw_tensor* tensors, int64_t count, cudaStream_t s) {
    Numbers number = {};
    number.lr = (float)d.lr;
    number.beta1 = twice(d.beta1); number.beta2 = twice(d.beta2);
    number.rest1 = twice(1.0 - d.beta1); number.rest2 = twice(1.0 - d.beta2);
    number.eps = twice(d.eps);
    number.grad_scale = twice(d.grad_scale);
    number.log_beta1 = (float)log(d.beta1); number.log_beta2 = (float)log(d.beta2);
    number.c1 = (float)(1.0 / (1.0 - pow(d.beta1, (double)d.step)));
    number.root_c2 = (float)sqrt(1.0 / (1.0 - pow(d.beta2, (double)d.step)));
    number.seed = d.seed;
    number.step = (uint32_t)d.step;
    number.lr_dev = d.lr_dev;
    number.step_dev = d.step_dev;
    const detox_adamw_tensor* end = tensors + count;
    Kind done[kKinds];
    int kinds = 0;
    for (const detox_adamw_tensor* t = tensors; t != end; ++t) {
        if (t->n == 0) continue;
        const Kind kind = kind_of(*t);
        bool seen = false;
        for (int i = 0; i < kinds; ++i) seen = seen || done[i] == kind;
        if (seen) continue;
        done[kinds++] = kind;
        const detox_status st = d.bits == 8 ? step_types<true>(number, kind, t, end, s) : step_types<false>(number, kind, t, end, s);
        if (st != DETOX_OK) return st;
    }
    return DETOX_OK;
}

}  // namespace detox
