// Token embedding: rows of a table, scaled, and the table's gradient.
//
// Lookup:    Y[t] = scale W[tokens[t]].  Bound by HBM; a warp takes 4 pieces of 16 bytes a lane of one row.  8192 x 4096 bf16 of 32000 rows: 16.7 us.
//
// Gradient:  dW[v] = scale sum of dY[t] over the rows t with tokens[t] = v.  Bound by HBM too (rows of dY read once, rows of dW
// written once), if the work is shared out evenly: tokens are as unevenly spread as words are, and a padded batch or a
// short vocabulary puts thousands of rows on one token.  No atomics: the order of the sums is fixed by sizes and tokens.
//   1. sort_tokens: a stable counting sort in one launch, without communication between CTAs.  Each of 2^k CTAs owns every 2^k-th row of the
//      vocabulary (neighbouring numbers are often equally frequent) and looks through all tokens, which lie in L2: it counts those of
//      the CTAs before it (where its output starts) and, warp by warp, those of each of its rows; then it goes through them again and writes the
//      row numbers in order.  (So all CTAs read all tokens, twice: 6 us for 8192, but 330 of 711 us for a million of them into 32000 x 64.)  The order of the tokens is that of their places: CTA by CTA, and in a CTA ascending.
//   2. sum_rows: the sorted tokens are cut into spans of equal length, whatever lies in them.  A warp has a span and a slice of the columns; it adds up
//      rows in registers and writes dW whenever the token changes.  The sum of a token that lies in several spans goes to the
//      workspace in parts, and the warp that leaves the last of them adds them, in the spans' order (a counter tells, so nobody waits).
//      Other CTAs of the same launch write zeros to the rows of tokens that do not occur.
// 8192 tokens, bf16, to 32000 x 2048 fp32: 61 to 63 us (floor 45): 6 of sorting, 50 of the second kernel at 5.8 TB/s.  Cut into spans of equal cost over tokens and rows of the table
// alike it took 123: adding is bound by latency, writing zeros by bandwidth, and a warp that does both in turn keeps neither busy.
#include "worker.cuh"

namespace detox {

namespace {

// ---- lookup -------------------------------------------------------------------------------------
constexpr int kThreads = 256;
constexpr int kPieces = 4;                     // 16-byte pieces of a lane

// LANES neighbouring lanes share a row's slice of LANES * kPieces pieces
template <typename T, typename I, int LANES, bool ANY>
__global__ void __launch_bounds__(kThreads) lookup_kernel(const T* __restrict__ W, int64_t ldw, Span span, int64_t vocab, int64_t cols,
                                                          int slices, const I* __restrict__ tokens, int64_t rows, float scale,
                                                          T* __restrict__ Y, int64_t ldy, bool y_vec) {
    constexpr int N = Piece<T>::N, kGroups = kThreads / LANES;
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x % LANES;
    const uint64_t scale2 = pair_of(scale, scale);
    for (int64_t item = (int64_t)blockIdx.x * kGroups + threadIdx.x / LANES; item < rows * slices; item += (int64_t)gridDim.x * kGroups) {
        const int64_t row = item / slices, c0 = (item - row * slices) * (LANES * kPieces * N) + lane * N;
        const int64_t token = (int64_t)tokens[row];
        const bool there = token >= 0 && token < vocab;
        const T* from = W + (there ? token : 0) * ldw;
        uint4 raw[kPieces];
#pragma unroll
        for (int i = 0; i < kPieces; ++i) raw[i] = load_piece<ANY>(from, c0 + i * LANES * N, there ? cols : (int64_t)0, span);
        const uint64_t factor = token < vocab ? scale2 : pair_of(__int_as_float(0x7fc00000), __int_as_float(0x7fc00000));
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            uint64_t f[N / 2];
            Piece<T>::split(raw[i], f);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) f[j] = mul2(f[j], factor);
            store_piece(Y + row * ldy, (int)(c0 + i * LANES * N), (int)cols, !ANY || y_vec, f);
        }
    }
}

// ---- the gradient's plan --------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32;
constexpr int kSortRows = kSortThreads;        // rows of the vocabulary that a CTA can own: a thread each
constexpr int kSumWarps = 48;                  // warps of an SM that there are spans for, where there are tokens enough
// Rows of dY that a warp has in flight; a span's length is a multiple.  With a gradient to add to, a warp waits for its row at every token, so spans are shorter
// where there are few tokens.
template <bool ADD> constexpr int kAhead = ADD ? 4 : 8;
constexpr int kSortAhead = 8;
constexpr int kManyTokens = 4096, kManyLength = 16;   // a frequent token of many has as many parts as spans, which one warp adds: fewer, longer ones (added to: 4097 x 64
// 23.3 -> 19.8 us, 6000 x 512 28.6 -> 22.4, 16384 x 64 52.4 -> 34.3, 30000 x 192 74.8 -> 58.3; overwritten: 40.8 -> 39.9 to 77.1 -> 56.1)
constexpr int kZeroPlaces = 32;                // places that a CTA looks after
constexpr int kZeroCtas = 6;                   // CTAs of an SM that there should be for that

// Place p is row (i << bits) + c of the vocabulary with c = p / per, i = p % per; a few at the ends of CTAs' stretches are none.
struct Places {
    int32_t vocab, per, bits;
    __host__ __device__ int32_t count() const { return per << bits; }
    __device__ __forceinline__ int64_t row(int32_t place) const {
        const int32_t c = place / per;
        return ((int64_t)(place - c * per) << bits) + c;
    }
};
struct Plan {
    int64_t rows, cols;
    Places places;
    int slices;                                // slices of 32 pieces
    int spans, length;                         // length: tokens of a span
    int64_t ldp;                               // pitch of the partial sums
    size_t order, sorted, starts, left, head, tail, bytes;   // offsets in the workspace
};
// `entries`: of a 16-byte piece
Plan plan_of(int64_t rows, int64_t vocab, int64_t cols, int entries, bool add) {
    const int ahead = add ? kAhead<true> : kAhead<false>;
    Plan p = {};
    p.rows = rows;
    p.cols = cols;
    int bits = 7;                              // 128 CTAs, more where a CTA's threads are too few for its rows
    while (((int64_t)kSortRows << bits) < vocab) ++bits;
    p.places = Places{(int32_t)vocab, (int32_t)ceil_div(vocab, (int64_t)1 << bits), bits};
    p.slices = (int)ceil_div(cols, (int64_t)32 * entries);
    p.ldp = ceil_div(cols, (int64_t)4) * 4;
    p.length = (int)(ceil_div(rows * p.slices, (int64_t)kSMs * kSumWarps * ahead) * ahead);
    if (p.length < ahead) p.length = ahead;
    if (rows > kManyTokens && p.length < kManyLength) p.length = kManyLength;
    p.spans = (int)ceil_div(rows, (int64_t)p.length);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t was = at; at = align_up(at + bytes); return was; };
    p.order = take((size_t)rows * 4);
    p.sorted = take((size_t)rows * 4);
    p.starts = take(((size_t)p.places.count() + 1) * 4);
    p.left = take((size_t)p.spans * (size_t)p.slices * 4);
    p.head = take((size_t)p.spans * (size_t)p.ldp * 4);
    p.tail = take((size_t)p.spans * (size_t)p.ldp * 4);
    p.bytes = at;
    return p;
}

// ---- 1. sorting -----------------------------------------------------------------------------------
// order: the rows by their tokens' places, those of a token ascending; sorted: those places; starts: where each place's rows start, and behind the
// last place how many there are (tokens outside the vocabulary are left out); left: counters for the next kernel, cleared.  Dynamic shared memory: per x (kSortWarps + 1) int32.
template <typename I>
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const I* __restrict__ tokens, int64_t rows, Places places,
                                                                   int32_t* __restrict__ order, int32_t* __restrict__ sorted,
                                                                   int32_t* __restrict__ starts, int32_t* __restrict__ left, int64_t counters) {
    extern __shared__ int32_t hist[];          // [row][warp], a column more so that threads stepping through their rows do not collide
    __shared__ int32_t sums[kSortWarps];
    __shared__ int32_t start_of[kSortRows];
    constexpr int kPitch = kSortWarps + 1;
    pdl_trigger();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, per = places.per;
    const int32_t own = (int32_t)blockIdx.x, mask = (1 << places.bits) - 1;
    for (int i = threadIdx.x; i < per * kPitch; i += kSortThreads) hist[i] = 0;
    pdl_wait();
    for (int64_t i = (int64_t)blockIdx.x * kSortThreads + threadIdx.x; i < counters; i += (int64_t)gridDim.x * kSortThreads) left[i] = 0;
    __syncthreads();
    // each warp has a stretch of the tokens
    const int64_t stretch = (rows + kSortWarps * 32 - 1) / (kSortWarps * 32) * 32;
    const int64_t begin = warp * stretch, end = begin + stretch < rows ? begin + stretch : rows;
    int32_t tok[kSortAhead];
    auto fetch = [&](int64_t t0) {
#pragma unroll
        for (int i = 0; i < kSortAhead; ++i) {
            const int64_t t = t0 + i * 32 + lane, token = t < end ? (int64_t)tokens[t] : -1;
            tok[i] = token >= 0 && token < places.vocab ? (int32_t)token : -1;
        }
    };
    int32_t below = 0;
    for (int64_t t0 = begin; t0 < end; t0 += 32 * kSortAhead) {
        fetch(t0);
#pragma unroll
        for (int i = 0; i < kSortAhead; ++i) {
            below += tok[i] >= 0 && (tok[i] & mask) < own;
            if (tok[i] >= 0 && (tok[i] & mask) == own) atomicAdd(&hist[(tok[i] >> places.bits) * kPitch + warp], 1);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) below += __shfl_xor_sync(0xffffffffu, below, o);
    if (lane == 0) sums[warp] = below;
    __syncthreads();
    below = sums[lane];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) below += __shfl_xor_sync(0xffffffffu, below, o);
    __syncthreads();
    // a thread for each row: counts to places within the row, and the row's total
    int32_t total = 0;
    if ((int)threadIdx.x < per) {
        int32_t* h = hist + threadIdx.x * kPitch;
#pragma unroll 8
        for (int w = 0; w < kSortWarps; ++w) {
            const int32_t n = h[w];
            h[w] = total;
            total += n;
        }
    }
    // exclusive sum over the rows
    int32_t upto = total;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int32_t x = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += x;
    }
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    int32_t before = lane < warp ? sums[lane] : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    start_of[threadIdx.x] = below + before + upto - total;
    if ((int)threadIdx.x < per) starts[own * per + threadIdx.x] = below + before + upto - total;
    if (threadIdx.x == kSortThreads - 1 && own == mask) starts[places.count()] = below + before + upto;
    __syncthreads();
    const bool again = end - begin > 32 * kSortAhead;   // (else they are still there)
    for (int64_t t0 = begin; t0 < end; t0 += 32 * kSortAhead) {
        if (again) fetch(t0);
#pragma unroll
        for (int i = 0; i < kSortAhead; ++i) {
            const bool mine = tok[i] >= 0 && (tok[i] & mask) == own;
            if (!__any_sync(0xffffffffu, mine)) continue;
            const int r = mine ? tok[i] >> places.bits : -1;
            const uint32_t peers = __match_any_sync(0xffffffffu, r);
            int32_t* h = hist + (mine ? r : 0) * kPitch + warp;
            const int32_t at = mine ? start_of[r] + *h + __popc(peers & ((1u << lane) - 1u)) : 0;
            __syncwarp();
            if (mine) {
                order[at] = (int32_t)(t0 + i * 32 + lane);
                sorted[at] = own * per + r;
                if (lane == __ffs(peers) - 1) *h += __popc(peers);
            }
            __syncwarp();
        }
    }
}

// ---- 2. sums --------------------------------------------------------------------------------------
struct SumRows {
    const void* dY;
    int64_t lddy;
    Span span;
    const int32_t *order, *sorted, *starts;
    Places places;
    int cols, slices, spans, length;
    unsigned sum_ctas, zero_splits;            // the CTAs behind them write zeros, so many to a stretch of places
    float scale;
    void* dW;
    int64_t lddw;
    bool w_vec;                                // 16-byte accesses to dW
    bool w_wide;                               // 32-byte stores
    int32_t* left;                             // for each span and slice: how many parts of the place that the span completes are there
    float *head, *tail;                        // parts: of the place that a span completes, of the one that goes on behind it
    int64_t ldp;
};

// N sums of a lane to entries c .. of a row: fp32, or rounded.  Eight fp32 sums leave in one 32-byte store: two of 16 bytes each fill half of every
// sector that they touch.  Rows that are not aligned go through the warp's `buffer`, so that its lanes store neighbouring entries (as each lane's own ones, one at a time, every
// store touches 32 sectors).  Whole warps call this.
template <typename D, int N>
__device__ __forceinline__ void store_sums(D* row, int c, int cols, bool vec, bool wide, const uint64_t (&p)[N / 2], float* buffer) {
    constexpr int M = Piece<D>::N;
    if (!vec) {
        const int lane = threadIdx.x % 32, c0 = c - lane * N;
#pragma unroll
        for (int j = 0; j < N / 2; ++j) *reinterpret_cast<uint64_t*>(buffer + lane * N + 2 * j) = p[j];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c0 + 32 * j + lane < cols) row[c0 + 32 * j + lane] = from_f32<D>(buffer[32 * j + lane]);
        __syncwarp();
        return;
    }
    if constexpr (sizeof(D) == 4 && N == 8) {
        if (wide && c + N <= cols) {
            asm volatile("st.global.cs.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(row + c), "l"(p[0]), "l"(p[1]), "l"(p[2]), "l"(p[3]) : "memory");
            return;
        }
    }
#pragma unroll
    for (int k = 0; k < N; k += M) {
        uint64_t part[M / 2];
#pragma unroll
        for (int j = 0; j < M / 2; ++j) part[j] = p[k / 2 + j];
        store_piece(row, c + k, cols, true, part);
    }
}
template <typename D, int N>
__device__ __forceinline__ void load_sums(const D* row, int c, int cols, bool vec, uint64_t (&p)[N / 2], float* buffer) {
    constexpr int M = Piece<D>::N;
    const int lane = threadIdx.x % 32, c0 = c - lane * N;
    if (vec && c0 + 32 * N <= cols) {          // (the same for all lanes)
#pragma unroll
        for (int k = 0; k < N; k += M) {
            uint64_t part[M / 2];
            Piece<D>::split(ld_stream_u4(row + c + k), part);
#pragma unroll
            for (int j = 0; j < M / 2; ++j) p[k / 2 + j] = part[j];
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) buffer[32 * j + lane] = c0 + 32 * j + lane < cols ? to_f32(row[c0 + 32 * j + lane]) : 0.f;
    __syncwarp();
#pragma unroll
    for (int j = 0; j < N / 2; ++j) p[j] = *reinterpret_cast<const uint64_t*>(buffer + lane * N + 2 * j);
    __syncwarp();
}

// N sums of a part, past L1 (another SM may have left them)
template <int N>
__device__ __forceinline__ void load_part(const float* row, int c, int cols, uint64_t (&p)[N / 2]) {
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (c + j < cols) x = __ldcg(reinterpret_cast<const float4*>(row + c + j));   // (cols: a multiple of 4)
        p[j / 2] = pair_of(x.x, x.y);
        p[j / 2 + 1] = pair_of(x.z, x.w);
    }
}

// zeros to one of `splits` stretches of the rows of kZeroPlaces places that have no tokens: 32 bytes a store, but for the ends of a stretch
template <typename D>
__device__ __forceinline__ void zero_rows(const SumRows& g, int64_t first, int split, int splits) {
    const int64_t place = first + threadIdx.x % 32;
    const int64_t row = place < g.places.count() ? g.places.row((int32_t)place) : g.places.vocab;
    uint32_t empty = __ballot_sync(0xffffffffu, row < g.places.vocab && g.starts[place] == g.starts[place + 1]);
    const int length = (g.cols + splits - 1) / splits, begin = split * length, end = begin + length < g.cols ? begin + length : g.cols;
    if (begin >= end) return;
    for (; empty; empty &= empty - 1) {
        D* to = static_cast<D*>(g.dW) + __shfl_sync(0xffffffffu, row, __ffs(empty) - 1) * g.lddw;
        const uintptr_t lo = reinterpret_cast<uintptr_t>(to + begin), hi = reinterpret_cast<uintptr_t>(to + end);
        uintptr_t from = (lo + 31) & ~(uintptr_t)31, until = hi & ~(uintptr_t)31;
        if (from > until) from = until = hi;   // (within 32 bytes)
        for (uintptr_t at = from + 32 * threadIdx.x; at < until; at += 32 * kThreads)
            asm volatile("st.global.cs.v4.b64 [%0], {%1, %1, %1, %1};" ::"l"(at), "l"(0ull) : "memory");
        const uintptr_t head = lo + sizeof(D) * threadIdx.x, tail = until + sizeof(D) * threadIdx.x;
        if (head < from) *reinterpret_cast<D*>(head) = from_f32<D>(0.f);
        if (tail < hi) *reinterpret_cast<D*>(tail) = from_f32<D>(0.f);
    }
}

template <typename T, typename D, bool ADD, bool ANY>
__global__ void __launch_bounds__(kThreads, 3) sum_rows_kernel(const __grid_constant__ SumRows g) {
    constexpr int N = Piece<T>::N;
    pdl_trigger();
    pdl_wait();
    if (!ADD && blockIdx.x >= g.sum_ctas) {
        const unsigned k = blockIdx.x - g.sum_ctas;
        zero_rows<D>(g, (int64_t)(k / g.zero_splits) * kZeroPlaces, (int)(k % g.zero_splits), (int)g.zero_splits);
        return;
    }
    __shared__ __align__(16) float buffers[kThreads / 32][32 * N];
    float* buffer = buffers[threadIdx.x / 32];
    const int lane = threadIdx.x % 32;
    const int warp = blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    const int span = warp / g.slices, slice = warp - span * g.slices;
    if (span >= g.spans) return;
    const int32_t n = g.starts[g.places.count()], from = span * g.length;
    const int32_t to = from + g.length < n ? from + g.length : n;
    if (from >= to) return;
    int32_t place = g.sorted[from];
    const bool open = from > 0 && g.sorted[from - 1] == place, goes_on = to < n && g.sorted[to] == g.sorted[to - 1];
    const int c = (slice * 32 + lane) * N;
    const T* dY = static_cast<const T*>(g.dY) + c;
    D* dW = static_cast<D*>(g.dW);
    uint64_t acc[N / 2];
#pragma unroll
    for (int j = 0; j < N / 2; ++j) acc[j] = 0ull;
    const uint64_t scale2 = pair_of(g.scale, g.scale);
    bool head = open;
    int64_t row = 0;                           // of dW, for `place`
    auto write = [&] {
        D* at = dW + row * g.lddw;
#pragma unroll
        for (int j = 0; j < N / 2; ++j) acc[j] = mul2(acc[j], scale2);
        if constexpr (ADD) {
            uint64_t old[N / 2];
            load_sums<D, N>(at, c, g.cols, g.w_vec, old, buffer);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) acc[j] = add2(acc[j], old[j]);
        }
        store_sums<D, N>(at, c, g.cols, g.w_vec, g.w_wide, acc, buffer);
    };
    // a part of a place's sum is complete; the warp that leaves the last one adds them all
    auto part = [&](float* to) {
        store_sums<float, N>(to + (int64_t)span * g.ldp, c, (int)g.ldp, true, false, acc, buffer);
        const int first = g.starts[place] / g.length, last = (g.starts[place + 1] - 1) / g.length;
        __threadfence();
        __syncwarp();
        int before = 0;
        if (lane == 0) before = atomicAdd(&g.left[(int64_t)last * g.slices + slice], 1);
        if (__shfl_sync(0xffffffffu, before, 0) < last - first) return;
        __threadfence();
#pragma unroll
        for (int j = 0; j < N / 2; ++j) acc[j] = 0ull;
#pragma unroll 8
        for (int s = first; s <= last; ++s) {
            uint64_t x[N / 2];
            load_part<N>((s < last ? g.tail : g.head) + (int64_t)s * g.ldp, c, (int)g.ldp, x);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) acc[j] = add2(acc[j], x[j]);
        }
        write();
    };
    // the sum of a place is complete here
    auto close = [&] {
        if (head) part(g.head);
        else write();
        head = false;
#pragma unroll
        for (int j = 0; j < N / 2; ++j) acc[j] = 0ull;
    };
    int32_t order = 0, its_place = 0;          // of 32 tokens, one a lane
    int64_t its_row = 0;
    for (int32_t k = from; k < to; k += kAhead<ADD>) {
        const int at = (k - from) & 31;
        if (at == 0) {
            const bool there = k + lane < to;
            order = there ? g.order[k + lane] : 0;
            its_place = there ? g.sorted[k + lane] : -1;
            its_row = there ? g.places.row(its_place) : 0;
        }
        uint4 raw[kAhead<ADD>];
#pragma unroll
        for (int i = 0; i < kAhead<ADD>; ++i)
            raw[i] = load_piece<ANY>(dY + (int64_t)__shfl_sync(0xffffffffu, order, at + i) * g.lddy, 0, k + i < to ? g.cols - c : 0, g.span);
#pragma unroll
        for (int i = 0; i < kAhead<ADD>; ++i) {
            const int32_t p = __shfl_sync(0xffffffffu, its_place, at + i);
            const int64_t r = __shfl_sync(0xffffffffu, its_row, at + i);
            if (p >= 0 && p != place) {
                close();
                place = p;
            }
            if (p >= 0) row = r;
            uint64_t f[N / 2];
            Piece<T>::split(raw[i], f);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) acc[j] = add2(acc[j], f[j]);
        }
    }
    if (goes_on) part(g.tail);
    else close();
}

template <typename T, typename I, int LANES>
detox_status lookup(const T* W, int64_t ldw, int64_t vocab, int64_t cols, const I* tokens, int64_t rows, float scale, T* Y, int64_t ldy,
                    cudaStream_t s) {
    constexpr int N = Piece<T>::N;
    const Span span = span_of<T>(W, ldw, vocab, cols);
    const bool y_vec = aligned16(Y) && ldy % N == 0;
    const int slices = (int)ceil_div(cols, (int64_t)LANES * kPieces * N);
    const int64_t need = ceil_div(rows * slices, (int64_t)(kThreads / LANES)), most = (int64_t)kSMs * 16;
    return launch_chained(cols % N == 0 && span.vec && y_vec ? lookup_kernel<T, I, LANES, false> : lookup_kernel<T, I, LANES, true>,
                          (unsigned)(need < most ? need : most), kThreads, 0, 1, s, W, ldw, span, vocab, cols, slices, tokens, rows, scale, Y,
                          ldy, y_vec);
}
template <typename T>
detox_status lookup(const void* W, int64_t ldw, int64_t vocab, int64_t cols, int index, const void* tokens, int64_t rows, float scale,
                    void* Y, int64_t ldy, cudaStream_t s) {
    const T* w = static_cast<const T*>(W);
    T* y = static_cast<T*>(Y);
    const bool narrow = cols <= 8 * kPieces * Piece<T>::N;   // eight lanes have room for a row
    if (index == DETOX_INDEX_INT32) {
        const int32_t* t = static_cast<const int32_t*>(tokens);
        return narrow ? lookup<T, int32_t, 8>(w, ldw, vocab, cols, t, rows, scale, y, ldy, s)
                      : lookup<T, int32_t, 32>(w, ldw, vocab, cols, t, rows, scale, y, ldy, s);
    }
    const int64_t* t = static_cast<const int64_t*>(tokens);
    return narrow ? lookup<T, int64_t, 8>(w, ldw, vocab, cols, t, rows, scale, y, ldy, s)
                  : lookup<T, int64_t, 32>(w, ldw, vocab, cols, t, rows, scale, y, ldy, s);
}

template <typename I>
detox_status sort_tokens(const void* tokens, const Plan& p, char* ws, cudaStream_t s) {
    const size_t smem = (size_t)p.places.per * (kSortWarps + 1) * sizeof(int32_t);
    if (smem > 40 * 1024 && cudaFuncSetAttribute(sort_tokens_kernel<I>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
        cudaGetLastError();
        return DETOX_ERR_CUDA;
    }
    return launch_chained(sort_tokens_kernel<I>, 1u << p.places.bits, kSortThreads, smem, 1, s, static_cast<const I*>(tokens), p.rows, p.places,
                          reinterpret_cast<int32_t*>(ws + p.order), reinterpret_cast<int32_t*>(ws + p.sorted),
                          reinterpret_cast<int32_t*>(ws + p.starts), reinterpret_cast<int32_t*>(ws + p.left), (int64_t)p.spans * p.slices);
}

template <typename T, typename D, bool ADD>
detox_status sums(const void* dY, int64_t lddy, float scale, void* dW, int64_t lddw, const Plan& p, char* ws, cudaStream_t s) {
    SumRows g;
    g.dY = dY; g.lddy = lddy;
    g.span = span_of<T>(dY, lddy, p.rows, p.cols);
    g.order = reinterpret_cast<int32_t*>(ws + p.order);
    g.sorted = reinterpret_cast<int32_t*>(ws + p.sorted);
    g.starts = reinterpret_cast<int32_t*>(ws + p.starts);
    g.places = p.places;
    g.cols = (int)p.cols; g.slices = p.slices; g.spans = p.spans; g.length = p.length;
    g.scale = scale;
    g.dW = dW; g.lddw = lddw;
    g.w_vec = aligned16(dW) && lddw % Piece<D>::N == 0;
    g.w_wide = aligned_to(dW, 32) && lddw * (int64_t)sizeof(D) % 32 == 0;
    g.left = reinterpret_cast<int32_t*>(ws + p.left);
    g.head = reinterpret_cast<float*>(ws + p.head);
    g.tail = reinterpret_cast<float*>(ws + p.tail);
    g.ldp = p.ldp;
    const bool any = !(p.cols % Piece<T>::N == 0 && g.span.vec);
    g.sum_ctas = (unsigned)ceil_div((int64_t)p.spans * p.slices, (int64_t)(kThreads / 32));
    // few places: several CTAs to a row, as long as each has a store for all its threads
    const int64_t stretches = ceil_div((int64_t)p.places.count(), (int64_t)kZeroPlaces), wide = ceil_div(p.cols * (int64_t)sizeof(D), (int64_t)32 * kThreads);
    const int64_t splits = ceil_div((int64_t)kSMs * kZeroCtas, stretches);
    g.zero_splits = (unsigned)(splits < wide ? splits : wide);
    const unsigned grid = g.sum_ctas + (ADD ? 0u : (unsigned)stretches * g.zero_splits);
    if (grid == 0) return DETOX_OK;
    return launch_chained(any ? sum_rows_kernel<T, D, ADD, true> : sum_rows_kernel<T, D, ADD, false>, grid, kThreads, 0, 1, s, g);
}
template <typename T>
detox_status sums(const void* dY, int64_t lddy, float scale, void* dW, int64_t lddw, bool wide, bool add, const Plan& p, char* ws,
                  cudaStream_t s) {
    if (wide) return add ? sums<T, float, true>(dY, lddy, scale, dW, lddw, p, ws, s) : sums<T, float, false>(dY, lddy, scale, dW, lddw, p, ws, s);
    return add ? sums<T, T, true>(dY, lddy, scale, dW, lddw, p, ws, s) : sums<T, T, false>(dY, lddy, scale, dW, lddw, p, ws, s);
}

}  // namespace

detox_status launch_embedding(int dtype, const void* W, int64_t ldw, int64_t vocab, int64_t cols, int index, const void* tokens,
                              int64_t rows, float scale, void* Y, int64_t ldy, cudaStream_t s) {
    if (rows == 0) return DETOX_OK;
    if (dtype == DETOX_DTYPE_FLOAT) return lookup<float>(W, ldw, vocab, cols, index, tokens, rows, scale, Y, ldy, s);
    if (dtype == DETOX_DTYPE_HALF) return lookup<__half>(W, ldw, vocab, cols, index, tokens, rows, scale, Y, ldy, s);
    return lookup<__nv_bfloat16>(W, ldw, vocab, cols, index, tokens, rows, scale, Y, ldy, s);
}

size_t embedding_backward_ws_bytes(int64_t rows, int64_t vocab, int64_t cols) {
    // (the larger of any type's; with `add` the spans are shorter, and more)
    const size_t a = plan_of(rows, vocab, cols, Piece<__half>::N, true).bytes, b = plan_of(rows, vocab, cols, Piece<float>::N, true).bytes;
    return a > b ? a : b;
}

detox_status launch_embedding_backward(int dtype, const void* dY, int64_t lddy, int index, const void* tokens, int64_t rows, int64_t vocab,
                                       int64_t cols, float scale, void* dW, int64_t lddw, int dw_dtype, bool add, void* ws, cudaStream_t s) {
    if (rows == 0 && add) return DETOX_OK;
    const Plan p = plan_of(rows, vocab, cols, dtype == DETOX_DTYPE_FLOAT ? Piece<float>::N : Piece<__half>::N, add);
    char* at = static_cast<char*>(ws);
    const detox_status st = index == DETOX_INDEX_INT32 ? sort_tokens<int32_t>(tokens, p, at, s) : sort_tokens<int64_t>(tokens, p, at, s);
    if (st != DETOX_OK) return st;
    const bool wide = dw_dtype == DETOX_DTYPE_FLOAT;
    if (dtype == DETOX_DTYPE_FLOAT) return sums<float>(dY, lddy, scale, dW, lddw, wide, add, p, at, s);
    if (dtype == DETOX_DTYPE_HALF) return sums<__half>(dY, lddy, scale, dW, lddw, wide, add, p, at, s);
    return sums<__nv_bfloat16>(dY, lddy, scale, dW, lddw, wide, add, p, at, s);
}

}  // namespace detox
