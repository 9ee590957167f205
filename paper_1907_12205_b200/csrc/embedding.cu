// Token embedding: rows of a table, scaled, and the table's gradient.
//
// Lookup:    Y[t] = scale W[tokens[t]].  Bound by HBM; a warp takes 4 pieces of 16 bytes a lane of one row.
//
// Gradient:  dW[v] = scale sum of dY[t] over the rows t with tokens[t] = v.  Bound by HBM too (rows of dY read once, rows of dW
// written once), if the work is shared out evenly: tokens are as unevenly spread as words are, and a padded batch or a
// short vocabulary puts thousands of rows on one token.  No atomics: the order of the sums is fixed by sizes and tokens.
//   1. sort_tokens: a stable counting sort in one launch, without communication between CTAs.  Each CTA owns a range of the
//      vocabulary and looks through all tokens, which lie in L2: it counts those below its range (where its output starts) and, warp by
//      warp, those of each of its rows; then it goes through them again and writes the row numbers in order.
//   2. sum_rows: the path that takes a step for every token (a row of dY read) and one for every row of the vocabulary (a row of dW
//      written), in sorted order, is cut into spans of equal cost.  A warp has a span and a slice of the columns; it adds up
//      rows in registers and writes dW whenever the token changes.  The sum of a token that lies in several spans goes to the
//      workspace in parts:
//   3. join_spans: adds those, span by span.
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
constexpr int kSpanWarps = 32;                 // resident warps of an SM that the spans are cut for
constexpr int kJoinThreads = 256;

struct Plan {
    int64_t rows, vocab, cols;
    int slices;                                // slices of 32 pieces
    int spans;
    int64_t ldp;                               // pitch of the partial sums
    size_t order, sorted, counted, info, head, tail, bytes;   // offsets in the workspace
};
// `entries`: of a 16-byte piece
Plan plan_of(int64_t rows, int64_t vocab, int64_t cols, int entries) {
    Plan p{rows, vocab, cols, (int)ceil_div(cols, (int64_t)32 * entries), 1, ceil_div(cols, (int64_t)4) * 4, 0, 0, 0, 0, 0, 0, 0};
    int64_t spans = (int64_t)kSMs * kSpanWarps / p.slices;
    if (spans < 1) spans = 1;
    if (spans > rows + vocab) spans = rows + vocab;
    p.spans = (int)spans;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t was = at; at = align_up(at + bytes); return was; };
    p.order = take((size_t)rows * 4);
    p.sorted = take((size_t)rows * 4);
    p.counted = take(4);
    p.info = take((size_t)p.spans * 8);
    p.head = take((size_t)p.spans * (size_t)p.ldp * 4);
    p.tail = take((size_t)p.spans * (size_t)p.ldp * 4);
    p.bytes = at;
    return p;
}

// ---- 1. sorting -----------------------------------------------------------------------------------
// order: the rows by token, those of a token ascending; sorted: their tokens; counted: how many there are (tokens outside the
// vocabulary are left out).  CTA b owns [b per, (b + 1) per).  Dynamic shared memory: per x (kSortWarps + 1) int32.
template <typename I>
__global__ void __launch_bounds__(kSortThreads) sort_tokens_kernel(const I* __restrict__ tokens, int64_t rows, int64_t vocab, int per,
                                                                   int32_t* __restrict__ order, int32_t* __restrict__ sorted,
                                                                   int32_t* __restrict__ counted) {
    extern __shared__ int32_t hist[];          // [row][warp], a column more so that threads stepping through their rows do not collide
    __shared__ int32_t sums[kSortWarps];
    __shared__ int32_t start_of[kSortRows];
    constexpr int kPitch = kSortWarps + 1, kAhead = 8;
    pdl_trigger();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int64_t v0 = (int64_t)blockIdx.x * per, v1 = v0 + per < vocab ? v0 + per : vocab;
    for (int i = threadIdx.x; i < per * kPitch; i += kSortThreads) hist[i] = 0;
    pdl_wait();
    __syncthreads();
    // each warp has a stretch of the tokens
    const int64_t stretch = (rows + kSortWarps * 32 - 1) / (kSortWarps * 32) * 32;
    const int64_t begin = warp * stretch, end = begin + stretch < rows ? begin + stretch : rows;
    int32_t below = 0;
    for (int64_t t0 = begin; t0 < end; t0 += 32 * kAhead) {
        int64_t tok[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t t = t0 + i * 32 + lane;
            tok[i] = t < end ? (int64_t)tokens[t] : -1;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            below += tok[i] >= 0 && tok[i] < v0;
            if (tok[i] >= v0 && tok[i] < v1) atomicAdd(&hist[(int)(tok[i] - v0) * kPitch + warp], 1);
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
    if (threadIdx.x == kSortThreads - 1 && v1 == vocab && v0 < vocab) *counted = below + before + upto;
    __syncthreads();
    for (int64_t t0 = begin; t0 < end; t0 += 32 * kAhead) {
        int64_t tok[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t t = t0 + i * 32 + lane;
            tok[i] = t < end ? (int64_t)tokens[t] : -1;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const bool own = tok[i] >= v0 && tok[i] < v1;
            if (!__any_sync(0xffffffffu, own)) continue;
            const int r = own ? (int)(tok[i] - v0) : -1;
            const uint32_t peers = __match_any_sync(0xffffffffu, r);
            int32_t* h = hist + (own ? r : 0) * kPitch + warp;
            const int32_t at = own ? start_of[r] + *h + __popc(peers & ((1u << lane) - 1u)) : 0;
            __syncwarp();
            if (own) {
                order[at] = (int32_t)(t0 + i * 32 + lane);
                sorted[at] = (int32_t)tok[i];
                if (lane == __ffs(peers) - 1) *h += __popc(peers);
            }
            __syncwarp();
        }
    }
}

// ---- 2. sums --------------------------------------------------------------------------------------
// Where the path of steps is cut: `rows` tokens of the sorted list are behind the cut, and the rows of dW below `v` are written; row v is
// open when some of its tokens are behind the cut already.
struct Cut {
    int32_t k, v;
    bool open;
};
// The cut at cost `at`: a token costs `b`, a row of dW `a`.  (a = 0: only rows with tokens count, with their tokens.)
// All lanes of a warp call this, each looking at a 32nd of the range.
__device__ __forceinline__ Cut cut_at(const int32_t* __restrict__ sorted, int32_t n, int32_t vocab, int64_t at, int a, int b, int lane) {
    // the first k with a sorted[k] + b k >= at
    int32_t lo = 0, hi = n;
    while (hi > lo) {
        const int32_t step = (hi - lo + 31) / 32, k = lo + lane * step;
        const bool less = k < hi && (int64_t)a * sorted[k] + (int64_t)b * k < at;
        const int below = __popc(__ballot_sync(0xffffffffu, less));   // the first `below` probes are
        if (below == 0) hi = lo;
        else {
            const int32_t next = lo + below * step;
            lo += (below - 1) * step + 1;
            hi = next < hi ? next : hi;
        }
    }
    const int32_t last = lo > 0 ? sorted[lo - 1] : 0, next = lo < n ? sorted[lo] : vocab;
    int64_t v = a > 0 ? (at - (int64_t)b * lo) / a : next;
    v = v < last ? last : (v > next ? next : v);
    return Cut{lo, (int32_t)v, lo > 0 && v < vocab && last == (int32_t)v};
}

struct SumRows {
    const void* dY;
    int64_t lddy;
    Span span;
    const int32_t *order, *sorted, *counted;
    int32_t vocab;
    int cols, slices, spans;
    int a, b;
    float scale;
    void* dW;
    int64_t lddw;
    bool w_vec;                                // 16-byte accesses to dW
    int32_t* info;                             // of each span: the row that was open at its start (or -1), the row at its end
    float *head, *tail;
    int64_t ldp;
};

// N sums of a lane to `to` (entries c .. of a row): fp32, or rounded
template <typename D, int N>
__device__ __forceinline__ void store_sums(D* row, int c, int cols, bool vec, const uint64_t (&p)[N / 2]) {
    if constexpr (sizeof(D) == 4 && N == 8) {
        if (vec && c + N <= cols) {
            float4* to = reinterpret_cast<float4*>(row + c);
            __stcs(to, make_float4(pair_lo(p[0]), pair_hi(p[0]), pair_lo(p[1]), pair_hi(p[1])));
            __stcs(to + 1, make_float4(pair_lo(p[2]), pair_hi(p[2]), pair_lo(p[3]), pair_hi(p[3])));
            return;
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c + j < cols) row[c + j] = j & 1 ? pair_hi(p[j / 2]) : pair_lo(p[j / 2]);
    } else {
        store_piece(row, c, cols, vec, p);
    }
}
template <typename D, int N>
__device__ __forceinline__ void load_sums(const D* row, int c, int cols, bool vec, uint64_t (&p)[N / 2]) {
    if constexpr (Piece<D>::N == N) {
        if (vec && c + N <= cols) {
            Piece<D>::split(ld_stream_u4(row + c), p);
            return;
        }
    }
    if constexpr (sizeof(D) == 4 && N == 8) {
        if (vec && c + N <= cols) {
            const float4 x = ld_stream_f4(row + c), y = ld_stream_f4(row + c + 4);
            p[0] = pair_of(x.x, x.y); p[1] = pair_of(x.z, x.w); p[2] = pair_of(y.x, y.y); p[3] = pair_of(y.z, y.w);
            return;
        }
    }
    float f[N];
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = c + j < cols ? to_f32(row[c + j]) : 0.f;
#pragma unroll
    for (int j = 0; j < N / 2; ++j) p[j] = pair_of(f[2 * j], f[2 * j + 1]);
}

template <typename T, typename D, bool ADD, bool ANY>
__global__ void __launch_bounds__(kThreads) sum_rows_kernel(const __grid_constant__ SumRows g) {
    constexpr int N = Piece<T>::N, kAhead = 8;
    pdl_trigger();
    pdl_wait();
    const int lane = threadIdx.x % 32;
    const int warp = blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    const int span = warp / g.slices, slice = warp - span * g.slices;
    if (span >= g.spans) return;
    const int32_t n = *g.counted;
    const int64_t cost = (int64_t)g.a * g.vocab + (int64_t)g.b * n;
    const Cut from = cut_at(g.sorted, n, g.vocab, cost / g.spans * span + cost % g.spans * span / g.spans, g.a, g.b, lane);
    Cut to{n, g.vocab, false};
    if (span + 1 < g.spans)
        to = cut_at(g.sorted, n, g.vocab, cost / g.spans * (span + 1) + cost % g.spans * (span + 1) / g.spans, g.a, g.b, lane);
    if (slice == 0 && lane == 0) {
        g.info[2 * span] = from.open ? from.v : -1;
        g.info[2 * span + 1] = to.v;
    }
    const int c = (slice * 32 + lane) * N;
    const T* dY = static_cast<const T*>(g.dY);
    uint64_t acc[N / 2];
    auto clear = [&] {
#pragma unroll
        for (int j = 0; j < N / 2; ++j) acc[j] = 0ull;
    };
    clear();
    const uint64_t scale2 = pair_of(g.scale, g.scale);
    int32_t v = from.v;
    bool any = from.open;                      // row v has tokens
    // row v is complete, and there are no tokens for those between it and `next`
    auto close = [&](int32_t next) {
        D* row = static_cast<D*>(g.dW) + (int64_t)v * g.lddw;
        if (from.open && v == from.v) {
            store_sums<float, N>(g.head + (int64_t)span * g.ldp, c, (int)g.ldp, true, acc);
        } else if (!ADD || any) {
#pragma unroll
            for (int j = 0; j < N / 2; ++j) acc[j] = mul2(acc[j], scale2);
            if constexpr (ADD) {
                uint64_t old[N / 2];
                load_sums<D, N>(row, c, g.cols, g.w_vec, old);
#pragma unroll
                for (int j = 0; j < N / 2; ++j) acc[j] = add2(acc[j], old[j]);
            }
            store_sums<D, N>(row, c, g.cols, g.w_vec, acc);
        }
        clear();
        any = false;
        if constexpr (!ADD) {
            for (++v, row += g.lddw; v < next; ++v, row += g.lddw) store_sums<D, N>(row, c, g.cols, g.w_vec, acc);
        }
        v = next;
    };
    int32_t order = 0, token = 0;              // of 32 tokens, one a lane
    for (int32_t k = from.k; k < to.k; k += kAhead) {
        const int at = (k - from.k) & 31;
        if (at == 0) {
            const bool there = k + lane < to.k;
            order = there ? g.order[k + lane] : 0;
            token = there ? g.sorted[k + lane] : 0;
        }
        uint4 raw[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int32_t row = __shfl_sync(0xffffffffu, order, at + i);
            raw[i] = load_piece<ANY>(dY + (int64_t)row * g.lddy, c, k + i < to.k ? g.cols : 0, g.span);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int32_t t = __shfl_sync(0xffffffffu, token, at + i);
            if (k + i >= to.k) break;
            if (t != v) close(t);
            any = true;
            uint64_t f[N / 2];
            Piece<T>::split(raw[i], f);
#pragma unroll
            for (int j = 0; j < N / 2; ++j) acc[j] = add2(acc[j], f[j]);
        }
    }
    if (v < to.v) close(to.v);
    if (to.open) store_sums<float, N>(g.tail + (int64_t)span * g.ldp, c, (int)g.ldp, true, acc);
}

// ---- 3. tokens that lie in several spans -----------------------------------------------------------
// A CTA for each span that completes a row which was open at its start: the sum of the earlier spans' parts and its own.
template <typename D, bool ADD>
__global__ void __launch_bounds__(kJoinThreads) join_spans_kernel(const int32_t* __restrict__ info, const float* __restrict__ head,
                                                                  const float* __restrict__ tail, int64_t ldp, int cols, float scale,
                                                                  D* __restrict__ dW, int64_t lddw) {
    pdl_trigger();
    pdl_wait();
    const int span = blockIdx.x, lane = threadIdx.x % 32;
    const int32_t v = info[2 * span];
    if (v < 0 || info[2 * span + 1] <= v) return;
    // the first span with a part: the last one before this at whose start the row was not open
    int first = span;
    for (bool more = true; more && first > 0;) {
        const int s = first - 1 - lane;
        const uint32_t began = __ballot_sync(0xffffffffu, s < 0 || info[2 * s] != v);
        more = began == 0;
        first -= more ? 32 : __ffs(began);
    }
    if (first < 0) first = 0;
    for (int c = threadIdx.x * 4; c < cols; c += kJoinThreads * 4) {
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int s = first; s < span; ++s) {
            const float4 x = *reinterpret_cast<const float4*>(tail + (int64_t)s * ldp + c);
            sum.x += x.x; sum.y += x.y; sum.z += x.z; sum.w += x.w;
        }
        const float4 x = *reinterpret_cast<const float4*>(head + (int64_t)span * ldp + c);
        const float f[4] = {sum.x + x.x, sum.y + x.y, sum.z + x.z, sum.w + x.w};
        D* to = dW + (int64_t)v * lddw + c;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (c + j < cols) to[j] = from_f32<D>(ADD ? fmaf(f[j], scale, to_f32(to[j])) : f[j] * scale);
    }
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
    // as many CTAs as SMs, more where a CTA's threads are too few for its rows
    const int64_t least = ceil_div(p.vocab, (int64_t)kSortRows);
    const int64_t ctas = p.vocab < kSMs ? p.vocab : (least > kSMs ? least : kSMs);
    const int per = (int)ceil_div(p.vocab, ctas);
    const size_t smem = (size_t)per * (kSortWarps + 1) * sizeof(int32_t);
    if (smem > 40 * 1024 && cudaFuncSetAttribute(sort_tokens_kernel<I>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) {
        cudaGetLastError();
        return DETOX_ERR_CUDA;
    }
    return launch_chained(sort_tokens_kernel<I>, (unsigned)ceil_div(p.vocab, (int64_t)per), kSortThreads, smem, 1, s,
                          static_cast<const I*>(tokens), p.rows, p.vocab, per, reinterpret_cast<int32_t*>(ws + p.order),
                          reinterpret_cast<int32_t*>(ws + p.sorted), reinterpret_cast<int32_t*>(ws + p.counted));
}

template <typename T, typename D, bool ADD>
detox_status sums(const void* dY, int64_t lddy, float scale, void* dW, int64_t lddw, const Plan& p, char* ws, cudaStream_t s) {
    SumRows g;
    g.dY = dY; g.lddy = lddy;
    g.span = span_of<T>(dY, lddy, p.rows, p.cols);
    g.order = reinterpret_cast<int32_t*>(ws + p.order);
    g.sorted = reinterpret_cast<int32_t*>(ws + p.sorted);
    g.counted = reinterpret_cast<int32_t*>(ws + p.counted);
    g.vocab = (int32_t)p.vocab;
    g.cols = (int)p.cols; g.slices = p.slices; g.spans = p.spans;
    g.a = ADD ? 0 : (int)sizeof(D);
    g.b = (int)sizeof(T);
    g.scale = scale;
    g.dW = dW; g.lddw = lddw;
    g.w_vec = aligned16(dW) && lddw % Piece<D>::N == 0;
    g.info = reinterpret_cast<int32_t*>(ws + p.info);
    g.head = reinterpret_cast<float*>(ws + p.head);
    g.tail = reinterpret_cast<float*>(ws + p.tail);
    g.ldp = p.ldp;
    const bool any = !(p.cols % Piece<T>::N == 0 && g.span.vec);
    const unsigned grid = (unsigned)ceil_div((int64_t)p.spans * p.slices, (int64_t)(kThreads / 32));
    const detox_status st = launch_chained(any ? sum_rows_kernel<T, D, ADD, true> : sum_rows_kernel<T, D, ADD, false>, grid, kThreads, 0, 1, s, g);
    if (st != DETOX_OK) return st;
    return launch_chained(join_spans_kernel<D, ADD>, (unsigned)p.spans, kJoinThreads, 0, 1, s, g.info, g.head, g.tail, p.ldp, (int)p.cols, scale,
                          static_cast<D*>(dW), lddw);
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
    // (whatever the type: 16-bit rows have fewer slices and with them more spans)
    return plan_of(rows, vocab, cols, Piece<__half>::N).bytes;
}

detox_status launch_embedding_backward(int dtype, const void* dY, int64_t lddy, int index, const void* tokens, int64_t rows, int64_t vocab,
                                       int64_t cols, float scale, void* dW, int64_t lddw, int dw_dtype, bool add, void* ws, cudaStream_t s) {
    if (rows == 0 && add) return DETOX_OK;
    const Plan p = plan_of(rows, vocab, cols, dtype == DETOX_DTYPE_FLOAT ? Piece<float>::N : Piece<__half>::N);
    char* at = static_cast<char*>(ws);
    const detox_status st = index == DETOX_INDEX_INT32 ? sort_tokens<int32_t>(tokens, p, at, s) : sort_tokens<int64_t>(tokens, p, at, s);
    if (st != DETOX_OK) return st;
    const bool wide = dw_dtype == DETOX_DTYPE_FLOAT;
    if (dtype == DETOX_DTYPE_FLOAT) return sums<float>(dY, lddy, scale, dW, lddw, wide, add, p, at, s);
    if (dtype == DETOX_DTYPE_HALF) return sums<__half>(dY, lddy, scale, dW, lddw, wide, add, p, at, s);
    return sums<__nv_bfloat16>(dY, lddy, scale, dW, lddw, wide, add, p, at, s);
}

}  // namespace detox
