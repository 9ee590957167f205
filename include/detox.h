/*
 * libdetox — DETOX parameter-server gradient aggregation for NVIDIA B200 (sm_100a).
 *
 * C ABI.  Every entry point enqueues its kernels on the caller's CUDA stream and returns without
 * synchronising the host.  The library allocates nothing and keeps no state between calls: every
 * buffer, including scratch ("workspace"), belongs to the caller (the one exception, a fixed
 * scratch array inside the library, is detox_vote_noalloc below).
 *
 * Notation follows arXiv 1907.12205: n compute nodes (the paper's p) each send a gradient of
 * dimension d; node groups have size r (odd, r divides n), so there are G = n / r votes; f is the
 * Byzantine tolerance handed to Multi-Krum / Bulyan.
 *
 * Common conventions
 *   - "dev" pointers are device pointers valid on the current device; "host" pointers are ordinary
 *     host memory, read before the call returns.
 *   - Matrices are row-major fp32 with a row stride `ld` in ELEMENTS (ld >= d).  The vectorised paths
 *     need a 16-byte aligned base and ld % 4 == 0; any other layout takes a slower scalar path with the
 *     same results.
 *   - Index outputs are int32.  Limits: n, m <= DETOX_MAX_ROWS; r <= DETOX_MAX_R.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default stream).
 *   - Workspace pointers must be 256-byte aligned; sizes come from the *_workspace_bytes helpers.
 *   - Errors: argument problems are reported before anything is launched; a failed launch returns
 *     DETOX_ERR_CUDA.  Nothing aborts or throws.  Multi-Krum and Bulyan run kernels that wait on
 *     asynchronous copies (9 to 16 long rows) or on the tensor cores (17 to 256 rows); every such
 *     device-side wait is bounded, and so are those of the gated products.  Device status word: the first int32
 *     of the workspace passed to agg_multikrum, agg_bulyan, agg_pairwise_sqdist, detox_aggregate, detox_gated or
 *     detox_gated_backward.  The call clears it; should a wait run out in any
 *     stage of the call it reads DETOX_ERR_TIMEOUT once the stream has been synchronised (0 otherwise),
 *     the outputs are then not valid (the index outputs still hold in-range indices), and nothing
 *     hangs or faults.
 *   - Non-finite values: the vote and the order statistics are fully defined on them (bit patterns).
 *     In Multi-Krum / Bulyan a row with an Inf or NaN entry is infinitely far from every other row
 *     (a NaN distance counts as +Inf), so it is never preferred to a finite row.
 *   - Ranking of values (medians, "closest to the median") uses the total order
 *     -NaN < -Inf < ... < -0 < +0 < ... < +Inf < +NaN on fp32 bit patterns.
 */
#ifndef DETOX_H_
#define DETOX_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define DETOX_MAX_ROWS 1024
#define DETOX_MAX_R 15

typedef enum {
    DETOX_OK = 0,
    DETOX_ERR_BAD_ARG = 1,      /* null pointer, size out of range, r even or not dividing n, bad partition */
    DETOX_ERR_UNSUPPORTED = 2,  /* valid request outside the built limits */
    DETOX_ERR_WORKSPACE = 3,    /* workspace missing, misaligned or too small */
    DETOX_ERR_CUDA = 4,         /* a CUDA call or launch failed */
    DETOX_ERR_TIMEOUT = 5       /* a bounded device-side wait ran out (reported through the status word) */
} detox_status;

typedef enum {
    DETOX_AGG_NONE = 0,         /* A_0 only: pass the votes through */
    DETOX_AGG_MEAN = 1,
    DETOX_AGG_COORD_MEDIAN = 2,
    DETOX_AGG_MULTIKRUM = 3,
    DETOX_AGG_BULYAN = 4,
    DETOX_AGG_TRIMMED_MEAN = 5, /* A_1 only: drops the f smallest and f largest values per coordinate */
    DETOX_AGG_GEOMETRIC_MEDIAN = 6, /* A_1 only: gm_iters Weiszfeld iterations over at most 32 rows */
    DETOX_AGG_SIGN_MAJORITY = 7 /* A_0 and A_1: coordinate-wise sign(sum of signs), the signSGD pairing */
} detox_agg;

const char* detox_status_string(detox_status s);

/* ---------------------------------------------------------------------------------------------
 * Filtering step (Section 3; Algorithm 1, "Filtering step"): for every node group A_j the majority
 * vote z_j = maj{ g_i : i in A_j }, and z_j = 0 when no value is sent by more than r/2 members.
 * Two members agree when their d-vectors are bitwise identical.
 *
 *   X        dev, n x ld      the n received gradients (read only)
 *   members  host, G*r        worker ids; group j owns members[j*r .. j*r+r-1]; a partition of 0..n-1
 *   Z        dev, G x ldz     out: the votes; may be NULL when only `winner` is wanted
 *   winner   dev, G           out: lowest worker id of the winning class, or -1 (then Z[j] = 0)
 *   ws       dev              detox_vote_workspace_bytes(n, r) bytes
 * ------------------------------------------------------------------------------------------- */
size_t detox_vote_workspace_bytes(int n, int r);
detox_status detox_vote(const float* X, int64_t ld, int n, int r, int64_t d, const int32_t* members,
                        float* Z, int64_t ldz, int32_t* winner, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * detox_vote without a workspace, for callers that must not allocate device memory.  (The paper has
 * no counterpart; this is a packaging variant of detox_vote and computes exactly the same votes.)
 *
 * Who needs it: code that runs where cudaMalloc is off limits - inside a framework's allocator
 * callback, in a latency-critical serving loop with a frozen memory plan, or in a process whose
 * memory budget is fixed at start-up - and that has nowhere to keep a workspace buffer.
 *
 * The scratch words of the vote live in a fixed array inside the library (4 KiB of global memory on
 * every GPU that loads the library, held until the process exits), so at most
 * DETOX_NOALLOC_MAX_GROUPS node groups (n / r) are accepted; more returns DETOX_ERR_UNSUPPORTED.
 * The call itself performs no cudaMalloc / cudaFree and calls no allocating routine.
 *
 *   - Arguments as in detox_vote, minus ws / ws_bytes.  Inputs and outputs are still the caller's.
 *   - The first call on each device looks up the device address of the built-in array (a one-time
 *     set-up step, done with that device current).  Make that first call before any stream capture.
 *   - All calls on a device share the one array.  Each call clears the words it uses before using
 *     them, so results never depend on an earlier call; but two calls whose kernels overlap on the
 *     GPU (different streams, no dependency between them) race on it.  Serialise them.
 * ------------------------------------------------------------------------------------------- */
#define DETOX_NOALLOC_MAX_GROUPS 256
detox_status detox_vote_noalloc(const float* X, int64_t ld, int n, int r, int64_t d, const int32_t* members,
                                float* Z, int64_t ldz, int32_t* winner, void* stream);

/* ---------------------------------------------------------------------------------------------
 * A_0 = mean over each vote group (Algorithm 2, step 3, with A_0 the mean as analysed in Section 4):
 * M[s] = (1/|Z_s|) sum_{j in Z_s} z_j.  A zero vote (no majority) counts as an ordinary member.
 *
 *   Z            dev, G x ldz   the votes
 *   set_offsets  host, S+1      set s owns set_members[set_offsets[s] .. set_offsets[s+1]-1]; sets may be
 *                               uneven (e.g. 7 and 8 out of 15, Appendix B.1) but not empty
 *   set_members  host, G        vote indices, a partition of 0..G-1
 *   M            dev, S x ldm   out
 * ------------------------------------------------------------------------------------------- */
detox_status detox_hier_mean(const float* Z, int64_t ldz, int G, int64_t d, const int32_t* set_offsets,
                             const int32_t* set_members, int S, float* M, int64_t ldm, void* stream);

/* ---------------------------------------------------------------------------------------------
 * detox_vote followed by detox_hier_mean, in one pass over X (Algorithm 1's filtering step and
 * Algorithm 2, step 3 with A_0 the mean): M[s] is the mean of the votes of set s, bit for bit what
 * the two calls give, but the votes are never written to memory (n*d*4 bytes read, S*d*4 written).
 * detox_aggregate uses this path whenever a0 = DETOX_AGG_MEAN.
 *
 *   arguments as in detox_vote (without Z) and detox_hier_mean (without Z, G);
 *   ws: detox_vote_workspace_bytes(n, r) bytes.
 * ------------------------------------------------------------------------------------------- */
detox_status detox_vote_hier_mean(const float* X, int64_t ld, int n, int r, int64_t d, const int32_t* members,
                                  const int32_t* set_offsets, const int32_t* set_members, int S, float* M,
                                  int64_t ldm, int32_t* winner, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * The same two steps for very many nodes with short vectors - the regime of the paper's synthetic
 * experiment (Section 5.3, "Mean estimation on synthetic data": p = 220,000 nodes, r = 11, d <= 100), where
 * the tables above (at most DETOX_MAX_ROWS nodes) do not reach.  One warp votes per node group; the
 * group table lives in device memory; a vote set is a run of consecutive groups (the group table is a
 * random partition already, so consecutive groups are a random set).  The S set means then go to
 * agg_geometric_median / agg_coord_median as ordinary rows.
 *
 *   X            dev, n x ld     n <= 2^30 nodes, d <= DETOX_MANY_MAX_D
 *   members      dev, n          worker ids, group j owns members[j*r .. j*r+r-1]; must be a partition of
 *                                0..n-1 (not checked; a group holding an id outside 0..n-1 gets no vote)
 *   set_offsets  host, S+1       set s owns the groups set_offsets[s] .. set_offsets[s+1]-1; S <= DETOX_MAX_ROWS
 *   M            dev, S x ldm    out: mean of the votes of each set (a group without a majority counts as a
 *                                zero vote); may be NULL, then only `winner` is produced and sets are ignored
 *   winner       dev, n / r      out, as in detox_vote
 * No workspace.
 * ------------------------------------------------------------------------------------------- */
#define DETOX_MANY_MAX_D 1024
detox_status detox_vote_hier_mean_many(const float* X, int64_t ld, int64_t n, int r, int d, const int32_t* members,
                                       const int32_t* set_offsets, int S, float* M, int64_t ldm, int32_t* winner,
                                       void* stream);

/* ---------------------------------------------------------------------------------------------
 * Coordinate-wise median (Section 4; Appendix B.1): out[c] = median_i X[i][c] over the m rows.
 * Odd m: the middle value, bit for bit one of the inputs.  Even m: fp32 (lo + hi) * 0.5f.
 *   out  dev, d.   ws: agg_coord_median_workspace_bytes(m, d) bytes.  Every size built so far works in
 *   registers or shared memory, so that is 0 and ws is not touched (pass NULL); the arguments keep the
 *   signature of the other aggregators.
 * ------------------------------------------------------------------------------------------- */
size_t agg_coord_median_workspace_bytes(int m, int64_t d);
detox_status agg_coord_median(const float* X, int64_t ld, int m, int64_t d, float* out, void* ws,
                              size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Coordinate-wise alpha-trimmed mean (one of the A_1 choices analysed in Section 4, Theorem 4 with
 * alpha = 1/4): per coordinate, drop the `trim` smallest and the `trim` largest of the m values and
 * average the other m - 2*trim.  0 <= trim, m - 2*trim >= 1.  trim = 0 is the plain mean.
 *   out  dev, d.   No workspace.
 * ------------------------------------------------------------------------------------------- */
detox_status agg_trimmed_mean(const float* X, int64_t ld, int m, int64_t d, int trim, float* out, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Coordinate-wise sign majority, the aggregator of signSGD with majority vote (Section 5.2, setup 4:
 * A_0 = A_1 = coordinate-wise majority): out[c] = sign(sum_i sign(X[i][c])), one of -1, 0, +1
 * (sign(0) = sign(NaN) = 0; a tie gives 0).
 *   out  dev, d.   No workspace.
 * ------------------------------------------------------------------------------------------- */
detox_status agg_sign_majority(const float* X, int64_t ld, int m, int64_t d, float* out, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Geometric median (one of the A_1 choices analysed in Section 4, Theorem 4; the paper does not fix
 * an algorithm).  Computed by Weiszfeld's iteration started at the mean:
 *     y <- sum_j w_j x_j / sum_j w_j,   w_j = 1 / max(||x_j - y||_2, eps),   `iters` times.
 * m <= 32 rows (it aggregates the few set results of the hierarchical step); more returns
 * DETOX_ERR_UNSUPPORTED.  iters >= 0 (0 gives the mean), eps > 0.
 *   out  dev, d.   ws: agg_geometric_median_workspace_bytes(m, d) bytes.
 * ------------------------------------------------------------------------------------------- */
size_t agg_geometric_median_workspace_bytes(int m, int64_t d);
detox_status agg_geometric_median(const float* X, int64_t ld, int m, int64_t d, int iters, float eps, float* out,
                                  void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Pairwise squared Euclidean distances between the m rows, the O(p^2 d) step that Section 4 ("Improved
 * speed") names as the cost of Krum, Multi-Krum and Bulyan: D[i][j] = sum_c (X[i][c] - X[j][c])^2.
 * This is the first stage of agg_multikrum / agg_bulyan on its own (same kernels, same results).
 *   D   dev, m x m fp64, row-major, symmetric, zero diagonal (8-byte aligned)
 *   ws  agg_pairwise_sqdist_workspace_bytes(m, d) bytes; its first int32 is the device status word
 * ------------------------------------------------------------------------------------------- */
size_t agg_pairwise_sqdist_workspace_bytes(int m, int64_t d);
detox_status agg_pairwise_sqdist(const float* X, int64_t ld, int m, int64_t d, double* D, void* ws, size_t ws_bytes,
                                 void* stream);

/* ---------------------------------------------------------------------------------------------
 * Multi-Krum (cited in Section 4 "Improved speed" as the O(p^2 d) aggregator; requirement
 * m >= 2f+3 in Appendix B.1).  score_i = sum of the nb smallest squared distances from row i to the
 * other rows, nb = m - f - 2 clamped to [1, m-1]; the m_sel rows of smallest score (equal scores:
 * lower index first) are averaged.  m < 2f+3 is accepted (the clamp applies) down to m >= 1.
 *
 *   out     dev, d         the average of the selected rows
 *   sel     dev, m_sel     out, ascending row indices; may be NULL
 *   scores  dev, m (fp64)  out; may be NULL
 *   ws      agg_multikrum_workspace_bytes(m, d) bytes
 * ------------------------------------------------------------------------------------------- */
size_t agg_multikrum_workspace_bytes(int m, int64_t d);
detox_status agg_multikrum(const float* X, int64_t ld, int m, int64_t d, int f, int m_sel, float* out,
                           int32_t* sel, double* scores, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Bulyan (cited in Section 4; requirement m >= 4f+3 in Appendix B.1, enforced here).  Stage 1:
 * theta = m - 2f rounds of Krum on the shrinking candidate set (scores recomputed from the cached
 * distances with nb = |remaining| - f - 2, clamped as above).  Stage 2, per coordinate: the median of
 * the theta selected values, then the mean of the beta = theta - 2f values closest to it (closeness
 * |v - median| in fp32; equally close: the smaller value first).
 *
 *   out  dev, d
 *   sel  dev, theta   out, row indices in the order they were selected; may be NULL
 *   ws   agg_bulyan_workspace_bytes(m, d) bytes
 * ------------------------------------------------------------------------------------------- */
size_t agg_bulyan_workspace_bytes(int m, int64_t d);
detox_status agg_bulyan(const float* X, int64_t ld, int m, int64_t d, int f, float* out, int32_t* sel,
                        void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * The whole parameter-server step (Algorithm 1, filtering + hierarchical aggregation; Algorithm 2):
 * vote over the node groups, A_0 over each vote group, A_1 over the results.
 *
 *   a0 = DETOX_AGG_NONE : the G votes go to A_1 directly (sets are ignored).  The votes are rows of X, so they are
 *        read through winner[] and not stored; with a1 = MULTIKRUM or BULYAN over 17 to 85 votes of groups of r = 3
 *        (16-byte aligned rows) the vote itself runs inside the distance pass, one pass over X for both (the votes are
 *        stored, and the pass repeated on them, only when a group has no majority or an entry leaves the range of the
 *        pass's fp16 operands; the results are the same either way)
 *   a0 = DETOX_AGG_MEAN : the S set means go to A_1 (with a1 = MEAN, COORD_MEDIAN or TRIMMED_MEAN over at most 16 sets,
 *        r in {1, 3, 5} and 16-byte aligned rows of X and out, the whole step is one pass over X and the set means
 *        are never stored; the result is bitwise the same either way)
 *   a0 = DETOX_AGG_SIGN_MAJORITY : the S coordinate-wise sign majorities of the sets go to A_1
 *   a0 = DETOX_AGG_MULTIKRUM | DETOX_AGG_BULYAN : the aggregator runs inside every vote set (the pairings the
 *        paper found most resilient, Section 5.2, setups 2 and 3; set shapes as in Appendix B.1, e.g. 7 + 8 or
 *        one set of 15) and its S results go to A_1, which must then be MEAN or COORD_MEDIAN.  f and m_sel
 *        belong to A_0: every set of k votes averages its m_sel best (m_sel = 0: its k - f best), or, for
 *        Bulyan, needs k >= 4f+3.
 *   a1 = MEAN | SIGN_MAJORITY | COORD_MEDIAN | TRIMMED_MEAN (f per side) | GEOMETRIC_MEDIAN (gm_iters, gm_eps; at most 32 rows
 *        enter it) | MULTIKRUM (f, m_sel) | BULYAN (f)
 *
 *   out          dev, d
 *   winner       dev, G        out, as in detox_vote; may be NULL
 *   sel          dev           out, rows chosen by Multi-Krum (m_sel, ascending) or Bulyan (theta, in
 *                              selection order): indices among the rows that entered A_1 when A_1 is the
 *                              Krum-type stage; vote (group) indices, set after set, when A_0 is; may be NULL
 *   sel_workers  dev           out, the same rows as worker ids (winner[vote]), meaningful whenever sel
 *                              indexes votes (a0 = NONE, MULTIKRUM or BULYAN); may be NULL
 *   ws           detox_aggregate_workspace_bytes(desc) bytes (holds the votes and set means too); its first
 *                int32 is the device status word of the whole step (see "Errors" above)
 * ------------------------------------------------------------------------------------------- */
typedef struct {
    int32_t n;                   /* compute nodes */
    int32_t r;                   /* redundancy ratio (odd, divides n) */
    int64_t d;                   /* gradient dimension */
    const int32_t* members;      /* host, G*r */
    int32_t a0;                  /* detox_agg: NONE, MEAN, SIGN_MAJORITY, MULTIKRUM or BULYAN */
    int32_t n_sets;              /* S, used unless a0 = NONE */
    const int32_t* set_offsets;  /* host, S+1 */
    const int32_t* set_members;  /* host, G */
    int32_t a1;                  /* detox_agg: MEAN, COORD_MEDIAN, TRIMMED_MEAN, GEOMETRIC_MEDIAN, MULTIKRUM or BULYAN */
    int32_t f;                   /* tolerance given to Multi-Krum / Bulyan */
    int32_t m_sel;               /* rows averaged by Multi-Krum */
    int32_t gm_iters;            /* Weiszfeld iterations when a1 = GEOMETRIC_MEDIAN */
    float gm_eps;                /* floor on the distances in its weights (> 0) */
} detox_pipeline_desc;

size_t detox_aggregate_workspace_bytes(const detox_pipeline_desc* desc);
detox_status detox_aggregate(const detox_pipeline_desc* desc, const float* X, int64_t ld, float* out,
                             int32_t* winner, int32_t* sel, int32_t* sel_workers, void* ws,
                             size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * The worker's side (Algorithm 1 lets a worker compute its gradient by any program; the paper fixes none): operators of
 * a pre-norm gated feed-forward sublayer,
 *     s = x + residual,   y = rmsnorm(s),   h = act(y Wg^T) * (y Wu^T),
 * with their backward passes and with the 8-bit form in which activations are kept between the two.  The vote compares
 * gradients bit for bit, so all of them add in a fixed order (no floating-point atomics): the same inputs give the same
 * bits in every call on every GPU of the kind.
 *
 *   - Matrices are row-major with a row stride in ELEMENTS (>= columns); a row is a token.  Sums, norms and products are
 *     accumulated in fp32, and every output is rounded once.
 *   - 16-byte aligned bases and strides take the vectorised paths (for the products: TMA); any other layout gives the same results
 *     more slowly (for the products through aligned copies in the workspace).
 *   - Zero rows are accepted: nothing is written but the weight gradients, which are zero.
 * ------------------------------------------------------------------------------------------- */
typedef enum {
    DETOX_DTYPE_FLOAT = 0,
    DETOX_DTYPE_HALF = 1,
    DETOX_DTYPE_BFLOAT = 2
} detox_dtype;

typedef enum {
    DETOX_ACT_SILU = 0,         /* g / (1 + exp(-g)) */
    DETOX_ACT_GELU = 1,         /* g (1 + erf(g / sqrt 2)) / 2 */
    DETOX_ACT_RELU = 2          /* max(g, 0); derivative 0 at 0 */
} detox_act;

/* ---------------------------------------------------------------------------------------------
 * Activation checkpoints in 8 bits.  Every block of DETOX_KEEP_BLOCK columns of a row (the last may be shorter) shares a
 * power-of-two scale 2^e, e the smallest integer with amax <= 448 * 2^e (amax over the block's finite entries, e >= -126);
 * an entry v is kept as the e4m3 number nearest to v * 2^-e (ties to even).  Inf and NaN are kept as NaN.  The scales
 * being powers of two, taking a value out again is exact in fp32, and in bf16 and fp16 for values that they hold.
 *
 *   X  dev, rows x ld     dtype FLOAT, HALF or BFLOAT
 *   Q  dev, rows x ldq    out: e4m3 numbers, one byte each
 *   E  dev, rows x lde    out: biased exponents e + 127 (the E8M0 format), ceil(cols / DETOX_KEEP_BLOCK) a row
 * detox_checkpoint_unpack is the way back: X[r][c] = Q[r][c] * 2^e, rounded to dtype (fp16: clamped to +-65504).
 * ------------------------------------------------------------------------------------------- */
#define DETOX_KEEP_BLOCK 128
detox_status detox_checkpoint_pack(int dtype, const void* X, int64_t ld, int64_t rows, int64_t cols, uint8_t* Q, int64_t ldq,
                                   uint8_t* E, int64_t lde, void* stream);
detox_status detox_checkpoint_unpack(int dtype, const uint8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t rows,
                                     int64_t cols, void* X, int64_t ld, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Root-mean-square norm with the residual's addition:
 *     s = x + residual,   rstd = 1 / sqrt(mean(s^2) + eps),   y = s * rstd * w      (the norm is of s before its rounding)
 *
 *   X, R   dev, rows x ldx / ldr    input, residual (NULL: none); same dtype as w and the outputs
 *   w      dev, cols                weight
 *   S      dev, rows x lds          out: the sum; NULL when not wanted.  May be X or R itself (same base and stride)
 *   Y      dev, rows x ldy          out: the normed rows; may be NULL
 *   Q, E   dev                      out: the normed rows in the 8-bit form above (taken from fp32); both may be NULL
 *   rstd   dev, rows (fp32)         out: for the backward pass; may be NULL
 * At least one of S, Y, Q, rstd is given.  eps >= 0.  cols <= DETOX_NORM_MAX_COLS (a CTA holds a row).  No workspace.
 * ------------------------------------------------------------------------------------------- */
#define DETOX_NORM_MAX_COLS 32768
detox_status detox_rmsnorm(int dtype, const void* X, int64_t ldx, const void* R, int64_t ldr, const void* w, int64_t rows,
                           int64_t cols, float eps, void* S, int64_t lds, void* Y, int64_t ldy, uint8_t* Q, int64_t ldq,
                           uint8_t* E, int64_t lde, float* rstd, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Its backward pass.  With hat = S * rstd:
 *     dx = dS + rstd * (w dY - hat * mean(w dY hat))      (also the gradient of the residual)
 *     dw = sum over the rows of dY * hat
 *   dY   dev, rows x lddy       gradient of the normed rows
 *   dS   dev, rows x ldds       gradient that reaches the sum by its other uses (NULL: none)
 *   S    dev, rows x lds        the forward pass's sum (its x when there was no residual); rstd as it left it
 *   dX   dev, rows x lddx       out; may be dY or dS itself (same base and stride).  NULL: only dw
 *   dw   dev, cols (fp32)       out.  NULL: only dX
 *   ws   detox_rmsnorm_backward_workspace_bytes(rows, cols) bytes
 * ------------------------------------------------------------------------------------------- */
size_t detox_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t cols);
detox_status detox_rmsnorm_backward(int dtype, const void* dY, int64_t lddy, const void* dS, int64_t ldds, const void* S,
                                    int64_t lds, const void* w, const float* rstd, int64_t rows, int64_t cols, void* dX,
                                    int64_t lddx, float* dw, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Gated pair of projections: h = act(g) * u with g = x Wg^T, u = x Wu^T in one kernel (g and u stay fp32 and are never
 * stored in full), and its backward pass
 *     dg = dh * u * act'(g),   du = dh * act(g),   dx = dg Wg + du Wu,   dWg = dg^T x,   dWu = du^T x.
 * dg and du are rounded to dtype, the type the tensor cores multiply; every sum over them is fp32.  Beside the rounding that is
 * a matter of range in HALF: an entry of dg or du above 65504 becomes Inf, and the row of dX and the rows of dWg and dWu that it enters
 * Inf or NaN, even where their sums would be in range; one below 2^-25 becomes 0, and below 2^-14 it has fewer bits.  Scale the
 * loss (dH) by a power of two so that they lie between; BFLOAT has the range of fp32.
 *
 * dtype is HALF or BFLOAT (FLOAT: DETOX_ERR_UNSUPPORTED); tokens, in_dim and hidden are at most 2^30.  No output
 * of either pass may overlap an input or another output.
 *
 * The input is X, or its 8-bit form XQ, XE (X = NULL).  With the kept buffers (all four or none) detox_gated leaves g and
 * u there in the 8-bit form, and detox_gated_backward reads them; without them it computes g and u again from the input.
 *
 *   H    dev, tokens x ldh      out
 *   dH   dev, tokens x lddh     gradient of h
 *   dX   dev, tokens x lddx     out; may be NULL
 *   dWg, dWu  dev, hidden x lddw   out, dtype `dw_dtype`: the descriptor's, or DETOX_DTYPE_FLOAT (then they can be
 *                               pieces of a row of the matrix that the vote reads); both may be NULL
 *   ws   detox_gated_workspace_bytes(desc) / detox_gated_backward_workspace_bytes(desc) bytes; its first int32 is the
 *        device status word (see "Errors" above)
 * ------------------------------------------------------------------------------------------- */
typedef struct {
    int32_t dtype;               /* detox_dtype: HALF or BFLOAT */
    int32_t act;                 /* detox_act */
    int64_t tokens, in_dim, hidden;
    const void* X;               /* dev, tokens x ldx; or NULL */
    int64_t ldx;
    const uint8_t* XQ;           /* dev, tokens x ldxq: used when X is NULL */
    int64_t ldxq;
    const uint8_t* XE;           /* dev, tokens x ldxe */
    int64_t ldxe;
    const void* Wg;              /* dev, hidden x ldwg */
    int64_t ldwg;
    const void* Wu;              /* dev, hidden x ldwu */
    int64_t ldwu;
    uint8_t* GQ;                 /* kept g: dev, tokens x ldq; or NULL */
    uint8_t* GE;                 /*         dev, tokens x lde */
    uint8_t* UQ;                 /* kept u, same strides */
    uint8_t* UE;
    int64_t ldq, lde;
} detox_gated_desc;

size_t detox_gated_workspace_bytes(const detox_gated_desc* desc);
detox_status detox_gated(const detox_gated_desc* desc, void* H, int64_t ldh, void* ws, size_t ws_bytes, void* stream);
size_t detox_gated_backward_workspace_bytes(const detox_gated_desc* desc);
detox_status detox_gated_backward(const detox_gated_desc* desc, const void* dH, int64_t lddh, void* dX, int64_t lddx,
                                  void* dWg, void* dWu, int64_t lddw, int dw_dtype, void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * The bounded waits of the gated products.  One that runs out sets the status word of its call, whose remaining products then
 * give up at once; every output that was not written is NaN (kept entries too); nothing hangs, and the next call is not affected.
 *
 * Large products, which pairs of CTAs multiply, are launched without overlap with the stream's other kernels.  While they
 * overlapped, full batches stopped making progress about once in some thousand steps; that it was the overlap is what long
 * series of steps since then say, not a proof.
 *
 * detox_gated_expired_waits: how many of them ran out on the current device since the host last cleared the count.  It does
 * not depend on a workspace, so it also tells of calls whose workspace is gone.  Synchronises the device.
 *   first  host, DETOX_EXPIRED_WORDS int32 (or NULL): what the first of them waited for, -1 where there is none:
 *          form (0 forward, 1 again for the backward pass, 2 dx, 3 weight gradients), CTAs that multiply a tile, its
 *          columns, CTAs that share its reduction, the CTA's rank, barrier (0 a stage free, 1 a stage's copies, 2 an accumulator
 *          free, 3 an accumulator complete), which stage or accumulator, tile (-1: after the last)
 *   clear  not 0: the count and the record start again
 * detox_gated_wait_limit: the limit of a wait in SM clocks, for launches from then on, in place of one that goes by the length of
 * the product (a tenth of a second and more).  0 restores that; any other value below DETOX_WAIT_LIMIT_MIN changes
 * nothing.  Returns the limit before (0: by the product's length).  A diagnostic: a limit that a product's own time exceeds makes it give up.
 * ------------------------------------------------------------------------------------------- */
#define DETOX_EXPIRED_WORDS 8
#define DETOX_WAIT_LIMIT_MIN 10000
unsigned long long detox_gated_expired_waits(int32_t* first, int clear);
int64_t detox_gated_wait_limit(int64_t clocks);

/* ---------------------------------------------------------------------------------------------
 * Token embedding, with the worker's side: rows of a table, scaled,
 *     Y[t] = scale * W[tokens[t]]
 * and the table's gradient
 *     dW[v] = (dW[v] +) scale * sum of dY[t] over the rows t with tokens[t] = v,
 * added in fp32 in an order that depends on the sizes and the tokens alone.  A negative token is padding: its row is zero and it has no
 * gradient.  A token >= vocab has a row of NaN, and no gradient either.
 *
 *   W       dev, vocab x ldw        dtype FLOAT, HALF or BFLOAT
 *   tokens  dev, rows               int32 or int64, see `index`
 *   Y       dev, rows x ldy         out, dtype
 *   dY      dev, rows x lddy        dtype
 *   dW      dev, vocab x lddw       out, dtype `dw_dtype`: dtype, or DETOX_DTYPE_FLOAT (then it can be a piece of a row of the matrix that the
 *                                   vote reads).  accumulate = 0: every row is written, those of tokens that do not occur with zeros.  Else the sums
 *                                   are added to what dW holds (fp32 sum, rounded once), and rows of tokens that do not occur are left alone
 *   ws      detox_embedding_backward_workspace_bytes(rows, vocab, cols) bytes
 * No output may overlap an input.
 * ------------------------------------------------------------------------------------------- */
typedef enum {
    DETOX_INDEX_INT32 = 0,
    DETOX_INDEX_INT64 = 1
} detox_index;

detox_status detox_embedding(int dtype, const void* W, int64_t ldw, int64_t vocab, int64_t cols, int index, const void* tokens,
                             int64_t rows, float scale, void* Y, int64_t ldy, void* stream);
size_t detox_embedding_backward_workspace_bytes(int64_t rows, int64_t vocab, int64_t cols);
detox_status detox_embedding_backward(int dtype, const void* dY, int64_t lddy, int index, const void* tokens, int64_t rows, int64_t vocab,
                                      int64_t cols, float scale, void* dW, int64_t lddw, int dw_dtype, int accumulate, void* ws,
                                      size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Losses over logits.  Z has a row of vocab logits for each token position, y the token chosen there; with temperature 1 / scale (scale > 0)
 *     lse[t] = log sum_j exp(scale Z[t][j]),     logp[t] = scale Z[t][y[t]] - lse[t]
 * Every dtype is computed in fp32 and rounded once.
 *   - y[t] < 0: the row has no chosen token.  Its logp is 0, it takes no part in a loss, and its gradient is zero.  Its lse does not depend on
 *     the token and is that of any row; where lse is not asked for (NULL, the losses, the backward pass) the row is not read.
 *     y[t] >= vocab: logp is NaN (and with it the loss and the row's gradient).
 *   - Logits of -Inf, or with scale Z below -2^31 ln 2 = -1.49e9, have probability and gradient 0 (masked entries; fp32 tells larger numbers of this size apart by 64 at
 *     best).  A row of nothing but such entries: lse, and with a chosen token logp, are -Inf, its gradient zero.  scale Z above
 *     2^31 ln 2 is out of range.
 *   - vocab <= DETOX_LOGITS_MAX_COLS (a cluster of CTAs holds a row).
 *   - dZ may be Z itself (same base and stride).
 *
 *   Z, dZ    dev, rows x ldz / lddz    dtype FLOAT, HALF or BFLOAT
 *   y        dev, rows                 int32 or int64 (`index`)
 *   logp, lse, dlogp                   dev, rows, fp32; of logp and lse either may be NULL
 * detox_token_logp_backward: dZ[t][j] = scale dlogp[t] (1[j = y[t]] - exp(scale Z[t][j] - lse[t])), lse as detox_token_logp left it.  A row whose
 * dlogp is 0 is not read, and its gradient is zero.  lse being fp32, its own rounding puts up to |lse| 2^-24 on every probability here (logits of a few tens: 10^-6), and
 * 1 - p of a token that a row is sure of is a difference; the losses, which keep more of it, have neither.
 * Precision: a row's sum is known to a few 2^-23 of itself; logp is -log(1 + q), q being the sum of the other tokens' probabilities over the chosen one's, so it is known
 * to as much of itself near 0, and elsewhere to as much in absolute numbers, before it is rounded to fp32.  Probabilities below 2^-126 of a row's largest count as 0.
 * ------------------------------------------------------------------------------------------- */
#define DETOX_LOGITS_MAX_COLS 262144
detox_status detox_token_logp(int dtype, const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y, float scale,
                              float* logp, float* lse, void* stream);
detox_status detox_token_logp_backward(int dtype, const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y,
                                       float scale, const float* lse, const float* dlogp, void* dZ, int64_t lddz, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Clipped policy loss with a KL term, and the gradient of the logits in the same pass over them.  With the ratio r = exp(logp - old[t]),
 *     pg[t] = -min(r A[t], min(max(r, 1 - clip_low), 1 + clip_high) A[t])
 *     kl[t] = exp(ref[t] - logp) - (ref[t] - logp) - 1                  (0 without ref; with kl_coef = 0 in stats alone, whatever it is)
 *     loss  = sum over t of w[t] (pg[t] + kl_coef kl[t])                (without w: w[t] = 1 / rows)
 *   old, A   dev, rows (fp32)    log-probability under the policy that chose the tokens, and advantage
 *   ref      dev, rows (fp32)    log-probability under the reference policy; may be NULL
 *   w        dev, rows (fp32)    weights, such as mask / number of tokens; may be NULL.  A row of weight 0 counts like one without a chosen token
 *                                (logp 0), whatever its logits, old, A and ref hold
 *   stats    dev, 4 (fp32)       out: loss, sum w pg, sum w kl, sum of w over the clipped tokens (r A > clipped r A); added in a fixed order
 *   logp     dev, rows (fp32)    out; may be NULL
 *   dZ       dev, rows x lddz    out: grad_scale * d loss / d Z; NULL: not wanted
 *   ws       detox_policy_loss_workspace_bytes(rows) bytes
 * clip_low in [0, 1], clip_high >= 0.  A ratio or an exp(ref - logp) beyond fp32's range is Inf; with an advantage of 0 the former's term is 0.
 * ------------------------------------------------------------------------------------------- */
typedef struct {
    int32_t dtype, index;        /* detox_dtype of the logits, detox_index of y */
    int64_t rows, vocab;
    const void* Z;               /* dev, rows x ldz */
    int64_t ldz;
    const void* y;               /* dev, rows */
    const float* old_logp;       /* dev, rows */
    const float* advantage;      /* dev, rows */
    const float* ref_logp;       /* dev, rows; or NULL */
    const float* weight;         /* dev, rows; or NULL */
    float clip_low, clip_high, kl_coef, scale, grad_scale;
} detox_policy_desc;

size_t detox_policy_loss_workspace_bytes(int64_t rows);
detox_status detox_policy_loss(const detox_policy_desc* desc, float* stats, float* logp, void* dZ, int64_t lddz, void* ws,
                               size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Preference loss of paired log ratios.  The rows are packed sequences: rows offsets[i] .. offsets[i + 1] - 1 are sequence i, and sequences 2p and
 * 2p + 1 are the preferred and the other answer of pair p.  S_i = sum of logp over sequence i (rows without a chosen token, such as a prompt's, add 0):
 *     margin[p] = beta ((S_2p - ref_2p) - (S_2p+1 - ref_2p+1))
 *     loss      = mean over p of -(1 - smoothing) log sigmoid(margin[p]) - smoothing log sigmoid(-margin[p])
 *   offsets  dev, 2 pairs + 1 (int32)   ascending, 0 .. rows (others are clamped; the results are then of no use).  Rows of no sequence have zero gradients
 *   ref      dev, 2 pairs (fp32)        the sums under the reference policy
 *   loss     dev, 1 (fp32)              out (0 pairs: 0)
 *   margin   dev, pairs (fp32)          out
 *   sums     dev, 2 pairs (fp32)        out: S
 *   dZ       dev, rows x lddz           out: grad_scale * d loss / d Z; NULL: not wanted
 *   ws       detox_preference_loss_workspace_bytes(rows, pairs) bytes
 * smoothing in [0, 1].  The sums over tokens are formed in 64 bits.
 * ------------------------------------------------------------------------------------------- */
typedef struct {
    int32_t dtype, index;
    int64_t rows, vocab, pairs;
    const void* Z;               /* dev, rows x ldz */
    int64_t ldz;
    const void* y;               /* dev, rows */
    const int32_t* offsets;      /* dev, 2 pairs + 1 */
    const float* ref;            /* dev, 2 pairs */
    float beta, smoothing, scale, grad_scale;
} detox_preference_desc;

size_t detox_preference_loss_workspace_bytes(int64_t rows, int64_t pairs);
detox_status detox_preference_loss(const detox_preference_desc* desc, float* loss, float* margin, float* sums, void* dZ, int64_t lddz,
                                   void* ws, size_t ws_bytes, void* stream);

/* ---------------------------------------------------------------------------------------------
 * One AdamW step over many tensors: what the server does with the aggregated gradient (whose pieces the tensors' gradients can be).
 *     m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2                      (g: the gradient times grad_scale)
 *     p <- p - lr (weight_decay p + (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps))
 * in fp32; with a master copy p is read from it and written to it unrounded, and P gets it rounded to its type.
 *
 * States in 32 bits: M and V hold m and v.  States in 8 bits: they hold m and sqrt(v) in the 8-bit form of the checkpoints above, taken over the
 * tensor's n entries as one row, except that an entry is rounded up or down at random, so that its mean is right (to the nearest,
 * sqrt(v) would not move at all: beta2 changes it by far less than the form's step).  A root that is not 0 is never kept as 0.  The step itself uses m and v
 * before they are rounded.  The random bits are a function of seed, step, the tensor's key and the entry alone, so every copy of a server gets the same states:
 *     mix(x): x ^= x >> 16;  x *= 0x85ebca6b;  x ^= x >> 13;  x *= 0xc2b2ae35;  x ^= x >> 16          (32 bits)
 *     h = mix(mix(mix(seed + 0x9e3779b9 step) + key) ^ entry),  m takes h & 0xffff, sqrt(v) h >> 16
 * and an entry between two neighbours is rounded away from zero when its distance from the lower one, in steps, plus those bits / 2^16 reaches 1.
 *
 * tensors: host, `count` of them; read before the call returns.  No two buffers of a call may overlap, but P may be the master itself (FLOAT; give
 * it as P alone).  Entries are contiguous; any alignment to the entry's size works, 16 bytes (8 for 16-bit entries, 4 for 8-bit ones) is faster.
 * A tensor without entries is passed over.  eps >= DETOX_ADAMW_LEAST_EPS, in 8
 * bits DETOX_ADAMW_LEAST_EPS_8 (fp32's squares end at 10^-45, and in 8 bits what is below 10^-38 counts as 0: beside a smaller eps a root would not be known, and eps itself
 * could be 0 in fp32); beta1 and beta2 in [0, 1).  FLOAT weights take a gradient of any type and have no master;
 * HALF and BFLOAT ones take a gradient of their own type or FLOAT (else DETOX_ERR_UNSUPPORTED).  A tensor whose buffers are all off a 16-byte boundary by
 * the same number of entries, as slices of vectors of one layout are, is as fast as an aligned one (32 bits; with 8-bit states a tensor
 * off the boundary takes 1.7 times as long).  No workspace.
 * ------------------------------------------------------------------------------------------- */
#define DETOX_ADAMW_LEAST_EPS 1e-18
#define DETOX_ADAMW_LEAST_EPS_8 1e-15
typedef struct {
    void* P;                     /* dev, n: the weights */
    const void* G;               /* dev, n: the gradient */
    float* master;               /* dev, n: fp32 copy of the weights; or NULL */
    void* M;                     /* dev, n: fp32, or e4m3 */
    uint8_t* ME;                 /* dev, ceil(n / DETOX_KEEP_BLOCK): scales; 32 bits: not used */
    void* V;
    uint8_t* VE;
    int64_t n;
    int32_t p_dtype, g_dtype;    /* detox_dtype */
    float weight_decay;
    uint32_t key;
} detox_adamw_tensor;

typedef struct {
    int32_t bits;                /* of the states: 32 or 8 */
    uint32_t seed;               /* 8 bits only */
    double lr, beta1, beta2, eps;
    float grad_scale;
    int64_t step;                /* >= 1: the number of this step */
    const float* lr_dev;         /* dev, 1: read instead of lr when the step runs (a captured one reads it at each replay); or NULL */
    const int64_t* step_dev;     /* dev, 1: likewise for step (taken as 1 when it is less); or NULL */
} detox_adamw_desc;

detox_status detox_adamw(const detox_adamw_desc* desc, const detox_adamw_tensor* tensors, int64_t count, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Self-test of the bounded device-side waits (no counterpart in the paper; a diagnostic).  Launches one
 * warp that waits, with the same wait routine the distance kernels use, on a barrier that nothing will
 * ever complete, for at most `limit_cycles` SM clocks (1 .. 2e9).  The wait must give up by itself: after
 * the stream has been synchronised *status reads DETOX_ERR_TIMEOUT (any other value is a failure of the
 * wait routine), the kernel has exited normally and the context is intact.
 *   status  dev, one int32 (cleared by the call)
 * ------------------------------------------------------------------------------------------- */
detox_status detox_selftest_bounded_wait(int32_t* status, int64_t limit_cycles, void* stream);

/* ---------------------------------------------------------------------------------------------
 * Which operand split the tensor-core distance pass (17 .. 256 aligned rows; Section 4, "Improved speed": the
 * O(p^2 d) part of Multi-Krum and Bulyan) tries first.  Process-wide; returns the previous mode; any other value of
 * `mode` only queries.
 *   DETOX_SPLIT_AUTO  (default) every entry as two fp16 numbers after a per-row power-of-two scale; a check after the
 *                     pass repeats it with the split-TF32 kernels when an entry left the fp16 range (distances are
 *                     the same to within the accuracy both give; only the time differs)
 *   DETOX_SPLIT_TF32  the split-TF32 kernels (three-product TF32 with the cross terms folded) from the start
 * A switch for measurements and tests; not meant to be flipped while calls are in flight on other threads.
 * ------------------------------------------------------------------------------------------- */
enum { DETOX_SPLIT_AUTO = 0, DETOX_SPLIT_TF32 = 1 };
int detox_tc_split_mode(int mode);

/* How many calls on the current device have had their tensor-core distance pass repeated so far in this process:
 * by the split-TF32 kernels after an entry left the fp16 range, or without the common vector after the check
 * withdrew it (a diagnostic counter, no counterpart in the paper).  Waits for the device's pending work;
 * ~0 on a CUDA error. */
unsigned long long detox_tc_repeated_passes(void);

/* Number of kernels this library has launched in this process so far (a diagnostic counter, no counterpart in
 * the paper; the one piece of state the library keeps, besides the scratch of detox_vote_noalloc). */
unsigned long long detox_kernel_launch_count(void);

#ifdef __cplusplus
}
#endif
#endif /* DETOX_H_ */
