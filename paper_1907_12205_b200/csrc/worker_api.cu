// C ABI of the worker-side operators: argument validation.  Nothing here touches data on the host, allocates, or
// synchronises.
#include <cmath>

#include "worker.cuh"

using namespace detox;

namespace {

constexpr int64_t kMaxDim = (int64_t)1 << 30;      // TMA coordinates and tile counts are 32-bit
constexpr int64_t kMaxNormCols = DETOX_NORM_MAX_COLS;   // a CTA of 1024 threads holds a row, 32 entries each

int dtype_size(int dtype) {
    return dtype == DETOX_DTYPE_FLOAT ? 4 : ((dtype == DETOX_DTYPE_HALF || dtype == DETOX_DTYPE_BFLOAT) ? 2 : 0);
}
// a matrix that is there: rows far enough apart, entries aligned to their size
bool matrix_ok(const void* p, int64_t ld, int64_t cols, int size) { return p && ld >= cols && aligned_to(p, (size_t)size); }
bool optional_ok(const void* p, int64_t ld, int64_t cols, int size) { return !p || matrix_ok(p, ld, cols, size); }
int64_t blocks_of(int64_t cols) { return ceil_div(cols, (int64_t)kKeepBlock); }

detox_status check_sizes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1) return DETOX_ERR_BAD_ARG;
    return rows > kMaxDim || cols > kMaxDim ? DETOX_ERR_UNSUPPORTED : DETOX_OK;
}
// Q and E of the 8-bit form
bool kept_ok(const uint8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t cols) {
    return Q && E && ldq >= cols && lde >= blocks_of(cols);
}

bool workspace_ok(const void* ws, size_t have, size_t need) {
    return need == 0 || (ws != nullptr && aligned_to(ws, 256) && have >= need);
}

detox_status check_gated(const detox_gated_desc* g) {
    if (!g || (g->dtype != DETOX_DTYPE_HALF && g->dtype != DETOX_DTYPE_BFLOAT && g->dtype != DETOX_DTYPE_FLOAT)) return DETOX_ERR_BAD_ARG;
    if (g->act < DETOX_ACT_SILU || g->act > DETOX_ACT_RELU) return DETOX_ERR_BAD_ARG;
    if (g->tokens < 0 || g->in_dim < 1 || g->hidden < 1) return DETOX_ERR_BAD_ARG;
    if (g->dtype == DETOX_DTYPE_FLOAT) return DETOX_ERR_UNSUPPORTED;   // the tensor cores multiply 16-bit entries
    if (g->tokens > kMaxDim || g->in_dim > kMaxDim || g->hidden > kMaxDim) return DETOX_ERR_UNSUPPORTED;
    if (!matrix_ok(g->Wg, g->ldwg, g->in_dim, 2) || !matrix_ok(g->Wu, g->ldwu, g->in_dim, 2)) return DETOX_ERR_BAD_ARG;
    if (g->tokens > 0) {
        if (g->X ? !matrix_ok(g->X, g->ldx, g->in_dim, 2) : !kept_ok(g->XQ, g->ldxq, g->XE, g->ldxe, g->in_dim)) return DETOX_ERR_BAD_ARG;
        if (g->GQ || g->GE || g->UQ || g->UE) {
            if (!kept_ok(g->GQ, g->ldq, g->GE, g->lde, g->hidden) || !kept_ok(g->UQ, g->ldq, g->UE, g->lde, g->hidden)) return DETOX_ERR_BAD_ARG;
        }
    }
    return DETOX_OK;
}

int index_size(int index) { return index == DETOX_INDEX_INT32 ? 4 : (index == DETOX_INDEX_INT64 ? 8 : 0); }
bool index_ok(const void* p, int index) { return p && aligned_to(p, (size_t)index_size(index)); }
bool vector_ok(const void* p) { return p && aligned_to(p, 4); }   // of fp32 or int32
bool finite(float x) { return std::isfinite(x); }

detox_status check_logits(int dtype, const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y, float scale) {
    const int size = dtype_size(dtype);
    if (size == 0 || index_size(index) == 0 || !(scale > 0.f) || !finite(scale)) return DETOX_ERR_BAD_ARG;
    const detox_status st = check_sizes(rows, vocab);
    if (st != DETOX_OK) return st;
    if (vocab > DETOX_LOGITS_MAX_COLS) return DETOX_ERR_UNSUPPORTED;
    return rows == 0 || (matrix_ok(Z, ldz, vocab, size) && index_ok(y, index)) ? DETOX_OK : DETOX_ERR_BAD_ARG;
}

}  // namespace

extern "C" {

detox_status detox_checkpoint_pack(int dtype, const void* X, int64_t ld, int64_t rows, int64_t cols, uint8_t* Q, int64_t ldq,
                                   uint8_t* E, int64_t lde, void* stream) {
    const int size = dtype_size(dtype);
    if (size == 0) return DETOX_ERR_BAD_ARG;
    const detox_status st = check_sizes(rows, cols);
    if (st != DETOX_OK || rows == 0) return st;
    if (!matrix_ok(X, ld, cols, size) || !kept_ok(Q, ldq, E, lde, cols)) return DETOX_ERR_BAD_ARG;
    return launch_checkpoint_pack(dtype, X, ld, rows, cols, Q, ldq, E, lde, static_cast<cudaStream_t>(stream));
}

detox_status detox_checkpoint_unpack(int dtype, const uint8_t* Q, int64_t ldq, const uint8_t* E, int64_t lde, int64_t rows,
                                     int64_t cols, void* X, int64_t ld, void* stream) {
    const int size = dtype_size(dtype);
    if (size == 0) return DETOX_ERR_BAD_ARG;
    const detox_status st = check_sizes(rows, cols);
    if (st != DETOX_OK || rows == 0) return st;
    if (!matrix_ok(X, ld, cols, size) || !kept_ok(Q, ldq, E, lde, cols)) return DETOX_ERR_BAD_ARG;
    return launch_checkpoint_unpack(dtype, Q, ldq, E, lde, rows, cols, X, ld, static_cast<cudaStream_t>(stream));
}

detox_status detox_rmsnorm(int dtype, const void* X, int64_t ldx, const void* R, int64_t ldr, const void* w, int64_t rows,
                           int64_t cols, float eps, void* S, int64_t lds, void* Y, int64_t ldy, uint8_t* Q, int64_t ldq,
                           uint8_t* E, int64_t lde, float* rstd, void* stream) {
    const int size = dtype_size(dtype);
    if (size == 0 || !(eps >= 0.f)) return DETOX_ERR_BAD_ARG;
    const detox_status st = check_sizes(rows, cols);
    if (st != DETOX_OK) return st;
    if (cols > kMaxNormCols) return DETOX_ERR_UNSUPPORTED;
    if (rows == 0) return DETOX_OK;
    if ((!S && !Y && !Q && !rstd) || !matrix_ok(X, ldx, cols, size) || !matrix_ok(w, cols, cols, size) || !optional_ok(R, ldr, cols, size) ||
        !optional_ok(S, lds, cols, size) || !optional_ok(Y, ldy, cols, size) || ((Q || E) && !kept_ok(Q, ldq, E, lde, cols)) ||
        !aligned_to(rstd, 4))
        return DETOX_ERR_BAD_ARG;
    return launch_rmsnorm(dtype, X, ldx, R, ldr, w, rows, cols, eps, S, lds, Y, ldy, Q, ldq, E, lde, rstd,
                          static_cast<cudaStream_t>(stream));
}

size_t detox_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (check_sizes(rows, cols) != DETOX_OK || cols > kMaxNormCols) return 0;
    return rmsnorm_backward_ws_bytes(rows, cols);
}

detox_status detox_rmsnorm_backward(int dtype, const void* dY, int64_t lddy, const void* dS, int64_t ldds, const void* S,
                                    int64_t lds, const void* w, const float* rstd, int64_t rows, int64_t cols, void* dX,
                                    int64_t lddx, float* dw, void* ws, size_t ws_bytes, void* stream) {
    const int size = dtype_size(dtype);
    if (size == 0 || (!dX && !dw) || !aligned_to(dw, 4)) return DETOX_ERR_BAD_ARG;
    const detox_status st = check_sizes(rows, cols);
    if (st != DETOX_OK) return st;
    if (cols > kMaxNormCols) return DETOX_ERR_UNSUPPORTED;
    if (rows > 0) {
        if (!matrix_ok(dY, lddy, cols, size) || !matrix_ok(S, lds, cols, size) || !matrix_ok(w, cols, cols, size) ||
            !optional_ok(dS, ldds, cols, size) || !optional_ok(dX, lddx, cols, size) || !rstd || !aligned_to(rstd, 4))
            return DETOX_ERR_BAD_ARG;
        if (dw && !workspace_ok(ws, ws_bytes, rmsnorm_backward_ws_bytes(rows, cols))) return DETOX_ERR_WORKSPACE;
    }
    return launch_rmsnorm_backward(dtype, dY, lddy, dS, ldds, S, lds, w, rstd, rows, cols, dX, lddx, dw, ws,
                                   static_cast<cudaStream_t>(stream));
}

size_t detox_gated_workspace_bytes(const detox_gated_desc* desc) {
    return check_gated(desc) == DETOX_OK ? gated_ws_bytes(*desc) : 0;
}

detox_status detox_gated(const detox_gated_desc* desc, void* H, int64_t ldh, void* ws, size_t ws_bytes, void* stream) {
    const detox_status st = check_gated(desc);
    if (st != DETOX_OK) return st;
    if (desc->tokens > 0 && !matrix_ok(H, ldh, desc->hidden, 2)) return DETOX_ERR_BAD_ARG;
    if (!workspace_ok(ws, ws_bytes, gated_ws_bytes(*desc))) return DETOX_ERR_WORKSPACE;
    return launch_gated(*desc, H, ldh, ws, static_cast<cudaStream_t>(stream));
}

size_t detox_gated_backward_workspace_bytes(const detox_gated_desc* desc) {
    return check_gated(desc) == DETOX_OK ? gated_backward_ws_bytes(*desc) : 0;
}

detox_status detox_gated_backward(const detox_gated_desc* desc, const void* dH, int64_t lddh, void* dX, int64_t lddx,
                                  void* dWg, void* dWu, int64_t lddw, int dw_dtype, void* ws, size_t ws_bytes, void* stream) {
    const detox_status st = check_gated(desc);
    if (st != DETOX_OK) return st;
    if ((dWg == nullptr) != (dWu == nullptr) || (!dX && !dWg)) return DETOX_ERR_BAD_ARG;
    if (dw_dtype != desc->dtype && dw_dtype != DETOX_DTYPE_FLOAT) return DETOX_ERR_BAD_ARG;
    const int dw_size = dtype_size(dw_dtype);
    if (!optional_ok(dWg, lddw, desc->in_dim, dw_size) || !optional_ok(dWu, lddw, desc->in_dim, dw_size)) return DETOX_ERR_BAD_ARG;
    if (desc->tokens > 0 && (!matrix_ok(dH, lddh, desc->hidden, 2) || !optional_ok(dX, lddx, desc->in_dim, 2))) return DETOX_ERR_BAD_ARG;
    if (!workspace_ok(ws, ws_bytes, gated_backward_ws_bytes(*desc))) return DETOX_ERR_WORKSPACE;
    return launch_gated_backward(*desc, dH, lddh, dX, lddx, dWg, dWu, lddw, dw_dtype, ws, static_cast<cudaStream_t>(stream));
}

detox_status detox_embedding(int dtype, const void* W, int64_t ldw, int64_t vocab, int64_t cols, int index, const void* tokens,
                             int64_t rows, float scale, void* Y, int64_t ldy, void* stream) {
    const int size = dtype_size(dtype);
    if (size == 0 || index_size(index) == 0 || vocab < 1) return DETOX_ERR_BAD_ARG;
    const detox_status st = check_sizes(rows, cols);
    if (st != DETOX_OK) return st;
    if (vocab > kMaxDim) return DETOX_ERR_UNSUPPORTED;
    if (rows == 0) return DETOX_OK;
    if (!matrix_ok(W, ldw, cols, size) || !matrix_ok(Y, ldy, cols, size) || !index_ok(tokens, index)) return DETOX_ERR_BAD_ARG;
    return launch_embedding(dtype, W, ldw, vocab, cols, index, tokens, rows, scale, Y, ldy, static_cast<cudaStream_t>(stream));
}

size_t detox_embedding_backward_workspace_bytes(int64_t rows, int64_t vocab, int64_t cols) {
    if (check_sizes(rows, cols) != DETOX_OK || check_sizes(rows, vocab) != DETOX_OK) return 0;
    return embedding_backward_ws_bytes(rows, vocab, cols);
}

detox_status detox_embedding_backward(int dtype, const void* dY, int64_t lddy, int index, const void* tokens, int64_t rows, int64_t vocab,
                                      int64_t cols, float scale, void* dW, int64_t lddw, int dw_dtype, int accumulate, void* ws,
                                      size_t ws_bytes, void* stream) {
    const int size = dtype_size(dtype);
    if (size == 0 || index_size(index) == 0 || vocab < 1 || (dw_dtype != dtype && dw_dtype != DETOX_DTYPE_FLOAT)) return DETOX_ERR_BAD_ARG;
    const detox_status st = check_sizes(rows, cols);
    if (st != DETOX_OK) return st;
    if (vocab > kMaxDim) return DETOX_ERR_UNSUPPORTED;
    if (!matrix_ok(dW, lddw, cols, dtype_size(dw_dtype))) return DETOX_ERR_BAD_ARG;
    if (rows > 0 && (!matrix_ok(dY, lddy, cols, size) || !index_ok(tokens, index))) return DETOX_ERR_BAD_ARG;
    if (!workspace_ok(ws, ws_bytes, embedding_backward_ws_bytes(rows, vocab, cols))) return DETOX_ERR_WORKSPACE;
    return launch_embedding_backward(dtype, dY, lddy, index, tokens, rows, vocab, cols, scale, dW, lddw, dw_dtype, accumulate != 0, ws,
                                     static_cast<cudaStream_t>(stream));
}

detox_status detox_token_logp(int dtype, const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y, float scale,
                              float* logp, float* lse, void* stream) {
    const detox_status st = check_logits(dtype, Z, ldz, rows, vocab, index, y, scale);
    if (st != DETOX_OK) return st;
    if (rows == 0) return DETOX_OK;
    if ((!logp && !lse) || !aligned_to(logp, 4) || !aligned_to(lse, 4)) return DETOX_ERR_BAD_ARG;
    return launch_token_logp(dtype, Z, ldz, rows, vocab, index, y, scale, logp, lse, static_cast<cudaStream_t>(stream));
}

detox_status detox_token_logp_backward(int dtype, const void* Z, int64_t ldz, int64_t rows, int64_t vocab, int index, const void* y,
                                       float scale, const float* lse, const float* dlogp, void* dZ, int64_t lddz, void* stream) {
    const detox_status st = check_logits(dtype, Z, ldz, rows, vocab, index, y, scale);
    if (st != DETOX_OK) return st;
    if (rows == 0) return DETOX_OK;
    if (!vector_ok(lse) || !vector_ok(dlogp) || !matrix_ok(dZ, lddz, vocab, dtype_size(dtype)) || (dZ == Z && lddz != ldz)) return DETOX_ERR_BAD_ARG;
    return launch_token_logp_backward(dtype, Z, ldz, rows, vocab, index, y, scale, lse, dlogp, dZ, lddz, static_cast<cudaStream_t>(stream));
}

size_t detox_policy_loss_workspace_bytes(int64_t rows) { return check_sizes(rows, 1) == DETOX_OK ? policy_loss_ws_bytes(rows) : 0; }

detox_status detox_policy_loss(const detox_policy_desc* d, float* stats, float* logp, void* dZ, int64_t lddz, void* ws, size_t ws_bytes,
                               void* stream) {
    if (!d) return DETOX_ERR_BAD_ARG;
    const detox_status st = check_logits(d->dtype, d->Z, d->ldz, d->rows, d->vocab, d->index, d->y, d->scale);
    if (st != DETOX_OK) return st;
    if (!(d->clip_low >= 0.f && d->clip_low <= 1.f) || !(d->clip_high >= 0.f) || !finite(d->clip_high) || !finite(d->kl_coef) || !finite(d->grad_scale))
        return DETOX_ERR_BAD_ARG;
    if (!vector_ok(stats) || !aligned_to(logp, 4)) return DETOX_ERR_BAD_ARG;
    if (d->rows > 0 && (!vector_ok(d->old_logp) || !vector_ok(d->advantage) || !aligned_to(d->ref_logp, 4) || !aligned_to(d->weight, 4) ||
                        !optional_ok(dZ, lddz, d->vocab, dtype_size(d->dtype)) || (dZ && dZ == d->Z && lddz != d->ldz)))
        return DETOX_ERR_BAD_ARG;
    if (!workspace_ok(ws, ws_bytes, policy_loss_ws_bytes(d->rows))) return DETOX_ERR_WORKSPACE;
    return launch_policy_loss(*d, stats, logp, dZ, lddz, ws, static_cast<cudaStream_t>(stream));
}

size_t detox_preference_loss_workspace_bytes(int64_t rows, int64_t pairs) {
    return check_sizes(rows, 1) == DETOX_OK && check_sizes(pairs, 1) == DETOX_OK ? preference_loss_ws_bytes(rows, pairs) : 0;
}

detox_status detox_preference_loss(const detox_preference_desc* d, float* loss, float* margin, float* sums, void* dZ, int64_t lddz, void* ws,
                                   size_t ws_bytes, void* stream) {
    if (!d) return DETOX_ERR_BAD_ARG;
    const detox_status st = check_logits(d->dtype, d->Z, d->ldz, d->rows, d->vocab, d->index, d->y, d->scale);
    if (st != DETOX_OK) return st;
    if (d->pairs < 0 || !(d->smoothing >= 0.f && d->smoothing <= 1.f) || !finite(d->beta) || !finite(d->grad_scale)) return DETOX_ERR_BAD_ARG;
    if (d->pairs > kMaxDim / 2) return DETOX_ERR_UNSUPPORTED;
    if (!vector_ok(loss) || (d->pairs > 0 && (!vector_ok(d->offsets) || !vector_ok(d->ref) || !vector_ok(margin) || !vector_ok(sums)))) return DETOX_ERR_BAD_ARG;
    if (d->rows > 0 && (!optional_ok(dZ, lddz, d->vocab, dtype_size(d->dtype)) || (dZ && dZ == d->Z && lddz != d->ldz))) return DETOX_ERR_BAD_ARG;
    if (!workspace_ok(ws, ws_bytes, preference_loss_ws_bytes(d->rows, d->pairs))) return DETOX_ERR_WORKSPACE;
    return launch_preference_loss(*d, loss, margin, sums, dZ, lddz, ws, static_cast<cudaStream_t>(stream));
}

detox_status detox_adamw(const detox_adamw_desc* d, const detox_adamw_tensor* tensors, int64_t count, void* stream) {
    if (!d || count < 0 || (count > 0 && !tensors) || (d->bits != 32 && d->bits != 8)) return DETOX_ERR_BAD_ARG;
    if (!(d->lr_dev || std::isfinite(d->lr)) || !(d->beta1 >= 0. && d->beta1 < 1.) || !(d->beta2 >= 0. && d->beta2 < 1.) || !(d->eps >= (d->bits == 8 ? DETOX_ADAMW_LEAST_EPS_8 : DETOX_ADAMW_LEAST_EPS)) ||
        !std::isfinite(d->eps) || !finite(d->grad_scale) || (!d->step_dev && d->step < 1) || !aligned_to(d->lr_dev, 4) || !aligned_to(d->step_dev, 8))
        return DETOX_ERR_BAD_ARG;
    for (int64_t i = 0; i < count; ++i) {
        const detox_adamw_tensor& t = tensors[i];
        const int ps = dtype_size(t.p_dtype), gs = dtype_size(t.g_dtype);
        if (t.n < 0 || ps == 0 || gs == 0 || !finite(t.weight_decay)) return DETOX_ERR_BAD_ARG;
        if (t.n == 0) continue;
        if (t.n > ((int64_t)1 << 40) || (t.p_dtype == DETOX_DTYPE_FLOAT ? t.master != nullptr : t.g_dtype != t.p_dtype && t.g_dtype != DETOX_DTYPE_FLOAT))
            return DETOX_ERR_UNSUPPORTED;
        if (!t.P || !aligned_to(t.P, (size_t)ps) || !t.G || !aligned_to(t.G, (size_t)gs) || !aligned_to(t.master, 4) || !t.M || !t.V) return DETOX_ERR_BAD_ARG;
        if (t.P == t.G || t.master == t.G || t.M == t.V) return DETOX_ERR_BAD_ARG;
        if (d->bits == 32 ? !aligned_to(t.M, 4) || !aligned_to(t.V, 4) : !t.ME || !t.VE) return DETOX_ERR_BAD_ARG;
    }
    return launch_adamw(*d, tensors, count, static_cast<cudaStream_t>(stream));
}

int64_t detox_gated_wait_limit(int64_t clocks) { return gated_wait_limit(clocks); }

unsigned long long detox_gated_expired_waits(int32_t* first, int clear) { return gated_expired_waits(first, clear != 0); }

}  // extern "C"
