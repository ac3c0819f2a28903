/*
 * haflo_local.h - operators of a party's local step, on plain values.
 *
 * A party of a federated model trains on its own data between two aggregations.
 * Where the model is large, what it trains, and what is then encrypted and
 * aggregated (haflo.h), is a low-rank adapter beside a projection that all
 * parties share. The operators of that step are here: dropout whose mask is
 * never stored, the shared projection with every row's own adapter and its
 * gradients, and the log-probabilities of labels with entropy, top alternatives
 * and gradient (logistic regression's loss for two classes or any number).
 * Gradients of adapters are float32, as haflo_encode_f32 takes them.
 *
 * The conventions of haflo.h hold: 0 or a negative HAFLO_E* code, no exception,
 * device pointers and sizes, a stream, no allocation and no synchronisation,
 * kernels only (a sequence of calls can be captured into a HIP graph). A call
 * works on the current device. Every sum is held in 32 bits; a result is
 * rounded to its type once. Results do not depend on timing: the same call on the
 * same device gives the same bits.
 *
 * Matrices are row-major; `ld*` is the distance between rows in elements, at
 * least the row's length. Elements need no more alignment than their type's, a workspace that of 16 bytes (else HAFLO_EINVAL). Outputs
 * may not overlap inputs except where it says so. Counts are below 2^31.
 */
#ifndef HAFLO_LOCAL_H
#define HAFLO_LOCAL_H

#include "haflo.h"

#ifdef __cplusplus
extern "C" {
#endif

enum haflo_type { HAFLO_F32 = 0, HAFLO_F16 = 1, HAFLO_BF16 = 2 };

/*
 * Dropout: y = keep(row, col) ? x / (1 - p) : 0, plus `d_residual` (or NULL).
 * An element is dropped when its 16-bit draw is below t = rint(65536 p); kept
 * ones are scaled by 65536 / (65536 - t), so that the mean is kept for the p that
 * 16 bits can hold. Draws come from Philox4x32-10 (Salmon et al., "Parallel random
 * numbers: as easy as 1, 2, 3", 2011): counter (col >> 3, row, low and high word of `offset`), key (low and high
 * word of `seed`); the call's four words give the draws of columns 8 (col >> 3) + 0 .. 7, the low
 * half of a word first. Dropped elements are 0 whatever x holds there. The gradient by x is the same call on
 * dy without a residual; the residual's is dy. d_y may be d_x or d_residual where the distances between rows are the same (else
 * HAFLO_EINVAL). 0 <= p <= 1.
 */
int haflo_dropout(int type, const void* d_x, size_t ldx, const void* d_residual, size_t ldr, void* d_y, size_t ldy,
                  size_t rows, size_t cols, double p, uint64_t seed, uint64_t offset, void* stream);

/*
 * The shared projection with each row's own low-rank adapter. Row t has adapter
 * a = d_index[t] of `parties`, or none for -1:
 *   h[t] = scale[a] A[a] drop(x[t])            (rank values, float32; zeros without adapter)
 *   y[t] = W x[t] + B[a] h[t]
 * d_w: outer x inner; d_a: parties x rank x inner; d_b: parties x outer x rank, both dense;
 * d_scale: float32[parties]; d_index: int32[rows], in any order; drop: as haflo_dropout of the
 * rows x inner matrix x (p = 0: none), on the adapter's side only.
 * d_h: float32, rows x rank, dense; the backward pass takes it. An index outside -1 .. parties - 1 counts as
 * -1 and HAFLO_ST_RANGE is OR-ed into d_status (one device uint32, or NULL).
 * 1 <= rank <= HAFLO_ADAPTER_MAX_RANK, 1 <= parties <= HAFLO_ADAPTER_MAX_PARTIES, inner, outer >= 1, matrices of at most 2^56 elements.
 */
#define HAFLO_ADAPTER_MAX_RANK 128
#define HAFLO_ADAPTER_MAX_PARTIES 4096
size_t haflo_adapter_workspace_bytes(int type, int backward, size_t rows, size_t inner, size_t outer, size_t parties,
                                     size_t rank); /* (size_t)-1: sizes that no call accepts */
int haflo_adapter_forward(int type, const void* d_x, size_t ldx, const void* d_w, size_t ldw, const void* d_a,
                          const void* d_b, const float* d_scale, const int32_t* d_index, size_t rows, size_t inner,
                          size_t outer, size_t parties, size_t rank, double p, uint64_t seed, uint64_t offset, void* d_y,
                          size_t ldy, float* d_h, uint32_t* d_status, void* d_workspace, size_t workspace_bytes,
                          void* stream);
/*
 * Its gradients, W staying as it is, for the forward call's x, p, seed, offset and h:
 *   g[t] = scale[a] B[a]^T dy[t]
 *   dx[t] = W^T dy[t] + drop'(A[a]^T g[t])     (drop': the forward mask and factor)
 *   dA[a] = sum over a's rows of g[t] drop(x[t])^T,  dB[a] = sum over a's rows of dy[t] h[t]^T
 * d_dx (type): rows x inner, or NULL; d_da (parties x rank x inner) and d_db
 * (parties x outer x rank): float32, dense; zeros for an adapter without rows.
 */
int haflo_adapter_backward(int type, const void* d_dy, size_t lddy, const void* d_x, size_t ldx, const void* d_w,
                           size_t ldw, const void* d_a, const void* d_b, const float* d_scale, const int32_t* d_index,
                           const float* d_h, size_t rows, size_t inner, size_t outer, size_t parties, size_t rank,
                           double p, uint64_t seed, uint64_t offset, void* d_dx, size_t lddx, float* d_da, float* d_db,
                           uint32_t* d_status, void* d_workspace, size_t workspace_bytes, void* stream);

/*
 * Log-probabilities of labels under softmax(logits), row by row:
 *   lse = ln sum_j e^(x_j), logp = x_label - lse, entropy = -sum_j p_j ln p_j, p_j = e^(x_j - lse)
 * and the `top` greatest logits as (x_j - lse, j), ties to the lowest column, NaN above everything.
 * d_label: int32[rows]; -1 is a row without a label, logp 0; another label outside the
 * row counts as -1 and HAFLO_ST_RANGE is OR-ed into d_status (or NULL). Masked logits are -inf or the type's lowest
 * value; they add nothing to the entropy. A row of -inf only has lse, logp and the alternatives' values
 * -inf, entropy 0 and gradient 0. A NaN or +inf in a row makes its lse, logp, entropy and gradient NaN.
 * Outputs are float32[rows], d_top_logp float32 and d_top_index int32 rows x top (unused for top = 0).
 * top <= HAFLO_LABEL_MAX_TOP and <= cols; cols >= 1.
 */
#define HAFLO_LABEL_MAX_TOP 64
size_t haflo_label_workspace_bytes(int type, size_t rows, size_t cols, size_t top);
int haflo_label_logprobs(int type, const void* d_logits, size_t ld, const int32_t* d_label, size_t rows, size_t cols,
                         size_t top, float* d_logp, float* d_entropy, float* d_lse, float* d_top_logp,
                         int32_t* d_top_index, uint32_t* d_status, void* d_workspace, size_t workspace_bytes,
                         void* stream);
/*
 * Gradient by the logits, from the forward call's lse, entropy and d_top_index:
 *   dx_j = p_j (-(dlogp + sum_k dtop_k) - dentropy (ln p_j + entropy)) + [j = label] dlogp + sum_k [j = top_k] dtop_k
 * p_j = e^(x_j - lse) / sum_i e^(x_i - lse): the sum is formed again, so that nothing is lost where float32 holds lse coarsely, in
 * rows far from zero and of the lowest value only.
 * d_dentropy and d_dtop (rows x top) may be NULL: zeros. dlogp of a row without label is
 * not used; a top index outside the row is left out. d_dx may be d_logits where the distances between rows are the same (else HAFLO_EINVAL).
 */
int haflo_label_logprobs_backward(int type, const void* d_logits, size_t ld, const int32_t* d_label, const float* d_lse,
                                  const float* d_entropy, const float* d_dlogp, const float* d_dentropy,
                                  const int32_t* d_top_index, const float* d_dtop, size_t rows, size_t cols, size_t top,
                                  void* d_dx, size_t lddx, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HAFLO_LOCAL_H */
