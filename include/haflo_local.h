/*
 * haflo_local.h - operators of a party's local step, on plain values.
 *
 * A party of a federated model trains on its own data between two aggregations.
 * Where the model is large, what it trains, and what is then encrypted and
 * aggregated (haflo.h), is a low-rank adapter beside a projection that all
 * parties share. The operators of that step are here: dropout whose mask is
 * never stored, the shared projection with every row's own adapter and its
 * gradients, and the log-probabilities of labels with entropy, top alternatives
 * and gradient (logistic regression's loss for two classes or any number); the
 * norms around a block of such a model, and orthogonalised updates of adapters.
 * The common model's answers may take its projections in eight bits.
 * Gradients of adapters are float32, as haflo_encode_f32 takes them.
 *
 * The conventions of haflo.h hold: 0 or a negative HAFLO_E* code, no exception,
 * device pointers and sizes, a stream, no allocation and no synchronisation,
 * kernels only (a sequence of calls can be captured into a HIP graph). A call
 * works on the current device. Every sum is held in 32 bits or more; a result is
 * rounded to its type once. Results do not depend on timing: the same call on the
 * same device gives the same bits.
 *
 * Matrices are row-major; `ld*` is the distance between rows in elements, at
 * least the row's length. Elements need no more alignment than their type's, a workspace that of 16 bytes (else HAFLO_EINVAL). Outputs
 * may not overlap inputs except where it says so, and there from the same address on; that they do not overlap otherwise is not looked for. Counts are below 2^31.
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

/*
 * The norms around a block of a model, with its gate and the residual stream, row by row:
 *   p = f / sqrt(mean f^2 + eps) * post   (d_post NULL: p = f)
 *   r = scale x + gate * p,   h = r / sqrt(mean r^2 + eps) * pre
 * x: the stream before the block, f: what the block gave, r: the stream behind it (d_r), h: what the next block takes (d_h). The gate is
 * d_gate (rows x cols), or d_gate_cols for all rows (float32[cols]), or 1 where both are NULL. d_pre NULL: no h. d_f
 * NULL: only h, of r = x, and scale has to be 1; not both NULL.
 * d_post, d_pre: float32[cols]. d_rstd: float32, 2 x rows, both roots' reciprocals (1 where there is no norm), which the
 * backward pass takes. h is formed from r before its rounding; means of squares are held in 64 bits. d_r and d_h may each be one of the
 * inputs where the distances between rows are the same (else HAFLO_EINVAL). cols >= 1; 2^-254 <= eps, finite; scale finite in float32.
 */
int haflo_residual_norm(int type, const void* d_x, size_t ldx, const void* d_f, size_t ldf, const float* d_post,
                        const void* d_gate, size_t ldg, const float* d_gate_cols, const float* d_pre, size_t rows,
                        size_t cols, double scale, double eps, void* d_r, size_t ldr, void* d_h, size_t ldh,
                        float* d_rstd, void* stream);
/*
 * Its gradients, for the forward call's arguments and its d_rstd, from dh (where there is h) and dr (NULL: zeros), the
 * gradient that r has from elsewhere:
 *   D = dr + gradient of h by r,   dx = scale D,   dgate = D * p (d_dgate, or summed over rows: d_dgate_cols),
 *   df = gradient of p by f for gate * D,   dpost, dpre: sums over rows
 * Each output may be NULL. dx, df, dgate: of `type`, each may be one of the inputs where the distances between rows are the same
 * (else HAFLO_EINVAL); dpost, dgate_cols, dpre: float32[cols], zeros for no rows.
 */
size_t haflo_residual_norm_workspace_bytes(int type, size_t rows, size_t cols);
int haflo_residual_norm_backward(int type, const void* d_dh, size_t lddh, const void* d_dr, size_t lddr, const void* d_x,
                                 size_t ldx, const void* d_f, size_t ldf, const float* d_post, const void* d_gate,
                                 size_t ldg, const float* d_gate_cols, const float* d_pre, const float* d_rstd,
                                 size_t rows, size_t cols, double scale, void* d_dx, size_t lddx, void* d_df, size_t lddf,
                                 void* d_dgate, size_t lddg, float* d_dgate_cols, float* d_dpost, float* d_dpre,
                                 void* d_workspace, size_t workspace_bytes, void* stream);

/*
 * Newton-Schulz orthogonalisation of `parties` matrices of rows x cols, of which the shorter side is at most
 * HAFLO_ADAPTER_MAX_RANK, as an adapter's gradient is:
 *   X = G / (|G|_F + eps);  for each step (a, b, c): K = X X^T, X <- a X + (b K + c K^2) X;   out = keep base + scale X
 * (of a matrix with more rows than columns K = X^T X, from the right). d_coefficients: host memory, steps x 3; five times
 * (3.4445, -4.7750, 2.0315) brings singular values between about 0.7 and 1.2, (1.5, -0.5, 0) towards 1. d_base NULL: none.
 * Matrices lie step_* elements apart; those of the result behind one another or with all their rows between each other's (else HAFLO_EINVAL). All products are held in 64 bits: X is off by some
 * 2^-53 of what the steps raise a direction by together (2^-29 of its greatest element for 512 and less). A list that raises by more
 * than 512 (five steps of 3.4445 do not) has K formed again from X on the way, by readings of G. A NaN or an infinity in a matrix makes its X NaN; one of
 * zeros gives X = 0. d_out may be d_g or d_base where all distances are the same (else HAFLO_EINVAL).
 * 1 <= steps <= HAFLO_UPDATE_MAX_STEPS, parties <= HAFLO_ADAPTER_MAX_PARTIES, parties times the longer side <= 2^38, ldo <= 2^32,
 * eps > 0, all factors finite.
 */
#define HAFLO_UPDATE_MAX_STEPS 16
size_t haflo_update_workspace_bytes(int type, size_t parties, size_t rows, size_t cols);
int haflo_orthogonal_update(int type, const void* d_g, size_t ldg, size_t step_g, const void* d_base, size_t ldb,
                            size_t step_b, size_t parties, size_t rows, size_t cols, const double* coefficients, int steps,
                            double keep, double scale, double eps, void* d_out, size_t ldo, size_t step_o, void* d_workspace,
                            size_t workspace_bytes, void* stream);

/*
 * Rows of eight bits: scale = amax / 127 and q = rint(x (127 / amax)), -127 .. 127, of each row, the quotients and the product
 * rounded to float32. d_q: rows of HAFLO_INT8_ROW * ceil(cols / HAFLO_INT8_ROW) bytes, dense, zeros behind the columns, at a 16-byte
 * boundary. A row of zeros has scale 0; a row with a NaN or an infinity has scale NaN and q = 0.
 * 1 <= cols <= HAFLO_INT8_MAX_COLS.
 */
#define HAFLO_INT8_ROW 128
#define HAFLO_INT8_MAX_COLS 130944
int haflo_quantize_rows(int type, const void* d_x, size_t ldx, size_t rows, size_t cols, int8_t* d_q, float* d_scale,
                        void* stream);
/*
 * A projection with weights of eight bits, as the common model answers with:
 *   y[t, o] = x_scale[t] w_scale[o] sum_k xq[t, k] wq[o, k] + bias[o] + residual[t, o]
 * d_xq, d_wq (outer rows): as haflo_quantize_rows lays them out, of `inner` columns; sums are exact. rows * outer <= 2^42. d_bias: float32[outer] or NULL;
 * d_residual (type, rows x outer) or NULL; d_y may be d_residual where the distances between rows are the same (else HAFLO_EINVAL).
 */
int haflo_int8_product(int type, const int8_t* d_xq, const float* d_x_scale, const int8_t* d_wq, const float* d_w_scale,
                       const float* d_bias, const void* d_residual, size_t ldr, size_t rows, size_t inner, size_t outer,
                       void* d_y, size_t ldy, void* stream);
/*
 * The same of x (type, rows x inner), which is brought to eight bits first, in the workspace. d_y may be d_x too, however far apart the rows of
 * either; the workspace is then at least that of 17 rows (else HAFLO_EINVAL), as calls of up to 16 rows may need none otherwise.
 */
size_t haflo_int8_workspace_bytes(int type, size_t rows, size_t inner, size_t outer);
int haflo_int8_forward(int type, const void* d_x, size_t ldx, const int8_t* d_wq, const float* d_w_scale,
                       const float* d_bias, const void* d_residual, size_t ldr, size_t rows, size_t inner, size_t outer,
                       void* d_y, size_t ldy, void* d_workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* HAFLO_LOCAL_H */
