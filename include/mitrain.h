/*
 * mitrain: the operators around the layers of miconv.h that begin and end a
 * network's training step, for AMD Instinct MI355X (gfx950), as a C ABI of
 * the same library: layer norm with its backward pass, log probabilities of
 * given tokens (or classes) with their gradient, and the global norm of a list
 * of gradients with their clipping.
 *
 * Ownership, streams, workspaces, errors and reproducibility are those of
 * miconv.h: device pointers owned by the caller, kernels enqueued on `stream`
 * without synchronising, no device memory allocated or pointer kept, every
 * argument check before any launch, statuses of miconv_status, results bit
 * for bit the same for the same arguments and device (sums run in a fixed
 * order).  As the calls only launch kernels, they can be captured into a HIP
 * graph.  Two things differ: a tensor has an element type, one of
 * MITRAIN_F32, _BF16 and _F16, and needs its type's alignment only (else
 * MICONV_ERR_ALIGN; the workspace 16 bytes); and a tensor of rows has a row
 * stride: row r of x begins at element r * ldx, its elements lie side by side.
 * A row stride is at least the row's length.  Two tensors of rows may be
 * interleaved (columns of one wider matrix), where both have the same stride
 * in bytes; an output overlaps no other tensor otherwise (MICONV_ERR_ALIAS).
 * Rows are below 2^31 and may be 0, a row's elements below 2^29, rows times row
 * stride at most 2^48 elements, rows times elements 2^37 (MICONV_ERR_SHAPE
 * otherwise).
 *
 * Sums, statistics and what stands between the steps below are held in 32 bits
 * or more; a result is rounded once to its type, to nearest even.
 */
#ifndef MITRAIN_H
#define MITRAIN_H

#include <stddef.h>
#include <hip/hip_runtime_api.h>
#include "miconv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MITRAIN_F32 0
#define MITRAIN_BF16 1
#define MITRAIN_F16 2

/*
 * Layer norm of each row of x [rows][cols]:
 *   mean = sum_j x_j / cols,  rstd = 1 / sqrt(sum_j (x_j - mean)^2 / cols + eps),
 *   y_j = (x_j - mean) rstd w_j + b_j.
 * x and y are of type xtype; w and b [cols] of type wtype, which is xtype or
 * MITRAIN_F32 (else MICONV_ERR_TYPE); either may be NULL (w = 1, b = 0).  mean
 * and rstd [rows] are fp32, what the backward pass takes; each may be NULL.
 * eps >= 0 and finite (else MICONV_ERR_VALUE).  cols >= 1.  A row of equal
 * elements has that number as its mean and b as its result, but with eps = 0 no
 * norm (NaN), nor has one with an infinity or NaN.  A row's sum and its sum of
 * squares about the mean are held in 32 bits, and have to be within their range.
 */
size_t layernorm_fwd_workspace_size(int xtype, long long rows, long long cols);
int layernorm_fwd(int xtype, int wtype, long long rows, long long cols, const void *x,
                  long long ldx, const void *w, const void *b, float eps, void *y, long long ldy,
                  float *mean, float *rstd, void *ws, size_t ws_bytes, hipStream_t stream);

/*
 * Its backward pass.  With u_j = (x_j - mean) rstd and g_j = dy_j w_j in a row,
 *   dx_j = rstd (g_j - sum_i g_i / cols - u_j sum_i g_i u_i / cols),
 *   dw_j = sum over the rows of dy_j u_j,   db_j = sum over the rows of dy_j.
 * dy, x and dx are of type xtype; w, dw and db of type wtype.  mean and rstd
 * are the forward pass's.  w may be NULL (w = 1); of dx, dw and db those that
 * are NULL are not computed (all three NULL: MICONV_ERR_NULL).  Without rows,
 * dw and db are 0.
 */
size_t layernorm_bwd_workspace_size(int xtype, long long rows, long long cols);
int layernorm_bwd(int xtype, int wtype, long long rows, long long cols, const void *dy,
                  long long lddy, const void *x, long long ldx, const float *mean,
                  const float *rstd, const void *w, void *dx, long long lddx, void *dw, void *db,
                  void *ws, size_t ws_bytes, hipStream_t stream);

/*
 * Log probabilities under the softmax of scale z for each row z of logits
 * [rows][vocab] of type xtype:
 *   lse = ln sum_j exp(scale z_j),     logp = scale z_t - lse of the given token t,
 *   entropy = -sum_j p_j ln p_j  with  p_j = exp(scale z_j - lse),
 *   stats = {peak, ln sum_j exp(scale (z_j - peak))}  with  peak = max_j z_j,
 * which [rows][2] the backward pass takes (lse = scale peak + the sum's
 * logarithm; taken apart, logits far from 0 keep their probabilities),
 * and the `top` likeliest tokens: top_index [rows][top], in falling order of z,
 * of equal ones the lowest index first, and top_logp [rows][top], their log
 * probabilities.  logp, lse, entropy, stats and top_logp are fp32, targets and
 * top_index int64.
 *   - targets[r] < 0: no token is given, logp = 0 and its gradient 0; at or
 *     above vocab: logp and the row's gradient are NaN.
 *   - a logit of -inf bans its token (p = 0).  A row that bans all: lse and
 *     every log probability -inf, entropy 0, stats {-inf, 0}, the gradient 0.
 *     Tokens at the type's lowest value are not banned: a row of nothing else
 *     is as likely for all of them at any scale, though its lse may be beyond
 *     32 bits, and then is -inf.
 *   - a NaN or +inf in a row makes its lse, log probabilities, entropy,
 *     stats' sum and gradient NaN; for top_index a NaN counts as -inf.
 * 1e-6 <= scale <= 1e6 (else MICONV_ERR_VALUE).  vocab >= 1; 0 <= top <=
 * min(vocab, MITRAIN_TOP_MAX) (else MICONV_ERR_SHAPE).  targets is required for
 * logp, top_logp and top_index for top > 0; logp, lse, entropy and stats may be
 * NULL.
 */
#define MITRAIN_TOP_MAX 64
size_t logprob_fwd_workspace_size(int xtype, long long rows, long long vocab, int top);
int logprob_fwd(int xtype, long long rows, long long vocab, const void *logits, long long ldl,
                const long long *targets, float scale, int top, float *logp, float *lse,
                float *entropy, float *stats, float *top_logp, long long *top_index, void *ws, size_t ws_bytes,
                hipStream_t stream);

/*
 * The gradient in the logits of  sum over the rows of dlogp logp + dentropy
 * entropy (dlogp and dentropy fp32 [rows], e.g. -1 / rows for a mean loss):
 *   dz_j = scale (dlogp ([j = t] - p_j) - dentropy p_j (ln p_j + entropy)).
 * stats and entropy are the forward pass's.  dlogp needs targets; dentropy needs
 * entropy; one of the two may be NULL (0), not both.  dlogits is of the
 * logits' type and may be the logits themselves (same pointer and row stride).
 */
int logprob_bwd(int xtype, long long rows, long long vocab, const void *logits, long long ldl,
                const long long *targets, float scale, const float *stats, const float *dlogp,
                const float *entropy, const float *dentropy, void *dlogits, long long ldd,
                hipStream_t stream);

/*
 * The global norm of n gradients, and their clipping to max_norm:
 *   norm = sqrt(sum over the tensors of the sum of g^2),
 *   out = g f  with  f = 1 where norm <= max_norm, else max_norm / norm.
 * grads and out are host arrays of n device pointers, count their elements
 * (>= 0, at most 2^37 in all), types their element types; the arrays are read
 * before the calls return.  out[i] may be grads[i] (clipping in place); the
 * tensors of out overlap no other tensor, nor norm or ws (MICONV_ERR_ALIAS).
 * The squares are summed in 64 bits, so their sum neither overflows nor loses
 * small ones; norm is one fp32 element (NULL in grad_clip: not wanted).  A NaN
 * among the gradients makes norm and every output NaN; an infinite one makes
 * norm infinite, and out 0, or NaN where g is infinite.  max_norm >= 0, not NaN
 * (else MICONV_ERR_VALUE); infinite: nothing is clipped.  A pointer may be NULL
 * where its count is 0; n may be 0 (norm 0).
 */
size_t grad_workspace_size(int n, const long long *count, const int *types);
int grad_norm(int n, const void *const *grads, const long long *count, const int *types,
              float *norm, void *ws, size_t ws_bytes, hipStream_t stream);
int grad_clip(int n, const void *const *grads, const long long *count, const int *types,
              float max_norm, void *const *out, float *norm, void *ws, size_t ws_bytes,
              hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MITRAIN_H */
