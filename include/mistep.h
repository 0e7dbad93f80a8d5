/*
 * mistep: more operators of a network's training step, for AMD Instinct MI355X
 * (gfx950), as a C ABI of the same library: dropout whose mask is never stored,
 * the end of a residual branch (dropout, sum and layer norm in one pass) with
 * its backward pass, and the losses of fine-tuning by sampled answers and by
 * preferences, with their gradients.
 *
 * Ownership, streams, workspaces, errors, reproducibility, element types, rows
 * and their strides, and their limits are those of mitrain.h.  A call that
 * may write in place says so below; in place means the same pointer and the
 * same row stride.
 *
 * Random numbers.  Element (r, c) of a tensor [rows][cols] has the index e = r
 * cols + c, however the tensor lies in memory, and 16 random bits: half word e
 * mod 8 (the low half of the first word is half word 0) of the four words that
 * Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as
 * easy as 1, 2, 3", SC 2011) makes of the key {seed mod 2^32, seed / 2^32} and
 * the counter {g mod 2^32, g / 2^32, step, layer} with g = e / 8 rounded down.
 * The element is dropped where its bits are below T, the integer nearest to
 * 65536 p (the even one of two).  What is kept is scaled by k = 65536 / (65536 -
 * T), so that the mean is kept at the probability T / 65536 that takes place.
 * p is in [0, 1] (else MICONV_ERR_VALUE); at T = 65536 all are dropped, at T = 0
 * none, and the numbers are not computed.  A forward pass and its backward pass
 * take the same seed, layer and step.  A program numbers its dropouts by
 * `layer`, and raises `step` each time: a captured call does not see that, so
 * `step_at`, if it is not NULL, is a device address whose int64 is read as the
 * kernels run and added to step (modulo 2^32).
 */
#ifndef MISTEP_H
#define MISTEP_H

#include <stddef.h>
#include <hip/hip_runtime_api.h>
#include "mitrain.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * y = residual + k x where x is kept, residual where it is dropped, whatever x
 * is there.  residual may be NULL (0).  All are of type xtype, [rows][cols];
 * y may be x or residual (in place).
 */
int dropout_fwd(int xtype, long long rows, long long cols, const void *x, long long ldx,
                const void *residual, long long ldr, double p, unsigned long long seed,
                unsigned layer, unsigned step, const long long *step_at, void *y, long long ldy,
                hipStream_t stream);

/*
 * Its gradient: dx = k dy where x was kept, 0 where it was dropped.  (The
 * residual's is dy itself.)  dx may be dy (in place).
 */
int dropout_bwd(int xtype, long long rows, long long cols, const void *dy, long long lddy,
                double p, unsigned long long seed, unsigned layer, unsigned step,
                const long long *step_at, void *dx, long long lddx, hipStream_t stream);

/*
 * The end of a residual branch x [rows][cols]:
 *   total = residual + dropout(x), rounded to xtype,
 *   y, mean, rstd = the layer norm of total's rows (layernorm_fwd of mitrain.h,
 *   with its weights, eps, types and special rows).
 * total may be residual (in place); mean and rstd may be NULL.
 */
size_t residual_norm_fwd_workspace_size(int xtype, long long rows, long long cols);
int residual_norm_fwd(int xtype, int wtype, long long rows, long long cols, const void *x,
                      long long ldx, const void *residual, long long ldr, double p,
                      unsigned long long seed, unsigned layer, unsigned step,
                      const long long *step_at, const void *w, const void *b, float eps,
                      void *total, long long ldt, void *y, long long ldy, float *mean,
                      float *rstd, void *ws, size_t ws_bytes, hipStream_t stream);

/*
 * Its backward pass: with dn the gradient that layernorm_bwd gives for dy at
 * total, and dtotal [rows][cols] what reaches total beside the norm (NULL: 0),
 *   g = dn + dtotal,   dresidual = g,   dx = k g where x was kept, else 0,
 * each rounded once, and dw, db as layernorm_bwd's.  Of dresidual, dx, dw and db
 * those that are NULL are not computed (all four NULL: MICONV_ERR_NULL).  With
 * nothing dropped dx is dresidual, and one of the two is enough.  dresidual may
 * be dtotal (in place).
 */
size_t residual_norm_bwd_workspace_size(int xtype, long long rows, long long cols);
int residual_norm_bwd(int xtype, int wtype, long long rows, long long cols, const void *dy,
                      long long lddy, const void *total, long long ldt, const float *mean,
                      const float *rstd, const void *w, const void *dtotal, long long lddt,
                      double p, unsigned long long seed, unsigned layer, unsigned step,
                      const long long *step_at, void *dresidual, long long lddr, void *dx,
                      long long lddx, void *dw, void *db, void *ws, size_t ws_bytes,
                      hipStream_t stream);

/*
 * The losses take the log probabilities of tokens (logprob_fwd's, fp32) side by
 * side, sequence after sequence.  starts [seqs + 1] (int64) says where each
 * sequence begins and the last one ends: sequence s is the tokens starts[s] <= t
 * < starts[s + 1].  It does not fall, from 0 or more to `tokens` or less; numbers
 * outside of that range count as its ends, and where it falls the results are
 * unspecified.  A sequence may be empty.  mask [tokens] (bytes; NULL: all 1): a
 * token counts where it is not 0 and the token is in a sequence.  What the other
 * tensors hold of a token that does not count is not used (it may be NaN), and
 * its gradients are 0.  0 <= tokens, seqs < 2^31 (else MICONV_ERR_SHAPE).
 * Weights, sums and the log ratios that pairs add are held in 64 bits.  The gradients
 * are those of the loss, times scale (finite, else MICONV_ERR_VALUE); they are NULL
 * where they are not wanted.
 */

/*
 * The clipped policy loss of sampled tokens.  For a token that counts, with its
 * log probability lp now (logp), lo when it was sampled (old_logp) and lr under a
 * reference (ref_logp), its entropy h and its advantage a (of the token, or, if
 * by_sequence is set, of its sequence: advantages [tokens] or [seqs]):
 *   d = lp - lo,   ratio = exp(d),
 *   surrogate = -min(ratio a, clamp(ratio, 1 - clip_low, 1 + clip_high) a),
 *               for a < 0 at most -dual_clip a,
 *   kl, with x = lr - lp:   MISTEP_KL_LINEAR  -x,   _SQUARE  x^2 / 2,
 *                           _LOW  exp(x) - 1 - x   (infinite where x is; 0 without ref_logp),
 *   loss = surrogate + kl_weight kl - entropy_weight h   (h = 0 without entropy).
 * The token is clipped where a > 0 and d > ln(1 + clip_high), a < 0 and d <
 * ln(1 - clip_low), or a < 0 and d > ln(dual_clip); d is compared in 64 bits.  The
 * surrogate's slope in lp is -ratio a, and 0 where it is clipped.  Where a is 0, both are
 * 0, for an infinite ratio too.  A token's terms and slopes are of 32 bits: exponentials
 * are infinite from 2^128 on, and 0 below 2^-126.
 * Each token's weight u is, by mean:
 *   MISTEP_MEAN_TOKENS     1 / (tokens that count),
 *   MISTEP_MEAN_SEQUENCES  1 / (those of its sequence) / (sequences that have any),
 *   MISTEP_MEAN_COUNT      1 / count.
 * stats[6] (fp32) are the sums over the tokens that count of u times loss,
 * surrogate, kl, h, ratio and [clipped] (all 0 if none counts); dlogp [tokens] and
 * dentropy [tokens] the loss's gradients, what logprob_bwd takes.
 * starts may be NULL (seqs = 0): then all tokens are in one sequence, and neither
 * by_sequence nor MISTEP_MEAN_SEQUENCES is allowed (MICONV_ERR_NULL).  ref_logp
 * may be NULL if kl_weight is 0, entropy if entropy_weight is and dentropy is NULL.
 * MICONV_ERR_VALUE: clip_low outside [0, 1], clip_high below 0, dual_clip below 1
 * (infinite ones do not clip), weights that are not finite, a form or mean that is not
 * listed; for MISTEP_MEAN_COUNT, which alone reads it, a count that is not above 0 and
 * finite, or whose 1 / count or scale / count is beyond 32 bits.
 */
#define MISTEP_KL_LINEAR 0
#define MISTEP_KL_SQUARE 1
#define MISTEP_KL_LOW 2
#define MISTEP_MEAN_TOKENS 0
#define MISTEP_MEAN_SEQUENCES 1
#define MISTEP_MEAN_COUNT 2
size_t policy_loss_workspace_size(long long tokens, long long seqs);
int policy_loss(long long tokens, long long seqs, const float *logp, const float *old_logp,
                const float *ref_logp, const float *entropy, const float *advantages,
                int by_sequence, const unsigned char *mask, const long long *starts,
                double clip_low, double clip_high, double dual_clip, int kl, double kl_weight,
                double entropy_weight, int mean, double count, double scale, float *stats,
                float *dlogp, float *dentropy, void *ws, size_t ws_bytes, hipStream_t stream);

/*
 * The loss of pairs of sequences, of which the first is preferred: sequence i and
 * sequence pairs + i, for 0 <= i < pairs; starts has 2 pairs + 1 entries.  With a
 * sequence's reward
 *   R = beta sum over its tokens that count of (logp - ref_logp)
 * (ref_logp may be NULL: 0; if length_mean is set, divided by their number; 0 if
 * there is none), a pair's gap g = R_i - R_{pairs + i} and x = g - margin:
 *   MISTEP_PREFER_SIGMOID  -(1 - smoothing) ln s(x) - smoothing ln s(-x),
 *                          s(x) = 1 / (1 + exp(-x)),
 *   MISTEP_PREFER_HINGE    max(0, 1 - x),
 *   MISTEP_PREFER_SQUARED  ((x - 1/2) / beta)^2.
 * A pair none of whose tokens counts is left out; stats[5] (fp32) are the means
 * over the others of the loss, g, [g > 0], R_i and R_{pairs + i} (0 if there is no
 * other).  rewards [2 pairs] (fp32) are the R; dlogp [tokens] the mean loss's
 * gradient.  rewards and dlogp may be NULL.  beta is above 0, smoothing in [0, 1]
 * (for _SIGMOID), margin finite (else MICONV_ERR_VALUE).
 */
#define MISTEP_PREFER_SIGMOID 0
#define MISTEP_PREFER_HINGE 1
#define MISTEP_PREFER_SQUARED 2
size_t preference_loss_workspace_size(long long tokens, long long pairs);
int preference_loss(long long tokens, long long pairs, const float *logp, const float *ref_logp,
                    const unsigned char *mask, const long long *starts, double beta, int form,
                    double smoothing, double margin, int length_mean, double scale, float *stats,
                    float *rewards, float *dlogp, void *ws, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* MISTEP_H */
