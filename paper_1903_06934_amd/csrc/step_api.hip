// C ABI of more of the training step's operators (declared in include/mistep.h):
// argument validation and launches on the caller's stream.
#include <math.h>
#include <stddef.h>

#include "mistep.h"
#include "checks.h"
#include "internal.h"
#include "step.h"

namespace miconv {

namespace {

constexpr long long kMaxTokens = (1LL << 31) - 1;

// false: p is no probability.
bool make_drop(double p, unsigned long long seed, unsigned layer, unsigned step,
               const long long *step_at, Drop *d)
{
    if (!(p >= 0 && p <= 1))
        return false;
    const double below = nearbyint(p * 65536);
    *d = Drop{(uint32_t)below,
              (uint32_t)seed,
              (uint32_t)(seed >> 32),
              step,
              layer,
              below < 65536 ? (float)(65536 / (65536 - below)) : 0.f,
              step_at};
    return true;
}

// The tensor to check beside an output: none, if the output is written in place.
const void *beside(const void *in, long long ldi, const void *out, long long ldo)
{
    return in == out && ldi == ldo ? nullptr : in;
}

bool in_floats(double v) { return isfinite(v) && isfinite((float)v); }

}  // namespace
}  // namespace miconv

using namespace miconv;

extern "C" {

int dropout_fwd(int xtype, long long rows, long long cols, const void *x, long long ldx,
                const void *residual, long long ldr, double p, unsigned long long seed,
                unsigned layer, unsigned step, const long long *step_at, void *y, long long ldy,
                hipStream_t stream)
{
    if (!known_type(xtype))
        return MICONV_ERR_TYPE;
    if (!good_shape(rows, cols) || !good_stride(rows, cols, ldx) ||
        !good_stride(rows, cols, ldy) || (residual && !good_stride(rows, cols, ldr)))
        return MICONV_ERR_SHAPE;
    DropoutArgs a{rows, cols, {x, ldx}, {residual, ldr}, {y, ldy}, {}};
    if (!make_drop(p, seed, layer, step, step_at, &a.drop))
        return MICONV_ERR_VALUE;
    const void *other = beside(x, ldx, y, ldy);
    const Buffer bufs[] = {
        rows_of(other, rows, cols, ldx, xtype, false, !x),
        rows_of(beside(residual, ldr, y, ldy), rows, cols, ldr, xtype, false, false),
        flat(step_at, 8, 8, false, false),
        rows_of(y, rows, cols, ldy, xtype, true, true),
    };
    int st = check(bufs, 4, nullptr, 0, 0);
    if (st != MICONV_OK || (st = ready()) != MICONV_OK)
        return st;
    return launch_status(launch_dropout(xtype, a, stream));
}

int dropout_bwd(int xtype, long long rows, long long cols, const void *dy, long long lddy,
                double p, unsigned long long seed, unsigned layer, unsigned step,
                const long long *step_at, void *dx, long long lddx, hipStream_t stream)
{
    return dropout_fwd(xtype, rows, cols, dy, lddy, nullptr, 0, p, seed, layer, step, step_at, dx,
                       lddx, stream);
}

size_t residual_norm_fwd_workspace_size(int xtype, long long rows, long long cols)
{
    return layernorm_fwd_workspace_size(xtype, rows, cols);
}

size_t residual_norm_bwd_workspace_size(int xtype, long long rows, long long cols)
{
    return layernorm_bwd_workspace_size(xtype, rows, cols);
}

int residual_norm_fwd(int xtype, int wtype, long long rows, long long cols, const void *x,
                      long long ldx, const void *residual, long long ldr, double p,
                      unsigned long long seed, unsigned layer, unsigned step,
                      const long long *step_at, const void *w, const void *b, float eps,
                      void *total, long long ldt, void *y, long long ldy, float *mean,
                      float *rstd, void *ws, size_t ws_bytes, hipStream_t stream)
{
    if (!known_type(xtype) || (wtype != xtype && wtype != MITRAIN_F32))
        return MICONV_ERR_TYPE;
    if (!good_shape(rows, cols) || !good_stride(rows, cols, ldx) ||
        !good_stride(rows, cols, ldr) || !good_stride(rows, cols, ldt) ||
        !good_stride(rows, cols, ldy))
        return MICONV_ERR_SHAPE;
    ResidualFwdArgs a{};
    if (!(eps >= 0) || !isfinite(eps) || !make_drop(p, seed, layer, step, step_at, &a.drop))
        return MICONV_ERR_VALUE;
    const size_t wsize = type_size(wtype);
    const Buffer bufs[] = {
        rows_of(x, rows, cols, ldx, xtype, false, true),
        rows_of(beside(residual, ldr, total, ldt), rows, cols, ldr, xtype, false, !residual),
        flat(step_at, 8, 8, false, false),
        flat(w, cols * (long long)wsize, wsize, false, false),
        flat(b, cols * (long long)wsize, wsize, false, false),
        rows_of(total, rows, cols, ldt, xtype, true, true),
        rows_of(y, rows, cols, ldy, xtype, true, true),
        flat(mean, rows * 4, 4, true, false),
        flat(rstd, rows * 4, 4, true, false),
    };
    int st = check(bufs, 9, ws, ws_bytes, residual_norm_fwd_workspace_size(xtype, rows, cols));
    if (st != MICONV_OK || (st = ready()) != MICONV_OK)
        return st;
    (NormFwdArgs &)a =
        NormFwdArgs{rows, cols, {x, ldx}, w, b, eps, {y, ldy}, mean, rstd, (float *)ws};
    a.residual = {residual, ldr};
    a.total = {total, ldt};
    return launch_status(launch_residual_fwd(xtype, wtype == MITRAIN_F32, a, stream));
}

int residual_norm_bwd(int xtype, int wtype, long long rows, long long cols, const void *dy,
                      long long lddy, const void *total, long long ldt, const float *mean,
                      const float *rstd, const void *w, const void *dtotal, long long lddt,
                      double p, unsigned long long seed, unsigned layer, unsigned step,
                      const long long *step_at, void *dresidual, long long lddr, void *dx,
                      long long lddx, void *dw, void *db, void *ws, size_t ws_bytes,
                      hipStream_t stream)
{
    if (!known_type(xtype) || (wtype != xtype && wtype != MITRAIN_F32))
        return MICONV_ERR_TYPE;
    if (!good_shape(rows, cols) || !good_stride(rows, cols, lddy) ||
        !good_stride(rows, cols, ldt) || (dtotal && !good_stride(rows, cols, lddt)) ||
        (dresidual && !good_stride(rows, cols, lddr)) || (dx && !good_stride(rows, cols, lddx)))
        return MICONV_ERR_SHAPE;
    ResidualBwdArgs a{};
    if (!make_drop(p, seed, layer, step, step_at, &a.drop))
        return MICONV_ERR_VALUE;
    if (!dresidual && !dx && !dw && !db)
        return MICONV_ERR_NULL;
    const size_t wsize = type_size(wtype);
    const Buffer bufs[] = {
        rows_of(dy, rows, cols, lddy, xtype, false, true),
        rows_of(total, rows, cols, ldt, xtype, false, true),
        flat(mean, rows * 4, 4, false, rows > 0),
        flat(rstd, rows * 4, 4, false, rows > 0),
        flat(w, cols * (long long)wsize, wsize, false, false),
        rows_of(beside(dtotal, lddt, dresidual, lddr), rows, cols, lddt, xtype, false, false),
        flat(step_at, 8, 8, false, false),
        rows_of(dresidual, rows, cols, lddr, xtype, true, false),
        rows_of(dx, rows, cols, lddx, xtype, true, false),
        flat(dw, cols * (long long)wsize, wsize, true, false),
        flat(db, cols * (long long)wsize, wsize, true, false),
    };
    int st = check(bufs, 11, ws, ws_bytes, residual_norm_bwd_workspace_size(xtype, rows, cols));
    if (st != MICONV_OK || (st = ready()) != MICONV_OK)
        return st;
    (NormBwdArgs &)a = NormBwdArgs{rows, cols, {dy, lddy}, {total, ldt}, mean,       rstd,
                                   w,    {dx, lddx}, dw,   db,           (float *)ws};
    a.dtotal = {dtotal, lddt};
    a.dresidual = {dresidual, lddr};
    return launch_status(launch_residual_bwd(xtype, wtype == MITRAIN_F32, a, stream));
}

size_t policy_loss_workspace_size(long long tokens, long long seqs)
{
    return tokens < 0 || tokens > kMaxTokens || seqs < 0 || seqs > kMaxTokens
               ? 0
               : policy_ws(tokens, seqs);
}

int policy_loss(long long tokens, long long seqs, const float *logp, const float *old_logp,
                const float *ref_logp, const float *entropy, const float *advantages,
                int by_sequence, const unsigned char *mask, const long long *starts,
                double clip_low, double clip_high, double dual_clip, int kl, double kl_weight,
                double entropy_weight, int mean, double count, double scale, float *stats,
                float *dlogp, float *dentropy, void *ws, size_t ws_bytes, hipStream_t stream)
{
    if (tokens < 0 || tokens > kMaxTokens || seqs < 0 || seqs > kMaxTokens || (!starts && seqs))
        return MICONV_ERR_SHAPE;
    if (!(clip_low >= 0 && clip_low <= 1) || !(clip_high >= 0) || !(dual_clip >= 1) ||
        kl < MISTEP_KL_LINEAR || kl > MISTEP_KL_LOW || !in_floats(kl_weight) ||
        !in_floats(entropy_weight) || mean < MISTEP_MEAN_TOKENS || mean > MISTEP_MEAN_COUNT ||
        (mean == MISTEP_MEAN_COUNT &&
         !(count > 0 && isfinite(count) && in_floats(1 / count) && in_floats(scale / count))) ||
        !in_floats(scale))
        return MICONV_ERR_VALUE;
    if (!starts && (by_sequence || mean == MISTEP_MEAN_SEQUENCES))
        return MICONV_ERR_NULL;
    const bool some = tokens > 0;
    const long long adv = by_sequence ? seqs : tokens;
    const Buffer bufs[] = {
        flat(logp, tokens * 4, 4, false, some),
        flat(old_logp, tokens * 4, 4, false, some),
        flat(ref_logp, tokens * 4, 4, false, some && kl_weight != 0),
        flat(entropy, tokens * 4, 4, false, some && (entropy_weight != 0 || dentropy)),
        flat(advantages, adv * 4, 4, false, adv > 0),
        flat(mask, tokens, 1, false, false),
        flat(starts, starts ? (seqs + 1) * 8 : 0, 8, false, false),
        flat(stats, 6 * 4, 4, true, true),
        flat(dlogp, tokens * 4, 4, true, false),
        flat(dentropy, tokens * 4, 4, true, false),
    };
    int st = check(bufs, 10, ws, ws_bytes, policy_loss_workspace_size(tokens, seqs));
    if (st != MICONV_OK || (st = ready()) != MICONV_OK)
        return st;
    const PolicyArgs a{(int)tokens,
                       (int)seqs,
                       logp,
                       old_logp,
                       ref_logp,
                       entropy,
                       advantages,
                       by_sequence != 0,
                       mask,
                       starts,
                       log1p(-clip_low),
                       log1p(clip_high),
                       log(dual_clip),
                       (float)(1 - clip_low),
                       (float)(1 + clip_high),
                       (float)dual_clip,
                       kl,
                       (float)kl_weight,
                       (float)entropy_weight,
                       mean,
                       mean == MISTEP_MEAN_COUNT ? count : 1.0,
                       scale,
                       stats,
                       dlogp,
                       dentropy,
                       ws};
    return launch_status(launch_policy(a, stream));
}

size_t preference_loss_workspace_size(long long tokens, long long pairs)
{
    return tokens < 0 || tokens > kMaxTokens || pairs < 0 || pairs > kMaxTokens / 2
               ? 0
               : preference_ws(tokens, pairs);
}

int preference_loss(long long tokens, long long pairs, const float *logp, const float *ref_logp,
                    const unsigned char *mask, const long long *starts, double beta, int form,
                    double smoothing, double margin, int length_mean, double scale, float *stats,
                    float *rewards, float *dlogp, void *ws, size_t ws_bytes, hipStream_t stream)
{
    if (tokens < 0 || tokens > kMaxTokens || pairs < 0 || pairs > kMaxTokens / 2)
        return MICONV_ERR_SHAPE;
    if (!(beta > 0) || !in_floats(beta) || form < MISTEP_PREFER_SIGMOID ||
        form > MISTEP_PREFER_SQUARED || !(smoothing >= 0 && smoothing <= 1) || !in_floats(margin) ||
        !in_floats(scale))
        return MICONV_ERR_VALUE;
    const Buffer bufs[] = {
        flat(logp, tokens * 4, 4, false, tokens > 0),
        flat(ref_logp, tokens * 4, 4, false, false),
        flat(mask, tokens, 1, false, false),
        flat(starts, (2 * pairs + 1) * 8, 8, false, true),
        flat(stats, 5 * 4, 4, true, true),
        flat(rewards, pairs * 8, 4, true, false),
        flat(dlogp, tokens * 4, 4, true, false),
    };
    int st = check(bufs, 7, ws, ws_bytes, preference_loss_workspace_size(tokens, pairs));
    if (st != MICONV_OK || (st = ready()) != MICONV_OK)
        return st;
    const PreferenceArgs a{(int)tokens, (int)pairs, logp,  ref_logp, mask,    starts, beta, form,
                           smoothing,   margin,     length_mean != 0, scale, stats, rewards, dlogp, ws};
    return launch_status(launch_preference(a, stream));
}

}  // extern "C"
