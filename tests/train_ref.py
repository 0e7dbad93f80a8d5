"""Plain 64-bit forms of the training step's operators (include/mitrain.h), on
CPU torch tensors, with the magnitudes that the tests' bounds are multiples of.
They share no code with the library."""
import math

import torch

U = 2.0 ** -24  # half a unit in the last place of 1, in 32 bits
INF = math.inf


def half_ulp(values, dtype):
    """Half the spacing of dtype at these values: what one rounding may cost."""
    bits, low = {torch.float32: (24, -149), torch.bfloat16: (8, -133),
                 torch.float16: (11, -24)}[dtype]
    exp = torch.frexp(values.abs().double())[1].double()
    exp = torch.where(torch.isfinite(values), exp, torch.zeros_like(exp))
    exp = torch.where(values == 0, torch.full_like(exp, low), exp)
    return 2.0 ** (torch.clamp(exp - bits, min=low) - 1)


# ---------------------------------------------------------------- layer norm
def layernorm_fwd(x, w=None, b=None, eps=1e-5):
    """(y, mean, rstd, scale of y's errors, scale of mean's)."""
    x = x.double()
    n = x.shape[1]
    w = torch.ones(n, dtype=torch.float64) if w is None else w.double()
    b = torch.zeros(n, dtype=torch.float64) if b is None else b.double()
    mean = x.sum(1) / n
    d = x - mean[:, None]
    rstd = 1 / torch.sqrt((d * d).sum(1) / n + eps)
    unit = d * rstd[:, None]
    y = unit * w + b
    size = x.abs().sum(1) / n
    return y, mean, rstd, (unit * w).abs() + b.abs() + (rstd * size)[:, None] * w.abs(), size


def layernorm_bwd(dy, x, mean, rstd, w=None):
    """((dx, scale), (dw, scale), (db, scale)); mean and rstd as given."""
    x, dy, mean, rstd = x.double(), dy.double(), mean.double(), rstd.double()
    n = x.shape[1]
    w = torch.ones(n, dtype=torch.float64) if w is None else w.double()
    u = (x - mean[:, None]) * rstd[:, None]
    g = dy * w
    m1, m2 = g.sum(1) / n, (g * u).sum(1) / n
    dx = rstd[:, None] * (g - m1[:, None] - u * m2[:, None])
    size = rstd[:, None] * (g.abs() + (g.abs().sum(1) / n)[:, None]
                            + u.abs() * ((g * u).abs().sum(1) / n)[:, None])
    return ((dx, size), ((dy * u).sum(0), (dy * u).abs().sum(0)), (dy.sum(0), dy.abs().sum(0)))


# --------------------------------------------------------- log probabilities
def logprob_fwd(z, targets=None, top=0, scale=1.0):
    """dict of logp, lse, entropy, stats, top_logp, top_index (the definition, with the
    special rows as the header states them)."""
    raw = z.double()
    s = raw * float(torch.tensor(scale, dtype=torch.float32))
    rows, vocab = s.shape
    out = {k: torch.zeros(rows, dtype=torch.float64) for k in ("logp", "lse", "entropy")}
    out["stats"] = torch.zeros(rows, 2, dtype=torch.float64)
    out["top_logp"] = torch.zeros(rows, top, dtype=torch.float64)
    out["top_index"] = torch.zeros(rows, top, dtype=torch.int64)
    for r in range(rows):
        row = s[r]
        bad = bool((torch.isnan(row) | (row == INF)).any())
        empty = bool((row == -INF).all())
        if bad:
            lp = torch.full_like(row, math.nan)
            lse, entropy, logsum = math.nan, math.nan, math.nan
        elif empty:
            lp, lse, entropy, logsum = row, -INF, 0.0, 0.0
        else:
            m = row.max()
            logsum = float(torch.log(torch.exp(row - m).sum()))
            lse = float(m) + logsum
            lp = row - m - logsum  # exact where lse rounds the sum away
            p = torch.exp(lp)
            entropy = -float(torch.where(p > 0, p * lp, torch.zeros_like(p)).sum())
        out["lse"][r], out["entropy"][r] = lse, entropy
        out["stats"][r, 0] = raw[r][~torch.isnan(raw[r])].max() if not raw[r].isnan().all() else -INF
        out["stats"][r, 1] = logsum
        if targets is not None and targets[r] >= 0:
            out["logp"][r] = lp[targets[r]] if targets[r] < vocab else math.nan
        if top:
            rank = torch.where(torch.isnan(raw[r]), torch.full_like(row, -INF), raw[r])
            keys = sorted(range(vocab), key=lambda j: (-float(rank[j]), j))[:top]
            out["top_index"][r] = torch.tensor(keys)
            out["top_logp"][r] = lp[keys]
    return out


def logprob_bwd(z, targets, scale, stats, dlogp=None, entropy=None, dentropy=None):
    """(dz, scale of its errors); stats and entropy as given."""
    raw = z.double()
    scale = float(torch.tensor(scale, dtype=torch.float32))
    rows, vocab = raw.shape
    dz, size = torch.zeros_like(raw), torch.zeros_like(raw)
    for r in range(rows):
        dl = 0.0
        if dlogp is not None and targets[r] >= 0:
            dl = float(dlogp[r]) if targets[r] < vocab else math.nan
        de = 0.0 if dentropy is None else float(dentropy[r])
        h = 0.0 if dentropy is None else float(entropy[r])
        if stats[r, 0] == -INF and stats[r, 1] == 0:
            dz[r] = 0.0 if dl == dl else math.nan
            continue
        lp = (raw[r] - float(stats[r, 0])) * scale - float(stats[r, 1])
        p = torch.exp(lp)
        lp = torch.where(p > 0, lp, torch.zeros_like(lp))
        one = torch.zeros(vocab, dtype=torch.float64)
        if dl == dl and dl != 0.0:
            one[targets[r]] = 1.0
        dz[r] = scale * (dl * (one - p) - de * p * (lp + h))
        size[r] = scale * (abs(dl) * (one + p * (1 + lp.abs()))
                           + abs(de) * p * (1 + lp.abs()) * (lp.abs() + abs(h)))
    return dz, size


# ------------------------------------------------------------------ clipping
def clip(grads, max_norm):
    """(norm, clipped gradients)."""
    norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in grads))
    max_norm = float(torch.tensor(max_norm, dtype=torch.float32))
    f = 1.0 if norm <= max_norm else max_norm / norm
    return norm, [g.double() * f for g in grads]


def assert_close(got, want, bound, what):
    """Each element within its bound; infinities and NaN in the same places."""
    got, want = got.detach().cpu().double(), want.double()
    bound = torch.as_tensor(bound, dtype=torch.float64).expand_as(want)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    fin = torch.isfinite(want)
    odd = ~fin & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd]), f"{what}: infinities differ"
    err = (got - want).abs()[fin]
    lim = bound[fin]
    bad = ~(err <= lim)
    if bad.any():
        i = int(torch.argmax(err - lim))
        raise AssertionError(f"{what}: {int(bad.sum())}/{bad.numel()} off; worst got "
                             f"{float(got[fin][i])!r} want {float(want[fin][i])!r} "
                             f"err {float(err[i]):.3e} bound {float(lim[i]):.3e}")
