"""Plain 64-bit forms of the operators of include/mistep.h, on CPU torch tensors, with
the magnitudes that the tests' bounds are multiples of.  They share no code with the
library."""
import math

import numpy as np
import torch

from train_ref import U


# --------------------------------------------------------------------- dropout
def philox(counter, key):
    """Philox4x32-10 of one counter (four words) and key (two words), in Python's
    integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p, q = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def threshold(p):
    return round(p * 65536)


def kept(elements, p, seed, layer=0, step=0):
    """Which of the elements with these indices (an int64 array) are kept."""
    e = np.asarray(elements, np.uint64)
    g, inverse = np.unique(e >> np.uint64(3), return_inverse=True)
    low = np.uint64(0xFFFFFFFF)
    c = [g & low, g >> np.uint64(32), np.full_like(g, step % (1 << 32)), np.full_like(g, layer)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low,
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    words = np.stack(c, 1).astype(np.uint32)[inverse.ravel()]
    h = (e & np.uint64(7)).astype(np.int64)
    bits = words[np.arange(len(e)), h // 2] >> (16 * (h % 2)).astype(np.uint32) & 0xFFFF
    return torch.from_numpy(bits.astype(np.int64) >= threshold(p))


def mask_of(rows, cols, p, seed, layer=0, step=0):
    return kept(np.arange(rows * cols), p, seed, layer, step).view(rows, cols)


def scale_of(p):
    t = threshold(p)
    return 65536 / (65536 - t) if t < 65536 else 0.0


def dropout(x, keep, p, residual=None):
    """(y, scale of its errors)."""
    x = x.double()
    v = torch.where(keep, x * scale_of(p), torch.zeros_like(x))
    y = v if residual is None else v + residual.double()
    # The scale's rounding and the product's, then the sum's.
    return y, 2 * v.abs() + y.abs()


# ---------------------------------------------------------------------- losses
def sequences(starts, tokens):
    """[(first, end)] of the sequences, cut to the tokens."""
    s = [min(max(int(v), 0), tokens) for v in starts]
    return [(a, max(a, b)) for a, b in zip(s[:-1], s[1:])]


def policy(logp, old, adv, by_sequence=False, ref=None, entropy=None, mask=None, starts=None,
           low=0.2, high=0.2, dual=math.inf, kl="low", kl_weight=0.0, entropy_weight=0.0,
           mean="tokens", scale=1.0):
    """((stats, their bounds), (dlogp, bounds), (dentropy, bounds)).

    The bounds count, in u = 2^-24: d's rounding moves the ratio by |d| u of it, its
    exponential by 2 u, the clip's border and the products by 1 u each; x's rounding moves
    the divergence by its slope; the series' terms and additions cost 8 u of it, and
    from |x| = 1 on, where it is a difference, 4 u of the terms; each sum of the loss, the
    weight 1 / n and the last rounding 1 u.  A term joins the sum of at most eight tokens by
    a fused product and addition in 32 bits, and passes the additions after it: at most
    8 roundings, each of at most u times the absolute values added so far, so that all of
    them cost at most 8 u of the terms' absolute values; what comes after is in 64 bits."""
    n = logp.numel()
    counted = torch.zeros(n, dtype=torch.bool)
    weight = torch.zeros(n, dtype=torch.float64)
    a = torch.zeros(n, dtype=torch.float64)
    on = torch.ones(n, dtype=torch.bool) if mask is None else mask.bool()
    ranges = [(0, n)] if starts is None else sequences(starts, n)
    given = 0
    for s, (b, e) in enumerate(ranges):
        here = torch.zeros(n, dtype=torch.bool)
        here[b:e] = on[b:e]
        counted |= here
        c = int(here.sum())
        given += c > 0
        if c:
            weight[here] = 1.0 / c if mean == "sequences" else 1.0
        a[b:e] = adv[s].double() if by_sequence else adv[b:e].double()
    if mean == "tokens":
        weight /= max(1, int(counted.sum()))
    elif mean == "sequences":
        weight /= max(1, given)
    else:
        weight /= mean
    zero = torch.zeros(n, dtype=torch.float64)
    only = lambda t: torch.where(counted, t.double(), zero)
    lp, lo, a = only(logp), only(old), only(a)
    d = lp - lo
    ratio = torch.exp(d)
    border = torch.where(a > 0, 1 + high, 1 - low)
    clipped = ((a > 0) & (d > math.log1p(high))) | (
        (a < 0) & (d < (math.log1p(-low) if low < 1 else -math.inf)))
    far = (a < 0) & (d > math.log(dual))
    border = torch.where(far, torch.full_like(border, dual), border)
    clipped |= far
    r = torch.where(clipped, border, ratio)
    surrogate = -a * r
    size_s = (surrogate.abs() * (5 + d.abs())).nan_to_num(0, 0, 0)
    slope = torch.where(clipped, zero, -a * ratio)
    size_g = torch.where(clipped, zero, size_s)
    loss, size_l = surrogate.clone(), size_s.clone()
    div, size_k = zero.clone(), zero.clone()
    if ref is not None:
        x = only(ref) - lp
        ex = torch.expm1(x)
        one = torch.ones_like(x)
        div, dslope, moved = {"linear": (-x, one, zero), "square": (x * x / 2, -x, one),
                              "low": (ex - x, -ex, torch.exp(x))}[kl]
        step = {"linear": one, "square": x.abs(), "low": ex.abs()}[kl]
        big = (x.abs() >= 0.999).double() * (torch.exp(x) + 1 + x.abs())
        size_k = 8 * div.abs() + x.abs() * step + (4 * big if kl == "low" else zero)
        size_d = 8 * dslope.abs() + x.abs() * moved + (4 * big if kl == "low" else zero)
        if kl_weight:
            loss += kl_weight * div
            slope = slope + kl_weight * dslope
            size_l += abs(kl_weight) * (size_k + 2 * div.abs())
            size_g = size_g + abs(kl_weight) * (size_d + 2 * dslope.abs())
    h = zero
    added = surrogate.abs() + abs(kl_weight) * div.abs()
    if entropy is not None:
        h = only(entropy)
        if entropy_weight:
            loss -= entropy_weight * h
            size_l += abs(entropy_weight) * 2 * h.abs()
            added = added + abs(entropy_weight) * h.abs()
    parts = [(loss, size_l + 9 * added), (surrogate, size_s), (div, size_k), (h, zero),
             (ratio, ratio * (3 + d.abs())), (clipped.double(), zero)]
    w = lambda v: torch.where(counted, v * weight, zero)
    stats = torch.stack([w(v).sum() for v, _ in parts])
    bounds = torch.stack([w(s + 9 * v.abs()).sum() for v, s in parts]) * U + U * stats.abs()
    g, gh = w(slope) * scale, w(torch.full_like(zero, -entropy_weight)) * scale
    return ((stats, bounds.nan_to_num(0, 0, 0) + 1e-40),
            (g, U * (abs(scale) * w(size_g) + 5 * g.abs()).nan_to_num(0, 0, 0) + 1e-40),
            (gh, 4 * U * gh.abs() + 1e-40))


def preference(logp, ref, starts, beta, form="sigmoid", smoothing=0.0, margin=0.0,
               length_mean=False, mask=None, scale=1.0):
    """((stats, their bounds), (rewards, bounds), (dlogp, bounds)).

    The bounds count one rounding of each token's ratio; what comes after is in 64 bits,
    up to one rounding of each result.  The losses move with a gap by their slope, the
    gradients by their curvature."""
    n = logp.numel()
    on = torch.ones(n, dtype=torch.bool) if mask is None else mask.bool()
    ranges = sequences(starts, n)
    pairs = len(ranges) // 2
    rewards = torch.zeros(2 * pairs, dtype=torch.float64)
    off = torch.zeros(2 * pairs, dtype=torch.float64)
    where, count = [], []
    for s, (b, e) in enumerate(ranges):
        at = torch.nonzero(on[b:e])[:, 0] + b
        v = logp[at].double()
        if ref is not None:
            v = v - ref[at].double()
        div = max(1, len(at)) if length_mean else 1
        rewards[s] = beta * float(v.sum()) / div
        off[s] = beta * float(v.abs().sum()) / div * U
        where.append(at)
        count.append(len(at))
    stats, bounds = np.zeros(5), np.zeros(5)
    dlogp, gb = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
    given = [i for i in range(pairs) if count[i] + count[pairs + i]]
    for i in given:
        gap = float(rewards[i] - rewards[pairs + i])
        moved = float(off[i] + off[pairs + i])
        x = gap - margin
        if form == "hinge":
            loss, slope, bend = max(0.0, 1 - x), -1.0 if x < 1 else 0.0, 0.0
        elif form == "squared":
            loss, slope, bend = ((x - 0.5) / beta) ** 2, 2 * (x - 0.5) / beta ** 2, 2 / beta ** 2
        else:
            up, down = float(np.logaddexp(0, -x)), float(np.logaddexp(0, x))
            loss = (1 - smoothing) * up + smoothing * down
            s = math.exp(-up)
            slope, bend = smoothing * s - (1 - smoothing) * math.exp(-down), 0.25
        stats += np.array([loss, gap, gap > 0, rewards[i], rewards[pairs + i]]) / len(given)
        bounds += np.array([abs(slope) * moved + bend * moved ** 2, moved, 0, float(off[i]),
                            float(off[pairs + i])]) / len(given)
        for s, sign in ((i, 1), (pairs + i, -1)):
            div = max(1, count[s]) if length_mean else 1
            f = scale * beta / len(given) / div
            dlogp[where[s]] = sign * slope * f
            gb[where[s]] = abs(f) * bend * moved
    stats = torch.from_numpy(stats)
    return ((stats, torch.from_numpy(bounds) * 1.01 + 2 * U * stats.abs() + 1e-40),
            (rewards, off * 1.01 + U * rewards.abs() + 1e-40),
            (dlogp, gb * 1.01 + 2 * U * dlogp.abs() + 1e-40))
