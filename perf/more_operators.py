"""Dropout, residual branches, and the losses of fine-tuning, as timed cases.

Operators beside layer norm and the log probabilities of given tokens:

dropout_fwd   dropout whose mask is computed from the element's index, a seed and
              the step, and stored nowhere; added to a residual where there is one
dropout_bwd   its gradient, from the same numbers
norm_fwd      the end of a residual branch: its output, dropped out, added to the
              residual stream, and the layer norm of the sum
norm_bwd      its backward pass: the gradients of the branch, the stream, the
              weight and the bias
policy        the clipped policy loss of sampled tokens with a penalty for leaving
              a reference and an entropy bonus, and its gradients in the tokens'
              log probabilities and entropies
preference    the loss of pairs of sequences by the log ratios of policy and
              reference, and its gradient in the tokens' log probabilities

run() computes a case in plain torch operations in 32 bits (own false), or
through the package's calls (own true).  A training program keeps its outputs
and workspaces from step to step, so prepare() makes those; a single token's
calls allocate theirs.
"""
import math

import numpy
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ------------------------------------------------------------------ cases
def _drop(name, op, rows, cols, x, p, gap=0, residual=False):
    """Rows x cols of type x, elements dropped with probability p; gap elements
    of other data lie between two rows."""
    return {"name": name, "op": op, "rows": rows, "cols": cols, "x": x, "p": p, "gap": gap,
            "residual": residual}


def _norm(name, op, rows, cols, x, w, p, gap=0, passed=True):
    """Rows x cols of type x, weight and bias of type w.  passed (backward): a
    gradient reaches the sum beside the norm's."""
    return {"name": name, "op": op, "rows": rows, "cols": cols, "x": x, "w": w, "p": p,
            "gap": gap, "passed": passed}


def _policy(name, tokens, seqs, by="token", kl="", entropy=False, masked=0.0, mean="tokens",
            dual=False, tail=0):
    """Tokens in seqs sequences of random lengths, tail tokens behind the last.
    by: an advantage for each token or sequence; kl: the penalty's form, or none;
    masked: the share of tokens that do not count."""
    return {"name": name, "op": "policy", "tokens": tokens, "seqs": seqs, "by": by, "kl": kl,
            "entropy": entropy, "masked": masked, "mean": mean, "dual": dual, "tail": tail}


def _preference(name, tokens, pairs, form="sigmoid", ref=True, masked=0.0, length_mean=False,
                smoothing=0.0, margin=0.0, tail=0):
    """Tokens in 2 x pairs sequences of random lengths, the preferred ones first."""
    return {"name": name, "op": "preference", "tokens": tokens, "pairs": pairs, "form": form,
            "ref": ref, "masked": masked, "length_mean": length_mean, "smoothing": smoothing,
            "margin": margin, "tail": tail}


def listed():
    return [
        # The inner-product layers of an AlexNet-shaped network, batch 128.
        _drop("drop_inner", "dropout_fwd", 128, 4096, "f32", 0.5),
        # A branch of a block added to the residual stream, 16384 tokens.
        _drop("drop_branch", "dropout_fwd", 16384, 4096, "bf16", 0.1, residual=True),
        # The gradient of dropout over 16384 tokens of a wider layer's half.
        _drop("drop_back_tokens", "dropout_bwd", 16384, 4096, "bf16", 0.1),
        # Odd rows that lie in wider ones, as many as 64 maps of 14 x 14 pixels have.
        _drop("drop_back_odd", "dropout_bwd", 12544, 513, "f32", 0.25, gap=3),
        # Serving: the end of a branch for four new tokens, nothing dropped.
        _norm("norm_token", "norm_fwd", 4, 2048, "bf16", "bf16", 0.0),
        # Training on 16384 tokens in half precision, the weight in 32 bits.
        _norm("norm_tokens", "norm_fwd", 16384, 4096, "bf16", "f32", 0.1),
        # Its backward pass.
        _norm("norm_back_tokens", "norm_bwd", 16384, 4096, "bf16", "f32", 0.1),
        # Odd rows inside wider ones; the last block, whose sum goes nowhere else.
        _norm("norm_back_odd", "norm_bwd", 12544, 513, "f32", "f32", 0.1, gap=3, passed=False),
        # A micro-batch of eight answers, an advantage for each token.
        _policy("policy_batch", 4000, 8, kl="low", masked=0.2),
        # All answers of a large rollout, an advantage for each answer.
        _policy("policy_rollout", 2000003, 1024, by="sequence", kl="low", entropy=True, masked=0.2,
                mean="sequences", dual=True, tail=509),
        # A micro-batch of four pairs.
        _preference("pairs_batch", 4001, 4, masked=0.3),
        # The pairs of a large batch, by the means of their tokens' log ratios.
        _preference("pairs_large", 2000003, 1024, masked=0.3, length_mean=True, smoothing=0.1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly multiples of 64, now and then any number."""
    c = _log(rng, lo, hi)
    return c if rng.random() < 0.35 else max(64, (c + 32) // 64 * 64)


def _draw(rng):
    op = rng.choice(["dropout_fwd", "dropout_bwd", "norm_fwd", "norm_bwd", "norm_bwd", "policy",
                     "policy", "preference", "preference"])
    x = rng.choice(["f32", "bf16", "bf16", "f16"])
    gap = rng.choice([0, 0, 0, 1, 8, 64])
    if op.startswith("dropout"):
        case = _drop("", op, _log(rng, 1, 32768), _width(rng, 24, 131072), x,
                     rng.choice([0.1, 0.1, 0.5, 0.9]), gap, op == "dropout_fwd" and rng.random() < 0.5)
    elif op.startswith("norm"):
        case = _norm("", op, _log(rng, 1, 32768), _width(rng, 24, 131072), x,
                     rng.choice(["f32", x]), rng.choice([0.0, 0.1, 0.5]), gap,
                     rng.random() < 0.7)
    else:
        groups = _log(rng, 1, 2048)
        tokens = _log(rng, groups, 4000000)
        masked, tail = rng.choice([0.0, 0.2, 0.7]), rng.choice([0, 0, 37])
        if op == "policy":
            case = _policy("", tokens, groups, rng.choice(["token", "sequence"]),
                           rng.choice(["", "linear", "square", "low"]), rng.random() < 0.5, masked,
                           rng.choice(["tokens", "sequences"]), rng.random() < 0.3, tail)
        else:
            case = _preference("", tokens, groups, rng.choice(["sigmoid", "sigmoid", "hinge", "squared"]),
                               rng.random() < 0.8, masked, rng.random() < 0.4,
                               rng.choice([0.0, 0.1]), rng.choice([0.0, 0.5]), tail)
    case.pop("name")
    return case


def draw(rng):
    while True:
        case = _draw(rng)
        if work(case)["bytes"] <= 5.3e8:
            return case


def work(case):
    op = case["op"]
    if op == "policy":
        n = case["tokens"]
        each = 12 + 4 * (case["by"] == "token") + 4 * bool(case["kl"]) + 8 * case["entropy"] + (
            case["masked"] > 0)
        return {"bytes": n * each + case["seqs"] * (8 + 4 * (case["by"] == "sequence")),
                "flops": 30 * n}
    if op == "preference":
        n = case["tokens"]
        return {"bytes": n * (8 + 4 * case["ref"] + (case["masked"] > 0)) + case["pairs"] * 24,
                "flops": 4 * n}
    rows, b = case["rows"], _BYTES[case["x"]]
    n = rows * case["cols"]
    if op.startswith("dropout"):
        return {"bytes": n * b * (3 if case["residual"] else 2), "flops": 3 * n}
    w = case["cols"] * _BYTES[case["w"]]
    if op == "norm_fwd":
        return {"bytes": 4 * n * b + 2 * w + 8 * rows, "flops": 10 * n}
    # The stream's gradient is the branch's where nothing is dropped.
    tensors = 3 + case["passed"] + (case["p"] > 0)
    return {"bytes": tensors * n * b + 3 * w + 8 * rows, "flops": 18 * n}


# ----------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(6934 * 1000003 + seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _uniform(g, *shape):
    return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)


def _rows(case, values):
    """values [rows, cols] as the case's rows lie in memory."""
    rows, cols = values.shape
    wide = torch.zeros(rows, cols + case["gap"], dtype=_TYPES[case["x"]], device="cuda")
    x = wide[:, :cols]
    x.copy_(values)
    return x


def _starts(g, tokens, seqs):
    """Where each of seqs sequences begins, and the last one ends: random lengths,
    none among them."""
    cuts = torch.randint(tokens + 1, (seqs + 1,), generator=g, device="cuda")
    cuts[0], cuts[-1] = 0, tokens
    return torch.sort(cuts)[0]


def _tokens(case, g, seqs):
    n, last = case["tokens"], case["tokens"] - case["tail"]
    d = {"starts": _starts(g, max(0, last), seqs), "logp": -2 * _normal(g, n).abs()}
    if case["masked"]:
        # Prompts and padding: stretches of tokens, and the whole first sequence.
        m = (_uniform(g, n // 16 + 1) >= case["masked"]).repeat_interleave(16)[:n]
        if seqs > 1:
            m &= torch.arange(n, device="cuda") >= d["starts"][1]
        d["mask"] = m
    return d


def _garbage(d, g, names):
    """What padding holds: tokens without a log probability, and no numbers."""
    if "mask" in d:
        odd = _uniform(g, d["logp"].numel())
        for k in names:
            d[k].masked_fill_(~d["mask"] & (odd < 0.3), -math.inf)
            d[k].masked_fill_(~d["mask"] & (odd > 0.9), math.nan)


def _inputs(case, seed):
    g = _generator(seed)
    op = case["op"]
    numbers = {"seed": seed * 0x9E3779B97F4A7C15 % (1 << 64), "layer": seed % 97, "step": 1000 + seed % 89}
    if op == "policy":
        n = case["tokens"]
        d = _tokens(case, g, case["seqs"])
        d["old"] = d["logp"] - 0.15 * _normal(g, n)
        d["advantages"] = _normal(g, case["seqs"] if case["by"] == "sequence" else n)
        names = ["logp", "old"]
        if case["kl"]:
            d["ref"] = d["logp"] + 0.3 * _normal(g, n)
            names.append("ref")
        if case["entropy"]:
            d["entropy"] = 3 * _uniform(g, n)
            names.append("entropy")
        _garbage(d, g, names)
        return d
    if op == "preference":
        n = case["tokens"]
        d = _tokens(case, g, 2 * case["pairs"])
        names = ["logp"]
        if case["ref"]:
            d["ref"] = d["logp"] + 0.1 * _normal(g, n)
            names.append("ref")
        _garbage(d, g, names)
        return d
    rows, cols, x_type = case["rows"], case["cols"], _TYPES[case["x"]]
    d = {"numbers": numbers}
    if op == "dropout_bwd":
        d["dy"] = _rows(case, 0.01 * _normal(g, rows, cols))
        return d
    if op == "dropout_fwd":
        d["x"] = _rows(case, _normal(g, rows, cols))
        if case["residual"]:
            d["residual"] = 3 * _normal(g, rows, cols).to(x_type)
        return d
    d["w"] = (1 + 0.2 * _normal(g, cols)).to(_TYPES[case["w"]])
    # Features of unequal scale, a few far larger than the rest, and rows off zero.
    spread = 0.5 + _uniform(g, cols)
    spread[torch.randint(cols, (max(1, cols // 500),), generator=g, device="cuda")] = 20.0
    stream = _normal(g, rows, cols) * spread + 0.3 * _normal(g, rows, 1)
    if op == "norm_fwd":
        d["b"] = (0.1 * _normal(g, cols)).to(_TYPES[case["w"]])
        d["x"] = _rows(case, _normal(g, rows, cols))
        d["residual"] = stream.to(x_type)
        return d
    d["total"] = stream.to(x_type)
    d["dy"] = _rows(case, 0.01 * _normal(g, rows, cols))
    if case["passed"]:
        d["dtotal"] = (0.01 * _normal(g, rows, cols)).to(x_type)
    f = d["total"].float()
    d["mean"] = f.mean(1)
    f -= d["mean"][:, None]
    d["rstd"] = torch.rsqrt(f.square_().mean(1) + 1e-5)
    return d


def prepare(case, seed):
    d = _inputs(case, seed)
    state = {"case": dict(case), "in": d, "out": {}}
    if not own:
        return state
    import paper_1903_06934_amd as m
    op, out = case["op"], state["out"]
    if "numbers" in d:
        # The step lies on the device, so that a captured call can be replayed.
        state["numbers"] = {"seed": d["numbers"]["seed"], "layer": d["numbers"]["layer"],
                            "step": torch.tensor([d["numbers"]["step"]], device="cuda")}
    if op == "policy":
        if case["tokens"] > 65536:
            out["dlogp"] = torch.empty_like(d["logp"])
            out["ws"] = m.policy_workspace(d["logp"], d["starts"])
            if case["entropy"]:
                out["dentropy"] = torch.empty_like(d["logp"])
    elif op == "preference":
        if case["tokens"] > 65536:
            out["dlogp"] = torch.empty_like(d["logp"])
            out["ws"] = m.preference_workspace(d["logp"], d["starts"])
    elif op == "dropout_fwd":
        out["y"] = torch.empty(d["x"].shape, dtype=d["x"].dtype, device="cuda")
    elif op == "dropout_bwd":
        out["dx"] = torch.empty(d["dy"].shape, dtype=d["dy"].dtype, device="cuda")
    elif op == "norm_bwd" or case["rows"] > 64:
        like = d["x"] if op == "norm_fwd" else d["dy"]
        new = lambda: torch.empty(like.shape, dtype=like.dtype, device="cuda")
        out["ws"] = m.residual_norm_workspace(op == "norm_bwd", like)
        if op == "norm_fwd":
            out["total"], out["y"] = new(), new()
            out["mean"], out["rstd"] = (torch.empty(case["rows"], device="cuda") for _ in range(2))
        else:
            out["dresidual"] = new()
            if case["p"]:
                out["dx"] = new()
            out["dw"], out["db"] = torch.empty_like(d["w"]), torch.empty_like(d["w"])
    return state


# -------------------------------------------------------------------- run
_CLIP = (0.2, 0.28)
_DUAL = 3.0
_KL_WEIGHT, _ENTROPY_WEIGHT = 0.05, 0.01
_BETA = 0.1


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_1903_06934_amd as m
    case, d, out = state["case"], state["in"], state["out"]
    op = case["op"]
    if op == "policy":
        r = m.policy_loss(d["logp"], d["old"], d["advantages"],
                          by_sequence=case["by"] == "sequence", ref_logp=d.get("ref"),
                          entropy=d.get("entropy"), mask=d.get("mask"), starts=d["starts"],
                          clip_low=_CLIP[0], clip_high=_CLIP[1],
                          dual_clip=_DUAL if case["dual"] else math.inf, kl=case["kl"] or "low",
                          kl_weight=_KL_WEIGHT if case["kl"] else 0.0,
                          entropy_weight=_ENTROPY_WEIGHT if case["entropy"] else 0.0,
                          mean=case["mean"], **out)
        res = {"stats": r.stats, "dlogp": r.dlogp}
        if case["entropy"]:
            res["dentropy"] = r.dentropy
        return res
    if op == "preference":
        r = m.preference_loss(d["logp"], d.get("ref"), d["starts"], _BETA, form=case["form"],
                              smoothing=case["smoothing"], margin=case["margin"],
                              length_mean=case["length_mean"], mask=d.get("mask"), **out)
        return {"stats": r.stats, "rewards": r.rewards, "dlogp": r.dlogp}
    num = state["numbers"]
    if op == "dropout_fwd":
        return {"y": m.dropout_fwd(d["x"], case["p"], residual=d.get("residual"), **num, **out)}
    if op == "dropout_bwd":
        return {"dx": m.dropout_bwd(d["dy"], case["p"], **num, **out)}
    if op == "norm_fwd":
        r = m.residual_norm_fwd(d["x"], d["residual"], d["w"], d["b"], 1e-5, p=case["p"], **num,
                                **out)
        return {"total": r.total, "y": r.y, "mean": r.mean, "rstd": r.rstd}
    dx, dres, dw, db = m.residual_norm_bwd(d["dy"], d["total"], d["mean"], d["rstd"], d["w"],
                                           dtotal=d.get("dtotal"), p=case["p"], **num, **out)
    return {"dx": dx, "dresidual": dres, "dw": dw, "db": db}


_LOW = 0xFFFFFFFF


def _random(num, n):
    """The 16 bits of each of n elements: Philox 4x32 in ten rounds (Salmon, Moraes,
    Dror and Shaw, 2011), whose key is the seed, and whose counter is the elements'
    eighth, the step and the layer; an element's bits are its half word of the four."""
    group = torch.arange((n + 7) // 8, device="cuda")
    a, b = group & _LOW, group >> 32
    c = torch.full_like(group, num["step"] & _LOW)
    d = torch.full_like(group, num["layer"] & _LOW)
    k0, k1 = num["seed"] & _LOW, num["seed"] >> 32
    for _ in range(10):
        p, q = a * 0xD2511F53, c * 0xCD9E8D57
        a, b, c, d = ((q >> 32) & _LOW) ^ b ^ k0, q & _LOW, ((p >> 32) & _LOW) ^ d ^ k1, p & _LOW
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    words = torch.stack([a, b, c, d], 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).view(-1)[:n]


def _dropped(case, num, x):
    """x in 32 bits, its dropped elements 0 and the others scaled."""
    few = round(case["p"] * 65536)
    if not few:
        return x.float()
    keep = (_random(num, x.numel()) >= few).view(x.shape)
    return torch.where(keep, x.float() * (65536 / (65536 - few)), torch.zeros((), device="cuda"))


def _run_plain(state):
    case, d = state["case"], state["in"]
    op = case["op"]
    if op == "policy":
        return _plain_policy(case, d)
    if op == "preference":
        return _plain_preference(case, d)
    num = d["numbers"]
    if op == "dropout_bwd":
        return {"dx": _dropped(case, num, d["dy"]).to(d["dy"].dtype)}
    if op == "dropout_fwd":
        y = _dropped(case, num, d["x"])
        if case["residual"]:
            y = d["residual"].float() + y
        return {"y": y.to(d["x"].dtype)}
    if op == "norm_fwd":
        total = (d["residual"].float() + _dropped(case, num, d["x"])).to(d["x"].dtype)
        x = total.float()
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = torch.rsqrt((x * x).mean(1) + 1e-5)
        y = x * rstd[:, None] * d["w"].float() + d["b"].float()
        return {"total": total, "y": y.to(d["x"].dtype), "mean": mean, "rstd": rstd}
    unit = (d["total"].float() - d["mean"][:, None]) * d["rstd"][:, None]
    dy = d["dy"].float()
    dw, db = (dy * unit).sum(0), dy.sum(0)
    g = dy * d["w"].float()
    m1, m2 = g.mean(1), (g * unit).mean(1)
    g = (g - m1[:, None] - unit * m2[:, None]) * d["rstd"][:, None]
    if case["passed"]:
        g = g + d["dtotal"].float()
    return {"dx": _dropped(case, num, g).to(d["dy"].dtype), "dresidual": g.to(d["dy"].dtype),
            "dw": dw.to(d["w"].dtype), "db": db.to(d["w"].dtype)}


def _sums(values, starts):
    """The sum of each sequence's values, in 64 bits."""
    total = torch.cumsum(values.double(), 0)
    total = torch.cat([total.new_zeros(1), total])
    return total[starts[1:]] - total[starts[:-1]]


def _counted(d, n):
    """(each token's sequence, whether it counts)."""
    seqs = d["starts"].numel() - 1
    seq = torch.searchsorted(d["starts"][1:], torch.arange(n, device="cuda"), right=True)
    counted = seq < seqs
    if "mask" in d:
        counted = counted & d["mask"]
    return seq.clamp(max=seqs - 1), counted


def _plain_policy(case, d):
    n = case["tokens"]
    seq, counted = _counted(d, n)
    zero = torch.zeros((), device="cuda")
    only = lambda t: torch.where(counted, t, zero)
    logp, old = only(d["logp"]), only(d["old"])
    if case["mean"] == "tokens":
        w = 1 / counted.sum().clamp(min=1).double()
    else:
        lengths = _sums(counted, d["starts"])
        w = (1 / (lengths * (lengths > 0).sum()).clamp(min=1))[seq]
    w = torch.where(counted, w, zero.double())
    a = d["advantages"][seq] if case["by"] == "sequence" else d["advantages"]
    a = only(a)
    log_ratio = logp.double() - old.double()  # in 64 bits: some are next to the clip's border
    ratio = torch.exp(log_ratio.float())
    clipped = ((a > 0) & (log_ratio > math.log1p(_CLIP[1]))) | (
        (a < 0) & (log_ratio < math.log1p(-_CLIP[0])))
    bound = torch.where(a > 0, 1 + _CLIP[1], 1 - _CLIP[0]).float()
    if case["dual"]:
        far = (a < 0) & (log_ratio > math.log(_DUAL))
        clipped, bound = clipped | far, torch.where(far, _DUAL, bound)
    surrogate = -a * torch.where(clipped, bound, ratio)
    dlogp = torch.where(clipped, zero, -a * ratio)
    loss, kl, entropy = surrogate, zero.expand(n), zero.expand(n)
    if case["kl"]:
        x = only(d["ref"]) - logp
        if case["kl"] == "linear":
            kl, slope = -x, torch.ones_like(x)
        elif case["kl"] == "square":
            kl, slope = 0.5 * x * x, -x
        else:
            kl = (torch.expm1(x.double()) - x.double()).float()  # the two are nearly equal
            slope = -torch.expm1(x)
        loss, dlogp = loss + _KL_WEIGHT * kl, dlogp + _KL_WEIGHT * slope
    if case["entropy"]:
        entropy = only(d["entropy"])
        loss = loss - _ENTROPY_WEIGHT * entropy
    parts = torch.stack([loss, surrogate, kl, entropy, ratio, clipped.float()]).double()
    out = {"stats": (parts * w).sum(1).float(), "dlogp": (dlogp * w).float()}
    if case["entropy"]:
        out["dentropy"] = (-_ENTROPY_WEIGHT * w).float()
    return out


def _plain_preference(case, d):
    n, pairs = case["tokens"], case["pairs"]
    seq, counted = _counted(d, n)
    ratio = d["logp"].double()
    if case["ref"]:
        ratio = ratio - d["ref"].double()  # sums over whole sequences
    length = _sums(counted, d["starts"])
    reward = _sums(torch.where(counted, ratio, ratio.new_zeros(())), d["starts"])
    if case["length_mean"]:
        reward = reward / length.clamp(min=1)
    reward = _BETA * reward
    some = (length[:pairs] > 0) | (length[pairs:] > 0)  # a pair without a token is none
    share = some / some.sum().clamp(min=1)
    gap = reward[:pairs] - reward[pairs:]
    x = gap - case["margin"]
    if case["form"] == "hinge":
        loss, slope = (1 - x).clamp(min=0), torch.where(x < 1, -1.0, 0.0).double()
    elif case["form"] == "squared":
        u = (x - 0.5) / _BETA
        loss, slope = u * u, 2 * u / _BETA
    else:
        e = case["smoothing"]
        log_sum = torch.log1p(torch.exp(-x.abs()))
        loss = (1 - e) * (log_sum + (-x).clamp(min=0)) + e * (log_sum + x.clamp(min=0))
        slope = torch.sigmoid(x) - (1 - e)
    each = slope * share * _BETA
    each = torch.cat([each, -each])
    if case["length_mean"]:
        each = each / length.clamp(min=1)
    dlogp = torch.where(counted, each[seq], each.new_zeros(())).float()
    stats = torch.stack([loss, gap, (gap > 0).double(), reward[:pairs], reward[pairs:]])
    return {"stats": (stats * share).sum(1).float(), "rewards": reward.float(), "dlogp": dlogp}


# ------------------------------------------------------------------ exact
def exact(case, seed):
    """The outputs from their definitions in 64 bits."""
    d = _inputs(case, seed)
    op = case["op"]
    if op in ("policy", "preference"):
        host = {k: v.cpu().numpy() for k, v in d.items()}
        with numpy.errstate(all="ignore"):
            out = (_exact_policy if op == "policy" else _exact_preference)(case, host)
        return {k: torch.from_numpy(v).cuda() for k, v in out.items()}
    rows, cols = case["rows"], case["cols"]
    kept = _exact_kept(case, d["numbers"], rows * cols)
    step = max(1, (1 << 25) // cols)
    parts = []
    for i in range(0, rows, step):
        r = slice(i, min(rows, i + step))
        keep = None if kept is None else kept[r.start * cols:r.stop * cols].view(-1, cols)
        parts.append(_exact_rows(case, d, r, keep))
    out = {}
    for k in parts[0]:
        v = [p[k] for p in parts]
        out[k] = torch.stack(v).sum(0) if k in ("dw", "db") else torch.cat(v)
    return out


def _exact_kept(case, num, n):
    """Which of n elements are kept; the generator's products by 16-bit digits."""
    few = round(case["p"] * 65536)
    if not few:
        return None
    group = torch.arange((n + 7) // 8, device="cuda")
    state = [group % (1 << 32), group // (1 << 32), torch.zeros_like(group) + num["step"],
             torch.zeros_like(group) + num["layer"]]
    key = [num["seed"] % (1 << 32), num["seed"] // (1 << 32)]

    def product(v, c):
        low, high = (v % 65536) * c, (v // 65536) * c  # below 2^48
        low_word = low % (1 << 32) + (high % 65536) * 65536
        return low // (1 << 32) + high // 65536 + low_word // (1 << 32), low_word % (1 << 32)

    for i in range(10):
        h0, l0 = product(state[0], 0xD2511F53)
        h1, l1 = product(state[2], 0xCD9E8D57)
        round_key = [(key[0] + i * 0x9E3779B9) % (1 << 32), (key[1] + i * 0xBB67AE85) % (1 << 32)]
        state = [h1 ^ state[1] ^ round_key[0], l1, h0 ^ state[3] ^ round_key[1], l0]
    kept = torch.empty(group.numel(), 8, dtype=torch.bool, device="cuda")
    for i in range(8):
        kept[:, i] = state[i // 2] // 65536 ** (i % 2) % 65536 >= few
    return kept.view(-1)[:n]


def _exact_rows(case, d, r, keep):
    op = case["op"]
    few = round(case["p"] * 65536)

    def dropped(v):
        return v if keep is None else (v * keep) * 65536 / (65536 - few)

    if op == "dropout_bwd":
        return {"dx": dropped(d["dy"][r].double())}
    if op == "dropout_fwd":
        y = dropped(d["x"][r].double())
        return {"y": y + d["residual"][r].double() if case["residual"] else y}
    w = d["w"].double()
    if op == "norm_fwd":
        total = d["residual"][r].double() + dropped(d["x"][r].double())
        # The norm is that of the sum as it is stored.
        x = total.to(d["x"].dtype).double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + 1e-5)
        y = torch.addcmul(d["b"].double(), (x - mean[:, None]) * rstd[:, None], w)
        return {"total": total, "y": y, "mean": mean, "rstd": rstd}
    n = case["cols"]
    dy, rstd = d["dy"][r].double(), d["rstd"][r].double()[:, None]
    unit = (d["total"][r].double() - d["mean"][r].double()[:, None]) * rstd
    g = dy * w
    # The Jacobian of a row: rstd (1 - P), P the projection on the row's ones and
    # normalised features.
    back = rstd * (g - g.sum(1, keepdim=True) / n - unit * ((unit * g).sum(1, keepdim=True) / n))
    if case["passed"]:
        back = back + d["dtotal"][r].double()
    return {"dx": dropped(back), "dresidual": back, "dw": (unit * dy).sum(0), "db": dy.sum(0)}


def _exact_policy(case, d):
    n, seqs, starts = case["tokens"], case["seqs"], d["starts"]
    stats = numpy.zeros(6)
    dlogp, weight = numpy.zeros(n), numpy.zeros(n)
    mask = d.get("mask", numpy.ones(n, bool))
    where = [numpy.flatnonzero(mask[starts[s]:starts[s + 1]]) + starts[s] for s in range(seqs)]
    counts = [len(w) for w in where]
    for s, at in enumerate(where):
        if not len(at):
            continue
        w = 1 / sum(counts) if case["mean"] == "tokens" else 1 / (len(at) * sum(map(bool, counts)))
        logp, old = (d[k][at].astype(numpy.float64) for k in ("logp", "old"))
        a = d["advantages"].astype(numpy.float64)
        a = numpy.full(len(at), a[s]) if case["by"] == "sequence" else a[at]
        ratio = numpy.exp(logp - old)
        gain = numpy.minimum(ratio * a, numpy.clip(ratio, 1 - _CLIP[0], 1 + _CLIP[1]) * a)
        if case["dual"]:
            gain = numpy.where(a < 0, numpy.maximum(gain, _DUAL * a), gain)
        # Clipped: the gain does not move with the ratio (an advantage of 0 aside).
        clipped = (gain != ratio * a) & (a != 0)
        each = [-gain, numpy.zeros(len(at)), numpy.zeros(len(at)), ratio, clipped]
        slope = numpy.where(clipped, 0, -ratio * a)
        if case["kl"]:
            x = d["ref"][at].astype(numpy.float64) - logp
            each[1], kl_slope = {"linear": (-x, 1.0), "square": (x * x / 2, -x),
                                 "low": (numpy.expm1(x) - x, -numpy.expm1(x))}[case["kl"]]
            slope = slope + _KL_WEIGHT * kl_slope
        if case["entropy"]:
            each[2] = d["entropy"][at].astype(numpy.float64)
        stats[1:] += [w * float(v.sum()) for v in each]
        dlogp[at], weight[at] = w * slope, w
    stats[0] = stats[1]
    if case["kl"]:
        stats[0] += _KL_WEIGHT * stats[2]
    if case["entropy"]:
        stats[0] -= _ENTROPY_WEIGHT * stats[3]
    out = {"stats": stats, "dlogp": dlogp}
    if case["entropy"]:
        out["dentropy"] = -_ENTROPY_WEIGHT * weight
    return out


def _exact_preference(case, d):
    n, pairs, starts = case["tokens"], case["pairs"], d["starts"]
    mask = d.get("mask", numpy.ones(n, bool))
    rewards, dlogp, stats = numpy.zeros(2 * pairs), numpy.zeros(n), numpy.zeros(5)
    where = [numpy.flatnonzero(mask[starts[s]:starts[s + 1]]) + starts[s] for s in range(2 * pairs)]
    for s, at in enumerate(where):
        v = d["logp"][at].astype(numpy.float64)
        if case["ref"]:
            v = v - d["ref"][at]
        rewards[s] = _BETA * float(v.sum()) / (max(1, len(at)) if case["length_mean"] else 1)
    given = [i for i in range(pairs) if len(where[i]) + len(where[pairs + i])]
    for i in given:
        gap = rewards[i] - rewards[pairs + i]
        x, e = gap - case["margin"], case["smoothing"]
        if case["form"] == "hinge":
            loss, slope = max(0.0, 1 - x), -1.0 if x < 1 else 0.0
        elif case["form"] == "squared":
            loss, slope = (gap - case["margin"] - 0.5) ** 2 / _BETA ** 2, (2 * x - 1) / _BETA ** 2
        else:
            loss = (1 - e) * numpy.logaddexp(0, -x) + e * numpy.logaddexp(0, x)
            slope = e / (1 + numpy.exp(-x)) - (1 - e) / (1 + numpy.exp(x))
        stats += numpy.array([loss, gap, gap > 0, rewards[i], rewards[pairs + i]]) / len(given)
        for s, sign in ((i, 1), (pairs + i, -1)):
            per = len(where[s]) if case["length_mean"] else 1
            dlogp[where[s]] = sign * slope * _BETA / len(given) / max(1, per)
    return {"stats": stats, "rewards": rewards, "dlogp": dlogp}
