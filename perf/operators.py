"""The end of a network's training step, and the scoring of its answers, as timed cases.

Four operators beside the convolution, pooling and inner-product layers:

norm_fwd      layer norm of rows of features, with the statistics that its
              backward pass takes
norm_bwd      its backward pass: the gradients of the rows, and those of the
              weight and the bias, summed over the rows
logprob_fwd   log probabilities of given tokens (or classes) under the softmax
              of each row of logits, with its entropy, its k likeliest
              alternatives and the statistics that the backward pass takes
logprob_bwd   the gradient of these log probabilities and entropies in the logits
clip          the global norm of a list of gradients and their clipping to it

run() computes a case in plain torch operations in 32 bits (own false), or
through the package's calls (own true).  A training program keeps its outputs
and workspaces from step to step, so prepare() makes those; a single token's
calls allocate theirs.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}


# ------------------------------------------------------------------ cases
def _norm(name, op, rows, cols, x, w, gap=0):
    """Layer norm of rows x cols of type x, weight and bias of type w; gap
    elements of other data lie between two rows of x."""
    return {"name": name, "op": op, "rows": rows, "cols": cols, "x": x, "w": w, "gap": gap}


def _logits(name, op, rows, vocab, x, top=0, scale=1.0, banned=0.0, skipped=0.0, entropy=False):
    """Rows of vocab logits of type x at inverse temperature scale, a share of
    them banned (-inf); a share of the rows has no given token (-1).  entropy:
    its gradient is wanted too (backward)."""
    return {"name": name, "op": op, "rows": rows, "vocab": vocab, "x": x, "top": top,
            "scale": scale, "banned": banned, "skipped": skipped, "entropy": entropy}


def listed():
    return [
        # The smallest call: the norm of four new tokens in serving, bound by
        # its launch.
        _norm("norm_token", "norm_fwd", 4, 2048, "bf16", "bf16"),
        # Training on 16384 tokens in half precision, the weight in 32 bits.
        _norm("norm_tokens", "norm_fwd", 16384, 4096, "bf16", "f32"),
        # Its backward pass.
        _norm("norm_back_tokens", "norm_bwd", 16384, 4096, "bf16", "f32"),
        # Odd rows that lie in wider ones (a slice of a fused projection),
        # as many as 64 maps of 14 x 14 pixels have.
        _norm("norm_back_odd", "norm_bwd", 12544, 513, "f32", "f32", gap=3),
        # Whole feature maps of a convolution layer (512 x 14 x 14) as rows: few
        # and long.
        _norm("norm_back_maps", "norm_bwd", 32, 100352, "f32", "f32"),
        # Four sequences' next-token logits in serving: the sampled tokens' log
        # probabilities and twenty alternatives, some tokens banned.
        _logits("logprob_next", "logprob_fwd", 4, 131072, "bf16", top=20, scale=1.25, banned=0.02),
        # A classifier's loss and its five best classes over a batch of images.
        _logits("logprob_classes", "logprob_fwd", 128, 1000, "f32", top=5),
        # A training step's loss over 4096 tokens, a tenth of them prompt.
        _logits("logprob_train", "logprob_fwd", 4096, 32000, "bf16", skipped=0.1),
        # Its gradient.
        _logits("logprob_back_train", "logprob_bwd", 4096, 32000, "bf16", skipped=0.1),
        # The gradient with an entropy bonus, an odd number of tokens.
        _logits("logprob_back_bonus", "logprob_bwd", 509, 8191, "f32", entropy=True),
        # The gradients of the convolution and inner-product layers of an
        # AlexNet-shaped network, in 32 bits.
        {"name": "clip_convnet", "op": "clip", "shape": "convnet", "depth": 0, "width": 0,
         "x": "f32", "max_norm": 1.0},
        # Many tensors: 24 blocks of width 512, matrices in half precision,
        # norms and biases in 32 bits.
        {"name": "clip_blocks", "op": "clip", "shape": "blocks", "depth": 24, "width": 512,
         "x": "bf16", "max_norm": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly multiples of 64, now and then any number."""
    c = _log(rng, lo, hi)
    return c if rng.random() < 0.35 else max(64, (c + 32) // 64 * 64)


def _draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "norm_bwd", "logprob_fwd", "logprob_fwd",
                     "logprob_bwd", "logprob_bwd", "clip"])
    if op in ("norm_fwd", "norm_bwd"):
        x = rng.choice(["f32", "bf16", "bf16", "f16"])
        case = _norm("", op, _log(rng, 1, 32768), _width(rng, 24, 131072), x,
                     rng.choice(["f32", x]), gap=rng.choice([0, 0, 0, 1, 8, 64]))
    elif op == "clip":
        case = {"op": op, "shape": "blocks", "depth": rng.randint(1, 40),
                "width": _log(rng, 24, 1024), "x": rng.choice(["f32", "bf16", "f16"]),
                "max_norm": rng.choice([0.1, 1.0, 1000.0])}
    else:
        back = op == "logprob_bwd"
        case = _logits("", op, _log(rng, 1, 8192), _log(rng, 10, 200000),
                       rng.choice(["f32", "bf16", "bf16", "f16"]),
                       top=0 if back else rng.choice([0, 1, 5, 10, 20]),
                       scale=rng.choice([1.0, 1.0, 0.7, 1.25]),
                       banned=rng.choice([0.0, 0.0, 0.02, 0.5]),
                       skipped=rng.choice([0.0, 0.1]), entropy=back and rng.random() < 0.4)
    case.pop("name", None)
    return case


def draw(rng):
    while True:
        case = _draw(rng)
        if case["op"] == "logprob_fwd" and case["top"] and case["rows"] * case["vocab"] > 1 << 24:
            continue  # the plain form sorts every row
        if work(case)["bytes"] <= 5.2e8:
            return case


def _tensors(case):
    """The (elements, type) of a clip case's gradients, in the order of the layers."""
    if case["shape"] == "convnet":
        filters = [(96, 3 * 121), (256, 48 * 25), (384, 256 * 9), (384, 192 * 9), (256, 192 * 9),
                   (4096, 9216), (4096, 4096), (1000, 4096)]
        return [(n, case["x"]) for k, c in filters for n in (k * c, k)]
    d, x = case["width"], case["x"]
    block = [(d, "f32"), (d, "f32"), (3 * d * d, x), (3 * d, "f32"), (d * d, x), (d, "f32"),
             (d, "f32"), (d, "f32"), (4 * d * d, x), (4 * d, "f32"), (4 * d * d, x), (d, "f32")]
    return block * case["depth"]


def work(case):
    op = case["op"]
    if op == "clip":
        sizes = _tensors(case)
        n = sum(s for s, _ in sizes)
        return {"bytes": 2 * sum(s * _BYTES[t] for s, t in sizes) + 4, "flops": 3 * n}
    rows, b = case["rows"], _BYTES[case["x"]]
    if op in ("norm_fwd", "norm_bwd"):
        n, w = rows * case["cols"], case["cols"] * _BYTES[case["w"]]
        if op == "norm_fwd":
            return {"bytes": 2 * n * b + 2 * w + 8 * rows, "flops": 8 * n}
        return {"bytes": 3 * n * b + 3 * w + 8 * rows, "flops": 15 * n}
    n = rows * case["vocab"]
    if op == "logprob_fwd":
        return {"bytes": n * b + rows * (8 + 20 + 12 * case["top"]), "flops": 6 * n}
    return {"bytes": 2 * n * b + rows * (20 + (8 if case["entropy"] else 0)), "flops": 8 * n}


# ----------------------------------------------------------------- inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1903 * 1000003 + seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _uniform(g, *shape):
    return torch.rand(shape, generator=g, device="cuda", dtype=torch.float32)


def _inputs(case, seed):
    g = _generator(seed)
    if case["op"] == "clip":
        # One scale for each tensor: gradients differ from layer to layer.
        return {"grads": [(_normal(g, n) * 10 ** float(-2 - 2 * _uniform(g, 1).item())).to(_TYPES[t])
                          for n, t in _tensors(case)]}
    x_type, rows = _TYPES[case["x"]], case["rows"]
    if case["op"] in ("norm_fwd", "norm_bwd"):
        # Features of unequal scale, a few far larger than the rest, and rows
        # off zero.
        cols = case["cols"]
        spread = 0.5 + _uniform(g, cols)
        spread[torch.randint(cols, (max(1, cols // 500),), generator=g, device="cuda")] = 20.0
        wide = torch.zeros(rows, cols + case["gap"], dtype=x_type, device="cuda")
        x = wide[:, :cols]
        x.copy_(_normal(g, rows, cols) * spread + 0.3 * _normal(g, rows, 1))
        d = {"x": x, "w": (1 + 0.2 * _normal(g, cols)).to(_TYPES[case["w"]]),
             "b": (0.1 * _normal(g, cols)).to(_TYPES[case["w"]])}
        if case["op"] == "norm_bwd":
            d["dy"] = (0.01 * _normal(g, rows, cols)).to(x_type)
            f = x.float()
            d["mean"] = f.mean(1)
            f -= d["mean"][:, None]
            d["rstd"] = torch.rsqrt(f.square_().mean(1) + 1e-5)
        return d
    vocab = case["vocab"]
    z = 2.5 * _normal(g, rows, vocab)
    if case["banned"]:
        ban = _uniform(g, rows, vocab) < case["banned"]
        ban[:, 0] = False  # a token is left in each row
        z.masked_fill_(ban, -math.inf)
    z = z.to(x_type)
    # Given tokens: one that the row's softmax favours, or any that is not banned.
    pick = torch.randint(vocab, (rows, 8), generator=g, device="cuda")
    best = z.gather(1, pick).max(1)
    given = torch.where(best[0] == -math.inf, torch.zeros_like(best[1]),
                        pick.gather(1, best[1][:, None])[:, 0])
    given = torch.where(_uniform(g, rows) < case["skipped"], torch.full_like(given, -1), given)
    d = {"logits": z, "targets": given}
    if case["op"] == "logprob_bwd":
        d["dlogp"] = -_uniform(g, rows) / rows  # a weighted mean of the losses
        f = z.float()
        peak = f.max(1)[0]
        s = (f - peak[:, None]) * case["scale"]
        d["stats"] = torch.stack([peak, torch.logsumexp(s, 1)], 1)
        if case["entropy"]:
            s -= d["stats"][:, 1:]
            d["entropy"] = -torch.where(s == -math.inf, torch.zeros_like(s), s * s.exp()).sum(1)
            d["dentropy"] = -0.01 * _uniform(g, rows) / rows
    return d


def prepare(case, seed):
    d = _inputs(case, seed)
    state = {"case": dict(case), "in": d, "out": {}}
    if not own:
        return state
    import paper_1903_06934_amd as m
    out = state["out"]
    if case["op"] == "clip":
        # The clipped gradients lie one after the other in a buffer for each
        # type, as an all-reduce or an optimizer over flat buffers takes them.
        total = {}
        for t in d["grads"]:
            total[t.dtype] = total.get(t.dtype, 0) + t.numel()
        out["flat"] = {k: torch.empty(n, dtype=k, device="cuda") for k, n in total.items()}
        out["clipped"], used = [], dict.fromkeys(total, 0)
        for t in d["grads"]:
            at = used[t.dtype]
            used[t.dtype] = at + t.numel()
            out["clipped"].append(out["flat"][t.dtype][at:at + t.numel()])
        out["norm"] = torch.empty(1, device="cuda")
        out["ws"] = m.grad_workspace(d["grads"])
    elif case["op"] == "norm_bwd" or (case["op"] == "norm_fwd" and case["rows"] > 64):
        rows, cols = case["rows"], case["cols"]
        out["ws"] = m.layernorm_workspace(case["op"] == "norm_bwd", d["x"])
        if case["op"] == "norm_bwd":
            out["dx"] = torch.empty(rows, cols, dtype=d["x"].dtype, device="cuda")
            out["dw"], out["db"] = torch.empty_like(d["w"]), torch.empty_like(d["w"])
        else:
            out["y"] = torch.empty(rows, cols, dtype=d["x"].dtype, device="cuda")
            out["mean"], out["rstd"] = (torch.empty(rows, device="cuda") for _ in range(2))
    elif case["op"] == "logprob_bwd":
        out["dlogits"] = torch.empty_like(d["logits"])
    return state


# -------------------------------------------------------------------- run
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_1903_06934_amd as m
    case, d, out = state["case"], state["in"], state["out"]
    op = case["op"]
    if op == "norm_fwd":
        y, mean, rstd = m.layernorm_fwd(d["x"], d["w"], d["b"], 1e-5, **out)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_bwd":
        dx, dw, db = m.layernorm_bwd(d["dy"], d["x"], d["mean"], d["rstd"], d["w"], **out)
        return {"dx": dx, "dw": dw, "db": db}
    if op == "logprob_fwd":
        r = m.logprob_fwd(d["logits"], d["targets"], top=case["top"], scale=case["scale"])
        res = {"logp": r.logp, "lse": r.lse, "entropy": r.entropy, "stats": r.stats}
        if case["top"]:
            res.update(top_logp=r.top_logp, top_index=r.top_index)
        return res
    if op == "logprob_bwd":
        return {"dlogits": m.logprob_bwd(d["logits"], d["stats"], d["targets"], d["dlogp"],
                                         d.get("entropy"), d.get("dentropy"),
                                         scale=case["scale"], **out)}
    norm = m.grad_clip(d["grads"], case["max_norm"], out=out["clipped"], norm=out["norm"],
                       ws=out["ws"])
    return {"norm": norm, **_by_type(out["flat"])}


def _by_type(flat):
    """The flat buffers of a clip case under the names of their types."""
    return {k: flat[t] for k, t in _TYPES.items() if t in flat}


def _flat(case, tensors):
    """A clip case's tensors one after the other, a buffer for each type."""
    out = {}
    for (_, k), t in zip(_tensors(case), tensors):
        out.setdefault(k, []).append(t)
    return {k: torch.cat(v) for k, v in out.items()}


def _run_plain(state):
    case, d = state["case"], state["in"]
    op = case["op"]
    if op == "norm_fwd":
        x = d["x"].float()
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = torch.rsqrt((x * x).mean(1) + 1e-5)
        y = x * rstd[:, None] * d["w"].float() + d["b"].float()
        return {"y": y.to(d["x"].dtype), "mean": mean, "rstd": rstd}
    if op == "norm_bwd":
        xhat = (d["x"].float() - d["mean"][:, None]) * d["rstd"][:, None]
        dy = d["dy"].float()
        dw, db = (dy * xhat).sum(0), dy.sum(0)
        g = dy * d["w"].float()
        m1, m2 = g.mean(1), (g * xhat).mean(1)
        dx = (g - m1[:, None] - xhat * m2[:, None]) * d["rstd"][:, None]
        return {"dx": dx.to(d["x"].dtype), "dw": dw.to(d["w"].dtype), "db": db.to(d["w"].dtype)}
    if op == "clip":
        total = sum((t.float() ** 2).sum() for t in d["grads"])
        norm = torch.sqrt(total).reshape(1)
        factor = torch.where(norm > case["max_norm"], case["max_norm"] / norm,
                             torch.ones_like(norm))
        clipped = [(t.float() * factor).to(t.dtype) for t in d["grads"]]
        return {"norm": norm, **_flat(case, clipped)}
    t = d["targets"]
    given = t >= 0
    at = t.clamp(min=0)[:, None]
    if op == "logprob_fwd":
        z = d["logits"].float()
        peak = z.max(1)[0]
        s = (z - peak[:, None]) * case["scale"]
        e = torch.exp(s)
        total = e.sum(1)
        lse = peak * case["scale"] + torch.log(total)
        logp = torch.where(given, s.gather(1, at)[:, 0] - torch.log(total), torch.zeros_like(lse))
        weighted = torch.where(e > 0, e * s, torch.zeros_like(s)).sum(1)
        out = {"logp": logp, "lse": lse, "entropy": torch.log(total) - weighted / total,
               "stats": torch.stack([peak, torch.log(total)], 1)}
        if case["top"]:
            # Ties go to the lowest index (+ 0.0: the two zeros are equal).
            index = torch.sort(z + 0.0, dim=1, descending=True, stable=True)[1][:, :case["top"]]
            out["top_logp"] = s.gather(1, index) - torch.log(total)[:, None]
            out["top_index"] = index
        return out
    s = (d["logits"].float() - d["stats"][:, :1]) * case["scale"] - d["stats"][:, 1:]
    p = torch.exp(s)
    dlogp = torch.where(given, d["dlogp"], torch.zeros_like(d["dlogp"]))
    dz = -p * dlogp[:, None]
    dz.scatter_add_(1, at, dlogp[:, None])
    if case["entropy"]:
        dz -= torch.where(p > 0, p * (s + d["entropy"][:, None]), torch.zeros_like(p)) * (
            d["dentropy"][:, None])
    return {"dlogits": (dz * case["scale"]).to(d["logits"].dtype)}


# ------------------------------------------------------------------ exact
def exact(case, seed):
    """The outputs from their definitions in 64 bits, a block of rows at a time."""
    d = _inputs(case, seed)
    op = case["op"]
    if op == "clip":
        norm = math.sqrt(math.fsum(float(torch.dot(t.double(), t.double())) for t in d["grads"]))
        factor = min(1.0, case["max_norm"] / norm) if norm > 0 else 1.0
        return {"norm": torch.tensor([norm], dtype=torch.float64, device="cuda"),
                **_flat(case, [t.double() * factor for t in d["grads"]])}
    rows = case["rows"]
    step = max(1, (1 << 25) // (case["cols"] if op.startswith("norm") else case["vocab"]))
    parts = [_exact_rows(case, d, slice(i, min(rows, i + step))) for i in range(0, rows, step)]
    out = {}
    for k in parts[0]:
        if k in ("dw", "db"):
            out[k] = torch.stack([p[k] for p in parts]).sum(0)
        else:
            out[k] = torch.cat([p[k] for p in parts])
    return out


def _exact_rows(case, d, r):
    op = case["op"]
    if op == "norm_fwd":
        x, w, b = d["x"][r].double(), d["w"].double(), d["b"].double()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + 1e-5)
        return {"y": torch.addcmul(b, (x - mean[:, None]) * rstd[:, None], w), "mean": mean,
                "rstd": rstd}
    if op == "norm_bwd":
        # The Jacobian of a row: dx = rstd (g - P g), P the projection on the
        # rows' ones and normalised features.
        x, dy, w = d["x"][r].double(), d["dy"][r].double(), d["w"].double()
        rstd = d["rstd"][r].double()[:, None]
        unit = (x - d["mean"][r].double()[:, None]) * rstd
        g = dy * w
        n = case["cols"]
        dx = rstd * (g - g.sum(1, keepdim=True) / n
                     - unit * ((unit * g).sum(1, keepdim=True) / n))
        return {"dx": dx, "dw": (unit * dy).sum(0), "db": dy.sum(0)}
    z = d["logits"][r].double() * case["scale"]
    t = d["targets"][r]
    one = torch.zeros_like(z)
    has = torch.nonzero(t >= 0)[:, 0]
    one[has, t[has]] = 1.0
    lp = torch.log_softmax(z, 1)
    p = lp.exp()
    plogp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    if op == "logprob_fwd":
        out = {"logp": torch.where(one > 0, lp, torch.zeros_like(lp)).sum(1),
               "lse": torch.logsumexp(z, 1), "entropy": -plogp.sum(1)}
        peak = d["logits"][r].max(1)[0].double()
        out["stats"] = torch.stack([peak, out["lse"] - peak * case["scale"]], 1)
        if case["top"]:
            order = torch.sort(d["logits"][r].double() + 0.0, dim=1, descending=True, stable=True)
            index = order.indices[:, :case["top"]]
            out["top_logp"] = lp.gather(1, index)
            out["top_index"] = index
        return out
    dz = d["dlogp"][r].double()[:, None] * (one - p * (t >= 0)[:, None])
    if case["entropy"]:
        dz += d["dentropy"][r].double()[:, None] * (p * plogp.sum(1, keepdim=True) - plogp)
    return {"dlogits": dz * case["scale"]}
