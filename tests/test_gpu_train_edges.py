"""The training step's operators on the GPU where rows and lists are unlike any
that training data makes: masks beyond 32 bits, equal elements, factors below
32 bits, tensors that nobody else holds.  Plain 64-bit forms from train_ref.py."""
import math

import pytest
import torch

import train_ref as ref
from train_ref import INF, U, assert_close, half_ulp

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAN = math.nan


def randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


# ---------------------------------------------------------------- layer norm
# Groups inside a wave, waves, workgroups, single elements beside packs, rows too
# long for held weights, pieces; each with few rows and with many.
EQUAL_COLS = [1, 3, 7, 20, 69, 197, 513, 700, 1025, 2049, 3080, 5000, 8193, 16385, 20011, 40001,
              100352]


@pytest.mark.parametrize("xt", [F32, BF16, F16])
@pytest.mark.parametrize("cols", EQUAL_COLS)
@pytest.mark.parametrize("rows", [5, 2100])
def test_layernorm_of_equal_elements(rows, cols, xt):
    """A row of one number has that number as its mean, no variance, and b as its
    result, whatever a sum of its elements rounds to; with eps = 0 it has no norm."""
    import paper_1903_06934_amd as m
    if rows * cols > 1 << 24:
        rows = 90
    values = torch.tensor([0.1, 1.7, -2.3e-4, 1.0e4, 2.5] + ([] if xt == F16 else [-3.3e7, 1e30]))
    x = values.to(xt)[torch.arange(rows) % len(values)][:, None].repeat(1, cols)
    w, b = randn(1, cols), randn(2, cols)
    y, mean, rstd = m.layernorm_fwd(x.cuda(), w.cuda(), b.cuda(), 1e-5)
    assert torch.equal(mean.cpu(), x[:, 0].float())
    want = torch.full((rows,), 1 / math.sqrt(float(torch.tensor(1e-5))), dtype=torch.float64)
    assert_close(rstd, want, 4 * U * want, "rstd")
    assert torch.equal(y.cpu(), b.to(xt).expand(rows, cols))
    y, mean, rstd = m.layernorm_fwd(x.cuda(), w.cuda(), b.cuda(), 0.0)
    assert torch.equal(mean.cpu(), x[:, 0].float())
    assert (rstd == INF).all() and torch.isnan(y).all()


@pytest.mark.parametrize("cols", [2, 9, 64, 197, 513, 1025, 3080, 16384])
@pytest.mark.parametrize("rows", [5, 2100])
def test_layernorm_of_neighbouring_numbers(rows, cols):
    """Elements that differ in their last places: the differences from the mean are
    whole numbers of these places, so the variance keeps its accuracy, and y is off
    by the rounding of the mean (u |mean| rstd) beside its own few."""
    import paper_1903_06934_amd as m
    if rows * cols > 1 << 24:
        rows = 90
    k = torch.randint(0, 4, (rows, cols), generator=torch.Generator().manual_seed(cols))
    k[:, 0], k[:, 1] = 0, 1  # no row of equal elements
    x = 8200.0 + k * 2.0 ** -10
    assert torch.equal(x.double(), 8200.0 + k.double() * 2.0 ** -10)
    y, mean, rstd = m.layernorm_fwd(x.cuda(), eps=1e-9)
    d = x.double()
    rmean = d.mean(1)
    rrstd = 1 / torch.sqrt(((d - rmean[:, None]) ** 2).mean(1) + float(torch.tensor(1e-9)))
    assert_close(mean, rmean, 1.01 * U * rmean.abs() + U * U, "mean")
    # Sums of small whole numbers; a thread's and the tree's roundings.
    assert_close(rstd, rrstd, 64 * U * rrstd, "rstd")
    ry = (d - rmean[:, None]) * rrstd[:, None]
    assert_close(y, ry, (1.05 * U * rmean.abs() * rrstd)[:, None] + 70 * U * ry.abs(), "y")


@pytest.mark.parametrize("cols", [20, 700, 40001])
@pytest.mark.parametrize("bad", [INF, -INF, NAN])
def test_layernorm_mean_of_infinite_rows(cols, bad):
    """An infinity among a row's elements is its mean; the row has no norm."""
    import paper_1903_06934_amd as m
    x = randn(3, 4, cols)
    x[1, cols - 1] = x[2, 0] = bad
    y, mean, rstd = (t.cpu() for t in m.layernorm_fwd(x.cuda()))
    for r in (1, 2):
        assert torch.isnan(y[r]).all() and torch.isnan(rstd[r])
        assert torch.isnan(mean[r]) if bad != bad else mean[r] == bad
    for r in (0, 3):
        assert torch.isfinite(y[r]).all()


@pytest.mark.parametrize("rows,cols,xt", [(0, 64, F32), (0, 20000, BF16), (1, 100352, F32),
                                          (32, 40001, BF16), (64, 9000, F32), (65, 9000, F32),
                                          (3, 700, F32), (600, 700, BF16)])
def test_layernorm_bwd_stays_inside_its_workspace(rows, cols, xt):
    """A workspace of the size asked for, between elements that stay as they are."""
    import paper_1903_06934_amd as m
    x, dy, w = (t.to(xt).cuda() for t in (randn(1, rows, cols), randn(2, rows, cols),
                                          randn(3, cols)))
    _, mean, rstd = m.layernorm_fwd(x, w)
    want = m.layernorm_bwd(dy, x, mean, rstd, w)
    need = m.layernorm_workspace(True, x)
    n = 0 if need is None else need.numel()
    room = torch.full((512 + n + 4096,), 77, dtype=torch.uint8, device="cuda")
    got = m.layernorm_bwd(dy, x, mean, rstd, w, ws=room[512:512 + n] if n else None)
    for p, q in zip(got, want):
        assert torch.equal(p, q)
    assert (room[:512] == 77).all() and (room[512 + n:] == 77).all()
    if not rows:
        assert n == 0 and (got[1] == 0).all() and (got[2] == 0).all()


# --------------------------------------------------------- log probabilities
# A wave a row, a workgroup of 256 or 1024 threads, pieces and their join.
@pytest.mark.parametrize("rows,vocab", [(600, 5), (600, 300), (8, 3000), (600, 9001), (100, 50001),
                                        (6, 70000)])
@pytest.mark.parametrize("xt", [F32, BF16])
@pytest.mark.parametrize("scale", [1.25, 2.0, 1e6])
def test_logprob_of_a_lowest_value_mask_beyond_32_bits(rows, vocab, xt, scale):
    """Rows masked with the type's lowest value, which times the scale is beyond 32
    bits: equally likely tokens all the same, not banned ones."""
    import paper_1903_06934_amd as m
    z = torch.full((6, vocab), float(torch.finfo(xt).min), dtype=xt)
    z[1, ::2] = -INF                                    # some banned as well
    z[2] = -INF                                         # all banned
    z[3] = (3 * randn(1, vocab)).to(xt)
    z[4, vocab // 2] = 0.0                              # one token left
    z[5, 1:] = -INF                                     # one masked, the others banned
    t = torch.tensor([1, 1, 0, vocab - 1, vocab // 2, 0])
    top = min(vocab, 20)
    out = m.logprob_fwd(z.repeat(rows // 6, 1).cuda(), t.repeat(rows // 6).cuda(), top=top,
                        scale=scale)
    want = ref.logprob_fwd(z, t, top, scale)
    base = 64 * U * (2 + math.log(vocab)) + vocab / 2048 * U
    last = slice((rows // 6 - 1) * 6, rows // 6 * 6)
    for name in ("lse", "logp", "entropy", "top_logp"):
        # What lies beyond 32 bits is infinite in the result.
        w = want[name].float().double()
        size = w.abs().nan_to_num(0, 0, 0)
        bound = base * (2 + math.log(vocab)) + 4 * U * size
        for got in (getattr(out, name)[:6], getattr(out, name)[last]):
            assert_close(got, w, bound, name)
    assert torch.equal(out.top_index[:6].cpu(), want["top_index"])
    assert_close(out.stats[:6], want["stats"], base + 4 * U * want["stats"].abs().nan_to_num(0, 0, 0),
                 "stats")
    dl = randn(2, 6)
    dz = m.logprob_bwd(z.cuda(), out.stats[:6], t.cuda(), dl.cuda(), scale=scale)
    rz, size = ref.logprob_bwd(z, t, scale, out.stats[:6].cpu(), dl)
    assert_close(dz, rz, 8 * U * size + half_ulp(rz, xt) * 1.01 + 1e-37, "dlogits")


@pytest.mark.parametrize("rows,vocab", [(600, 70), (8, 3000), (600, 9001), (2, 70000)])
@pytest.mark.parametrize("scale", [1e-6, 0.25])
def test_logprob_of_logits_further_apart_than_32_bits(rows, vocab, scale):
    """The difference of two logits may be beyond 32 bits where its scaled one, the
    log probability, is not."""
    import paper_1903_06934_amd as m
    big = 3e38
    z = torch.full((2, vocab), -big)
    z[0, 7] = z[1, 3] = big
    z[1, 4], z[1, 5] = 0.0, -INF
    t = torch.tensor([0, 2])
    top = 9
    out = m.logprob_fwd(z.repeat(rows // 2, 1).cuda(), t.repeat(rows // 2).cuda(), top=top,
                        scale=scale)
    want = ref.logprob_fwd(z, t, top, scale)
    for name in ("lse", "logp", "entropy", "top_logp"):
        w = want[name].repeat(rows // 2, *[1] * (want[name].dim() - 1))
        assert_close(getattr(out, name), w, 4 * U * w.abs().nan_to_num(0, 0, 0) + 64 * U, name)
    assert torch.equal(out.top_index.cpu(), want["top_index"].repeat(rows // 2, 1))


@pytest.mark.parametrize("rows", [6, 1200])
@pytest.mark.parametrize("vocab,left,top", [(9, 1, 9), (70, 3, 64), (500, 10, 64), (1100, 5, 40)])
@pytest.mark.parametrize("xt", [F32, BF16])
def test_top_of_rows_that_ban_nearly_all(rows, vocab, left, top, xt):
    """Fewer tokens left than are asked for, in rows that leave threads without an
    element: the banned ones follow in the order of their indices."""
    import paper_1903_06934_amd as m
    z = torch.full((6, vocab), -INF)
    for r in range(6):
        z[r, torch.randperm(vocab, generator=torch.Generator().manual_seed(r))[:left * r // 2]] = r
    z = z.to(xt)
    out = m.logprob_fwd(z.repeat(rows // 6, 1).cuda(), top=top)
    want = ref.logprob_fwd(z, None, top)
    assert torch.equal(out.top_index.cpu(), want["top_index"].repeat(rows // 6, 1))
    logp = want["top_logp"].repeat(rows // 6, 1)
    assert_close(out.top_logp, logp, 64 * U * (2 + math.log(vocab)), "top_logp")


# ------------------------------------------------------------------ clipping
@pytest.mark.parametrize("sizes", [[1], [300] * 3, [1000] * 150, [3, 70000, 2048, 1] * 5])
@pytest.mark.parametrize("iterable", [tuple, iter, lambda ts: (t * 2 for t in ts)],
                         ids=["tuple", "iterator", "temporaries"])
def test_gradients_from_any_iterable(sizes, iterable):
    """Gradients that only the call holds stay whole until it has read them, though
    norm and workspace are allocated after them."""
    import paper_1903_06934_amd as m
    dev = [randn(i, n).cuda() for i, n in enumerate(sizes)]
    given = [t.cpu() for t in iterable(dev)]
    norm, want = ref.clip(given, 0.25)
    for _ in range(3):
        assert_close(m.grad_norm(iterable(dev)), torch.tensor([norm]), 2 * U * norm, "norm")
        assert m.grad_workspace(iterable(dev)).numel() == m.grad_workspace(dev).numel()
        out = [torch.full_like(t, NAN) for t in dev]
        got = m.grad_clip(iterable(dev), 0.25, out=iter(out))
        assert_close(got, torch.tensor([norm]), 2 * U * norm, "norm")
        for o, w in zip(out, want):
            assert_close(o, w, 4 * U * w.abs() + half_ulp(w, F32) * 1.01, "clipped")


def test_lists_that_are_none():
    import paper_1903_06934_amd as m
    for bad in (3, None):
        with pytest.raises(TypeError):
            m.grad_norm(bad)

    def broken():
        yield torch.ones(3, device="cuda")
        raise KeyError("from the generator")

    with pytest.raises(KeyError):
        m.grad_norm(broken())


@pytest.mark.parametrize("max_norm", [1e-5, 1e-9, 3e-12, 1e-20, 1e-38])
@pytest.mark.parametrize("count", [1, 5, 200])
def test_clip_by_factors_below_32_bits(max_norm, count):
    """max_norm / norm below 32 bits' smallest numbers: the clipped gradients have
    their own size's accuracy all the same, in place and beside."""
    import paper_1903_06934_amd as m
    grads = [randn(i, 700 + i) * 2e30 for i in range(count)]
    grads.append((randn(9, 333) * 1e30).to(BF16))
    norm, want = ref.clip(grads, max_norm)
    dev = [t.cuda() for t in grads]
    out = [torch.full_like(t, NAN) for t in dev]
    got = m.grad_clip(dev, max_norm, out=out)
    assert_close(got, torch.tensor([norm]), 2 * U * norm, "norm")
    m.grad_clip(dev, max_norm)
    for o, i, w in zip(out, dev, want):
        # The factor, the product and a shift, which rounds below the normal numbers.
        assert_close(o, w, 4 * U * w.abs() + 2.0 ** -149 + half_ulp(w, o.dtype) * 1.01, "clipped")
        assert torch.equal(o, i)


# ------------------------------------------------------------ results in place
def test_results_in_given_tensors_are_seen_by_autograd():
    """A tensor that torch has saved for a backward pass and that a call overwrites
    afterwards is reported, not used."""
    import paper_1903_06934_amd as m
    x, w = randn(1, 6, 50).cuda(), torch.ones(50, device="cuda")
    t, dl = torch.arange(6, device="cuda"), torch.ones(6, device="cuda")
    y, mean, rstd = m.layernorm_fwd(x, w, w)
    stats = m.logprob_fwd(x, t).stats
    new = lambda *s: torch.zeros(s, device="cuda")

    def layernorm(a, b, c):
        m.layernorm_fwd(x, w, w, y=a, mean=b, rstd=c)

    def layernorm_back(a, b, c):
        m.layernorm_bwd(x, x, mean, rstd, w, dx=a, dw=b, db=c)

    cases = [(layernorm, [new(6, 50), new(6), new(6)]),
             (layernorm_back, [new(6, 50), new(50), new(50)]),
             (lambda a: m.logprob_bwd(a, stats, t, dl, dlogits=a), [x.clone()]),
             (lambda a: m.logprob_bwd(x, stats, t, dl, dlogits=a), [new(6, 50)]),
             (lambda a, b: m.grad_clip([a, b], 1.0), [x.clone(), w.clone()]),
             (lambda a, b, n: m.grad_clip([x, w], 1.0, out=[a, b], norm=n),
              [new(6, 50), new(50), new(1)]),
             (lambda n: m.grad_norm([x, w], norm=n), [new(1)])]
    for call, given in cases:
        v = torch.ones(1, device="cuda", requires_grad=True)
        saved = [(g * v).sum() for g in given]  # each product saves its tensor
        before = [g._version for g in given]
        call(*given)
        for g, b, s in zip(given, before, saved):
            assert g._version > b
            with pytest.raises(RuntimeError, match="inplace"):
                s.backward()
    # What is only read keeps its version; tensors of inference mode have none.
    before = x._version
    m.layernorm_fwd(x, w, w)
    m.grad_norm([x, w])
    m.grad_clip([x, w], 1.0, out=[new(6, 50), new(50)])
    assert x._version == before
    with torch.inference_mode():
        z = x.clone()
        m.grad_clip([z], 1.0)
        m.layernorm_fwd(x, w, w, y=z)
    m.layernorm_fwd(x, w, w, y=z)


@pytest.mark.parametrize("shape", [(6, 50), (2, 3, 9000), (1, 70001), (500,)])
@pytest.mark.parametrize("given", ["logp", "lse", "entropy", "stats", "top_logp", "top_index",
                                   "all"])
def test_logprob_into_given_tensors(shape, given):
    """Any of the results, or all, in the caller's tensors; the others are new."""
    import paper_1903_06934_amd as m
    z = randn(4, *shape).cuda()
    t = torch.zeros(shape[:-1], dtype=torch.int64, device="cuda")
    want = m.logprob_fwd(z, t, top=4, scale=0.7)
    mine = {k: torch.full_like(v, 77) for k, v in want._asdict().items() if given in (k, "all")}
    version = {k: v._version for k, v in mine.items()}
    got = m.logprob_fwd(z, t, top=4, scale=0.7, **mine)
    for k, v in want._asdict().items():
        assert torch.equal(getattr(got, k), v), k
    for k, v in mine.items():
        assert getattr(got, k).data_ptr() == v.data_ptr() and v._version > version[k]
        assert torch.equal(v, getattr(want, k))


def test_logprob_refuses_given_tensors():
    import paper_1903_06934_amd as m
    z, t = randn(5, 6, 50).cuda(), torch.arange(6, device="cuda")
    new = lambda *s: torch.zeros(s, device="cuda")
    for bad in ({"lse": new(5)}, {"lse": new(6).double()}, {"entropy": new(6).cpu()},
                {"stats": new(6)}, {"stats": new(2, 6).t()}, {"top_logp": new(6, 2)},
                {"top_index": new(6, 3)}, {"logp": new(12)[::2]}):
        with pytest.raises(ValueError):
            m.logprob_fwd(z, t, top=3, **bad)
    with pytest.raises(ValueError):
        m.logprob_fwd(z, t, top_logp=new(6, 3))  # without a top
    both = new(6)
    for bad in ({"lse": both, "entropy": both}, {"lse": z[0, :6]}):
        with pytest.raises(m.MiconvError):
            m.logprob_fwd(z, t, top=3, **bad)
    with pytest.raises(m.MiconvError):
        m.logprob_fwd(z, logp=new(6))  # of no targets
    assert m.logprob_fwd(z, ws=None).logp is None
