"""The training step's operators on the GPU against their plain 64-bit forms
(train_ref.py), over types, row lengths on both sides of every launch rule,
strides, alignments and special rows.

Bounds, with u = 2^-24: a sum of n terms in 32 bits that a thread adds one by
one over m of them and a tree over the rest is off by at most (m + log n) u times
the sum of the terms' magnitudes; each result adds the roundings of its few
operations, and half a unit in its type's last place.  Where a test multiplies u
by a constant, that constant is this count, rounded up."""
import math

import pytest
import torch

import train_ref as ref
from train_ref import INF, U, assert_close, half_ulp

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAN = math.nan


def gen(*seed):
    s = 17
    for v in seed:
        s = (s * 1000003 + int(v)) % (1 << 62)
    return torch.Generator().manual_seed(s)


def randn(g, *shape):
    return torch.randn(shape, generator=g)


def strided(t, gap, shift=0):
    """A device copy of t [rows, cols] inside a wider matrix of NaN: gap elements
    between rows, the first row shift elements into it."""
    rows, cols = t.shape
    wide = torch.full((rows * (cols + gap) + shift,), NAN, dtype=t.dtype, device="cuda")
    v = wide[shift:shift + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]
    v.copy_(t)
    return v, wide


def untouched(view, wide):
    """The elements of wide outside the view are the NaN that they were."""
    keep = wide.clone()
    inner = keep.as_strided(view.shape, view.stride(), view.storage_offset())
    inner.fill_(NAN)
    assert torch.isnan(keep).all()


# ---------------------------------------------------------------- layer norm
# Sub-wave groups, one wave, several waves, a workgroup's limit, pieces.
COLS = [1, 2, 7, 8, 24, 64, 100, 197, 255, 512, 513, 1000, 2048, 4096, 5000, 16384, 16385, 20011,
        32768, 32769, 100352]


def rows_for(cols):
    return 37 if cols <= 5000 else 5


def norm_terms(cols):
    """Terms a thread adds one by one, and the tree's steps, at most."""
    return 48 + cols // 1024


@pytest.mark.parametrize("xt,wt", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("cols", COLS)
def test_layernorm(cols, xt, wt):
    import paper_1903_06934_amd as m
    rows = rows_for(cols)
    g = gen(cols, rows)
    x = (randn(g, rows, cols) * (0.5 + torch.rand(cols, generator=g)) + randn(g, rows, 1)).to(xt)
    w, b = (1 + 0.3 * randn(g, cols)).to(wt), randn(g, cols).to(wt)
    dy = randn(g, rows, cols).to(xt)
    gap, shift = (0, 0) if cols % 3 else (5, 3)
    xv, _ = strided(x, gap, shift)
    yv, wide = strided(torch.zeros(rows, cols, dtype=xt), gap + 1, shift)
    y, mean, rstd = m.layernorm_fwd(xv, w.cuda(), b.cuda(), 1e-5, y=yv)
    ry, rmean, rrstd, size, msize = ref.layernorm_fwd(x, w, b)
    k = norm_terms(cols) * U
    assert_close(mean, rmean, k * msize, "mean")
    # rstd's error: of the variance's terms, and of the mean's error squared.
    assert_close(rstd, rrstd, rrstd * (k + (k * msize * rrstd) ** 2), "rstd")
    assert_close(y, ry, 2 * k * size + half_ulp(ry, xt) * 1.01, "y")
    untouched(yv, wide)

    dyv, _ = strided(dy, gap, shift)
    dxv, wide = strided(torch.zeros(rows, cols, dtype=xt), gap + 2, shift)
    dx, dw, db = m.layernorm_bwd(dyv, xv, mean, rstd, w.cuda(), dx=dxv)
    want = ref.layernorm_bwd(dy, x, mean.cpu(), rstd.cpu(), w)
    assert_close(dx, want[0][0], k * want[0][1] + half_ulp(want[0][0], xt) * 1.01, "dx")
    for got, (val, mag), name in ((dw, want[1], "dw"), (db, want[2], "db")):
        assert got.dtype == wt
        assert_close(got, val, 64 * U * mag + half_ulp(val, wt) * 1.01, name)
    untouched(dxv, wide)
    # Bit for bit the same again, and in parts.
    again = m.layernorm_bwd(dyv, xv, mean, rstd, w.cuda())
    for p, q in zip(again, (dx, dw, db)):
        assert torch.equal(p, q)
    only = m.layernorm_bwd(dyv, xv, mean, rstd, w.cuda(), with_input=False, with_bias=False)
    assert only[0] is None and only[2] is None and torch.equal(only[1], dw)
    only = m.layernorm_bwd(dyv, xv, mean, rstd, w.cuda(), with_weight=False, with_bias=False)
    assert only[1] is None and torch.equal(only[0], dx)


@pytest.mark.parametrize("xt", [F32, BF16])
@pytest.mark.parametrize("rows", [9, 130, 1030])
def test_layernorm_row_lengths(rows, xt):
    """Many row lengths: every share of a row among threads and packs."""
    import paper_1903_06934_amd as m
    g = gen(rows, 9)
    lengths = torch.randint(1, 9000, (24,), generator=g).tolist() + [4500, 6500, 8192, 8193]
    for cols in lengths if rows < 1000 else lengths[:4] + [5000, 3000, 1700]:
        x, dy = randn(g, rows, cols).to(xt), randn(g, rows, cols).to(xt)
        w = randn(g, cols).to(xt)
        y, mean, rstd = m.layernorm_fwd(x.cuda(), w.cuda())
        ry, rmean, rrstd, size, msize = ref.layernorm_fwd(x, w)
        k = norm_terms(cols) * U
        assert_close(mean, rmean, k * msize, f"mean {cols}")
        assert_close(y, ry, 2 * k * size + half_ulp(ry, xt) * 1.01, f"y {cols}")
        dx, dw, db = m.layernorm_bwd(dy.cuda(), x.cuda(), mean, rstd, w.cuda())
        want = ref.layernorm_bwd(dy, x, mean.cpu(), rstd.cpu(), w)
        assert_close(dx, want[0][0], k * want[0][1] + half_ulp(want[0][0], xt) * 1.01,
                     f"dx {cols}")
        for got, (val, mag), name in ((dw, want[1], "dw"), (db, want[2], "db")):
            assert_close(got, val, 300 * U * mag + half_ulp(val, xt) * 1.01, f"{name} {cols}")


@pytest.mark.parametrize("xt,wt", [(F32, F32), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("base", [40, 1200, 4352, 9000, 20000, 40000])
def test_layernorm_short_vectors(base, xt, wt):
    """Every number of elements that the row's end leaves of a vector, in every form."""
    import paper_1903_06934_amd as m
    rows = 90 if base > 16384 else 37
    for cols in range(base, base + 8):
        g = gen(cols, 37)
        x, dy = randn(g, rows, cols).to(xt), randn(g, rows, cols).to(xt)
        w, b = randn(g, cols).to(wt), randn(g, cols).to(wt)
        yv, wide = strided(torch.zeros(rows, cols, dtype=xt), 3, 1)
        y, mean, rstd = m.layernorm_fwd(x.cuda(), w.cuda(), b.cuda(), y=yv)
        ry, rmean, rrstd, size, msize = ref.layernorm_fwd(x, w, b)
        k = norm_terms(cols) * U
        assert_close(rstd, rrstd, rrstd * (k + (k * msize * rrstd) ** 2), f"rstd {cols}")
        assert_close(y, ry, 2 * k * size + half_ulp(ry, xt) * 1.01, f"y {cols}")
        untouched(yv, wide)
        dxv, wide = strided(torch.zeros(rows, cols, dtype=xt), 1, 1)
        dx, dw, db = m.layernorm_bwd(dy.cuda(), x.cuda(), mean, rstd, w.cuda(), dx=dxv)
        want = ref.layernorm_bwd(dy, x, mean.cpu(), rstd.cpu(), w)
        assert_close(dx, want[0][0], k * want[0][1] + half_ulp(want[0][0], xt) * 1.01,
                     f"dx {cols}")
        untouched(dxv, wide)
        for got, (val, mag), name in ((dw, want[1], "dw"), (db, want[2], "db")):
            assert_close(got, val, 300 * U * mag + half_ulp(val, wt) * 1.01, f"{name} {cols}")


@pytest.mark.parametrize("xt", [F32, BF16, F16])
@pytest.mark.parametrize("cols", [5, 9, 10, 33, 69, 80, 81, 130, 140, 144, 145, 256, 257, 288,
                                  320, 321, 513, 576, 769, 1025, 1088, 1089, 2049, 2176, 3080,
                                  4100])
def test_layernorm_row_tails(cols, xt):
    """Many rows some elements longer than whole vectors of a wave or some waves:
    the elements beside them, and what lies beside the rows."""
    import paper_1903_06934_amd as m
    rows = 2100
    g = gen(cols, 31)
    x, dy = randn(g, rows, cols).to(xt), randn(g, rows, cols).to(xt)
    w, b = randn(g, cols), randn(g, cols)
    xv, _ = strided(x, 3, 1)
    dyv, _ = strided(dy, 0, 1)
    yv, wide = strided(torch.zeros(rows, cols, dtype=xt), 1, 2)
    y, mean, rstd = m.layernorm_fwd(xv, w.cuda(), b.cuda(), y=yv)
    ry, rmean, rrstd, size, msize = ref.layernorm_fwd(x, w, b)
    k = norm_terms(cols) * U
    assert_close(mean, rmean, k * msize, "mean")
    assert_close(rstd, rrstd, rrstd * (k + (k * msize * rrstd) ** 2), "rstd")
    assert_close(y, ry, 2 * k * size + half_ulp(ry, xt) * 1.01, "y")
    untouched(yv, wide)
    dxv, wide = strided(torch.zeros(rows, cols, dtype=xt), 2, 1)
    dx, dw, db = m.layernorm_bwd(dyv, xv, mean, rstd, w.cuda(), dx=dxv)
    want = ref.layernorm_bwd(dy, x, mean.cpu(), rstd.cpu(), w)
    assert_close(dx, want[0][0], k * want[0][1] + half_ulp(want[0][0], xt) * 1.01, "dx")
    untouched(dxv, wide)
    for got, (val, mag), name in ((dw, want[1], "dw"), (db, want[2], "db")):
        assert_close(got, val, (300 + rows / 256) * U * mag, name)


@pytest.mark.parametrize("rows", [0, 1, 2, 255, 4097])
@pytest.mark.parametrize("cols,xt", [(48, BF16), (513, F32), (3000, BF16), (40000, F32)])
def test_layernorm_rows(rows, cols, xt):
    """One row, odd numbers of rows, none; no weight or bias."""
    import paper_1903_06934_amd as m
    if rows * cols > 1 << 24:
        rows = 300
    g = gen(rows, cols, 3)
    x, dy = randn(g, rows, cols).to(xt), randn(g, rows, cols).to(xt)
    y, mean, rstd = m.layernorm_fwd(x.cuda())
    ry, rmean, rrstd, size, msize = ref.layernorm_fwd(x)
    k = norm_terms(cols) * U
    assert_close(mean, rmean, k * msize, "mean")
    assert_close(y, ry, 2 * k * size + half_ulp(ry, xt) * 1.01, "y")
    dx, dw, db = m.layernorm_bwd(dy.cuda(), x.cuda(), mean, rstd)
    want = ref.layernorm_bwd(dy, x, mean.cpu(), rstd.cpu())
    assert_close(dx, want[0][0], k * want[0][1] + half_ulp(want[0][0], xt) * 1.01, "dx")
    # Rows are added in runs of at most rows / 256, their sums by 256 and less.
    for got, (val, mag), name in ((dw, want[1], "dw"), (db, want[2], "db")):
        assert got.dtype == F32
        assert_close(got, val, (300 + rows / 256) * U * mag, name)


def test_layernorm_far_from_zero():
    """Rows whose mean is 1000 times their spread: the variance is taken about it."""
    import paper_1903_06934_amd as m
    for cols in (64, 2000, 50000):
        x = 1000 + randn(gen(cols, 5), 6, cols)
        y, _, rstd = m.layernorm_fwd(x.cuda())
        ry, _, rrstd, size, msize = ref.layernorm_fwd(x)
        k = norm_terms(cols) * U
        assert_close(rstd, rrstd, rrstd * (k + (k * msize * rrstd) ** 2), f"rstd {cols}")
        assert_close(y, ry, 2 * k * size, f"y {cols}")


@pytest.mark.parametrize("cols", [20, 700, 40000])
def test_layernorm_special_rows(cols):
    """A row of equal elements is 0 times w plus b; infinities and NaN stay in their
    rows."""
    import paper_1903_06934_amd as m
    x = randn(gen(cols), 6, cols)
    x[1] = 2.5
    x[3, 7], x[4, cols - 1] = INF, NAN
    y, _, rstd = m.layernorm_fwd(x.cuda())
    y, rstd = y.cpu(), rstd.cpu()
    assert (y[1] == 0).all() and abs(float(rstd[1]) * math.sqrt(1e-5) - 1) < 1e-6
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).all()
    for r in (0, 2, 5):
        assert torch.isfinite(y[r]).all()


@pytest.mark.parametrize("cols", [3, 9, 21])
def test_layernorm_of_large_equal_elements(cols):
    """|mean| rstd beyond 32 bits: the places past the row's end add nothing."""
    import paper_1903_06934_amd as m
    x = torch.full((4, cols), 1e37)
    dy = randn(gen(cols, 8), 4, cols)
    y, mean, rstd = m.layernorm_fwd(x.cuda())
    # Sums of up to 21 equal numbers are off by a few roundings: so is the mean.
    dx = m.layernorm_bwd(dy.cuda(), x.cuda(), x[:, 0].cuda(), torch.full((4,), 300.0).cuda())[0]
    want = 300.0 * (dy - dy.double().mean(1, keepdim=True))
    assert_close(dx, want, 32 * U * 300 * (dy.abs() + 1), "dx")


def test_layernorm_gradient_by_differences():
    """dx, dw and db against differences of the forward pass along random
    directions."""
    import paper_1903_06934_amd as m
    rows, cols = 9, 130
    g = gen(4)
    x, w, b, dy = (randn(g, *s).double() for s in ((rows, cols), (cols,), (cols,), (rows, cols)))
    f32 = [t.float().cuda() for t in (x, w, b, dy)]
    _, mean, rstd = m.layernorm_fwd(*f32[:3])
    dx, dw, db = m.layernorm_bwd(f32[3], f32[0], mean, rstd, f32[1])
    h = 1e-6
    for i, grad in ((0, dx), (1, dw), (2, db)):
        base = [t.float().double() for t in (x, w, b)]
        v = randn(g, *base[i].shape).double()
        up, down = list(base), list(base)
        up[i], down[i] = base[i] + h * v, base[i] - h * v
        diff = ((ref.layernorm_fwd(*up)[0] - ref.layernorm_fwd(*down)[0])
                * dy.float().double()).sum() / (2 * h)
        got = (grad.cpu().double() * v).sum()
        assert abs(float(got - diff)) < 1e-4 * (1 + abs(float(diff)))


# --------------------------------------------------------- log probabilities
VOCABS = [1, 2, 9, 64, 250, 1000, 1001, 8191, 32000, 65537, 131072]


def logits(g, rows, vocab, xt, banned=0.0):
    z = 3 * randn(g, rows, vocab)
    if banned:
        z[torch.rand(rows, vocab, generator=g) < banned] = -INF
    return z.to(xt)


def prob_bounds(want, vocab, scale, z):
    """Errors of lse, log probabilities and entropy: a sum's tree and its terms'
    exponents, whose weighted size is at most 1 + ln vocab."""
    base = 64 * U * (2 + math.log(vocab)) + vocab / 2048 * U
    return (base + 4 * U * want["lse"].abs().nan_to_num(0, 0, 0),
            base + 4 * U * want["logp"].abs().nan_to_num(0, 0, 0),
            base * (2 + math.log(vocab)))


@pytest.mark.parametrize("xt", [F32, BF16, F16])
@pytest.mark.parametrize("vocab", VOCABS)
def test_logprob(vocab, xt):
    import paper_1903_06934_amd as m
    rows = 7 if vocab <= 8191 else 3
    top, scale = min(vocab, 20 if vocab % 2 else 5), 1.0 if vocab % 2 else 0.7
    g = gen(vocab, 1)
    z = logits(g, rows, vocab, xt, 0.1 if vocab > 60 else 0.0)
    t = torch.randint(vocab, (rows,), generator=g)
    t[1] = -1
    zv, _ = strided(z, 3, 1)
    out = m.logprob_fwd(zv, t.cuda(), top=top, scale=scale)
    want = ref.logprob_fwd(z, t, top, scale)
    bl, bp, be = prob_bounds(want, vocab, scale, z)
    assert_close(out.lse, want["lse"], bl, "lse")
    assert_close(out.logp, want["logp"], bp, "logp")
    assert_close(out.entropy, want["entropy"], be, "entropy")
    assert_close(out.stats, want["stats"], torch.stack([0 * bl, bl], 1), "stats")
    assert torch.equal(out.top_index.cpu(), want["top_index"])
    assert_close(out.top_logp, want["top_logp"],
                 bp.max() + 4 * U * want["top_logp"].abs().nan_to_num(0, 0, 0), "top_logp")

    dlogp, dent = randn(g, rows), randn(g, rows)
    for dl, de in ((dlogp, None), (None, dent), (dlogp, dent)):
        dzv, wide = strided(torch.zeros(rows, vocab, dtype=xt), 2, 1)
        dz = m.logprob_bwd(zv, out.stats, None if dl is None else t.cuda(),
                           None if dl is None else dl.cuda(),
                           None if de is None else out.entropy, None if de is None else de.cuda(),
                           scale=scale, dlogits=dzv)
        rz, size = ref.logprob_bwd(z, t, scale, out.stats.cpu(), dl, out.entropy.cpu(), de)
        assert_close(dz, rz, 8 * U * size + half_ulp(rz, xt) * 1.01 + 1e-37, "dlogits")
        untouched(dzv, wide)
    # In place.
    zc = z.cuda()
    m.logprob_bwd(zc, out.stats, t.cuda(), dlogp.cuda(), out.entropy, dent.cuda(), scale=scale,
                  dlogits=zc)
    assert torch.equal(zc, dz)


@pytest.mark.parametrize("rows,vocab", [(0, 10), (1, 10), (300, 10), (2000, 37), (260, 5000),
                                        (1, 200003), (40, 50001), (129, 9000)])
@pytest.mark.parametrize("top", [0, 1, 8])
def test_logprob_rows(rows, vocab, top):
    """Few and many rows, those that are cut into pieces among them."""
    import paper_1903_06934_amd as m
    g = gen(rows, vocab)
    z = logits(g, rows, vocab, BF16)
    t = torch.randint(vocab, (rows,), generator=g)
    some = torch.randperm(rows, generator=g)[:12]
    out = m.logprob_fwd(z.cuda(), t.cuda(), top=top)
    want = ref.logprob_fwd(z[some], t[some], top)
    bl, bp, be = prob_bounds(want, vocab, 1.0, z)
    assert_close(out.lse[some.cuda()], want["lse"], bl, "lse")
    assert_close(out.logp[some.cuda()], want["logp"], bp, "logp")
    assert_close(out.entropy[some.cuda()], want["entropy"], be, "entropy")
    if top:
        assert torch.equal(out.top_index.cpu()[some], want["top_index"])
    dlogp = randn(g, rows)
    dz = m.logprob_bwd(z.cuda(), out.stats, t.cuda(), dlogp.cuda())
    rz, size = ref.logprob_bwd(z[some], t[some], 1.0, out.stats.cpu()[some], dlogp[some])
    assert_close(dz[some.cuda()], rz, 8 * U * size + half_ulp(rz, BF16) * 1.01 + 1e-37, "dlogits")


@pytest.mark.parametrize("vocab", [5, 300, 3000, 70000])
@pytest.mark.parametrize("xt", [F32, BF16])
def test_logprob_special_rows(vocab, xt):
    """Rows that ban all tokens, all but a few, hold the type's lowest value as a
    mask, NaN, infinities, one equal value; tokens not given or past the end."""
    import paper_1903_06934_amd as m
    g = gen(vocab, 2)
    low = float(torch.finfo(xt).min)
    z = logits(g, 10, vocab, xt)
    z[0] = -INF
    z[1] = -INF
    z[1, vocab - 2], z[1, 2] = 0.5, 0.25
    z[2] = low
    z[3, 1:] = low
    z[4, vocab // 2] = NAN
    z[5, vocab - 1] = INF
    z[6] = 1.25
    z[7, ::2] = 0.0
    z[7, 1::2] = -0.0
    z[8] = NAN
    t = torch.tensor([1, 2, 3, 0, 0, 1, 4, 3, 1, vocab])
    top = min(vocab, 9)
    out = m.logprob_fwd(z.cuda(), t.cuda(), top=top)
    want = ref.logprob_fwd(z, t, top)
    bl, bp, be = prob_bounds(want, vocab, 1.0, z)
    assert_close(out.lse, want["lse"], bl, "lse")
    assert_close(out.logp, want["logp"], bp, "logp")
    assert_close(out.entropy, want["entropy"], be, "entropy")
    assert_close(out.stats, want["stats"], torch.stack([0 * bl, bl], 1), "stats")
    assert torch.equal(out.top_index.cpu(), want["top_index"])
    assert_close(out.top_logp, want["top_logp"],
                 bp.max() + 4 * U * want["top_logp"].abs().nan_to_num(0, 0, 0), "top_logp")
    dlogp, dent = randn(g, 10), randn(g, 10)
    dz = m.logprob_bwd(z.cuda(), out.stats, t.cuda(), dlogp.cuda(), out.entropy, dent.cuda())
    rz, size = ref.logprob_bwd(z, t, 1.0, out.stats.cpu(), dlogp, out.entropy.cpu(), dent)
    assert_close(dz, rz, 8 * U * size + half_ulp(rz, xt) * 1.01 + 1e-37, "dlogits")


@pytest.mark.parametrize("vocab", [2000, 40000])
@pytest.mark.parametrize("kind", ["rising", "falling", "few values", "periodic", "one run"])
@pytest.mark.parametrize("rows", [1, 300])
def test_top_of_ordered_rows(vocab, kind, rows):
    """Rows whose large logits come in orders that a selection by threads meets
    worst, with many ties."""
    import paper_1903_06934_amd as m
    j = torch.arange(vocab, dtype=torch.float64)
    z = {"rising": j / vocab, "falling": -j / vocab, "few values": j % 3,
         "periodic": torch.where(j % 2048 < 64, 1 + j / vocab, 0 * j),
         "one run": torch.where((j > 900) & (j < 1400), 2 + 0 * j, 0 * j)}[kind].to(BF16)
    z = z.repeat(rows, 1)
    top = 64
    out = m.logprob_fwd(z.cuda(), top=top)
    assert out.logp is None
    want = ref.logprob_fwd(z[:1], None, top)
    assert torch.equal(out.top_index.cpu(), want["top_index"].expand(rows, top))


@pytest.mark.parametrize("rows", [1, 300])
@pytest.mark.parametrize("wide,levels", [(256, 0), (600, 0), (256, 40), (600, 3), (1500, 2)])
@pytest.mark.parametrize("top", [3, 40])
def test_top_of_many_large_logits_in_few_threads(rows, wide, levels, top):
    """More logits above the rest than are held at once, all different or of a few
    values, where the threads' maxima say little."""
    import paper_1903_06934_amd as m
    j = torch.arange(50000)
    large = 1 + torch.rand(50000, generator=gen(wide), dtype=torch.float64)
    if levels:
        large = torch.round(large * levels) / levels
    z = torch.where(j % 2048 < wide, large, -(j % 7).double()).float().repeat(rows, 1)
    out = m.logprob_fwd(z.cuda(), top=top)
    want = ref.logprob_fwd(z[:1], None, top)
    assert torch.equal(out.top_index.cpu(), want["top_index"].expand(rows, top))


@pytest.mark.parametrize("vocab", [1, 2, 7, 33, 63, 64])
@pytest.mark.parametrize("rows", [1, 700])
def test_top_of_the_whole_row(vocab, rows):
    """top = vocab: every token, in order; logits of fewer dimensions."""
    import paper_1903_06934_amd as m
    z = torch.round(2 * randn(gen(vocab, rows), rows, vocab))
    out = m.logprob_fwd(z.cuda(), top=vocab)
    want = ref.logprob_fwd(z, None, vocab)
    assert torch.equal(out.top_index.cpu(), want["top_index"])
    one = m.logprob_fwd(z[0].cuda(), torch.tensor(0, device="cuda"), top=vocab)
    assert one.lse.shape == () and one.stats.shape == (2,) and one.top_index.shape == (vocab,)
    assert torch.equal(one.top_index, out.top_index[0])
    more = m.logprob_fwd(z.cuda(), top=vocab + 9)  # a row has no more tokens
    assert torch.equal(more.top_index, out.top_index)
    cube = m.logprob_fwd(z.view(rows, 1, vocab).cuda(), top=vocab)
    assert cube.lse.shape == (rows, 1) and cube.top_logp.shape == (rows, 1, vocab)
    assert torch.equal(cube.top_logp[:, 0], out.top_logp)


@pytest.mark.parametrize("inference", [False, True])
def test_results_are_ordinary_tensors(inference):
    """Results that share a buffer: written in place, differentiated, saved apart."""
    import io

    import paper_1903_06934_amd as m
    z = randn(gen(77), 6, 50)
    with torch.inference_mode(inference):
        out = m.logprob_fwd(z.cuda(), torch.arange(6, device="cuda"), top=3)
        again = m.logprob_fwd(z.cuda(), torch.arange(6, device="cuda"), top=3)
        _, mean, rstd = m.layernorm_fwd(z.cuda())
        both = mean.clone(), rstd.clone()
        mean.zero_()
        assert torch.equal(rstd, both[1])
        for i, t in enumerate(out):
            t.fill_(7)
            for j, (u, v) in enumerate(zip(out, again)):
                assert torch.equal(u, v) == (j > i)
    if not inference:
        w = again.logp.requires_grad_()
        (w * w).sum().backward()
        assert torch.allclose(w.grad, 2 * w.detach())
    buf = io.BytesIO()
    torch.save([t.detach() for t in again], buf)
    buf.seek(0)
    for t, s in zip(torch.load(buf, weights_only=True), again):
        assert torch.equal(t, s)


def test_logprob_far_from_zero():
    """Logits around 20000: log probabilities and gradient keep their own size's
    accuracy."""
    import paper_1903_06934_amd as m
    z = 20000 + torch.round(4 * randn(gen(6), 5, 3001))
    t = torch.arange(5)
    out = m.logprob_fwd(z.cuda(), t.cuda())
    want = ref.logprob_fwd(z, t)
    bl, bp, be = prob_bounds(want, 3001, 1.0, z)
    assert_close(out.lse, want["lse"], bl, "lse")
    assert_close(out.logp, want["logp"], bp, "logp")
    assert_close(out.entropy, want["entropy"], be, "entropy")
    dl = randn(gen(7), 5)
    dz = m.logprob_bwd(z.cuda(), out.stats, t.cuda(), dl.cuda())
    rz, size = ref.logprob_bwd(z, t, 1.0, want["stats"], dl)
    assert_close(dz, rz, (8 * U + bl.new_tensor(64 * U * 10)) * size, "dlogits")


def test_logprob_gradient_by_differences():
    import paper_1903_06934_amd as m
    g = gen(12)
    rows, vocab, h = 6, 75, 1e-6
    z, t = logits(g, rows, vocab, F32), torch.randint(vocab, (rows,), generator=g)
    dl, de, v = randn(g, rows), randn(g, rows), randn(g, rows, vocab).double()
    out = m.logprob_fwd(z.cuda(), t.cuda())
    dz = m.logprob_bwd(z.cuda(), out.stats, t.cuda(), dl.cuda(), out.entropy, de.cuda())

    def loss(zz):
        o = ref.logprob_fwd(zz, t)
        return (o["logp"] * dl + o["entropy"] * de).sum()

    diff = (loss(z.double() + h * v) - loss(z.double() - h * v)) / (2 * h)
    assert abs(float((dz.cpu().double() * v).sum() - diff)) < 1e-4 * (1 + abs(float(diff)))


# ------------------------------------------------------------------ clipping
SIZES = [
    [1], [0], [], [16384], [16385, 0, 3], [7] * 300, [1000003, 5, 64, 4096 * 11],
    [33] * 111 + [0] * 5 + [2, 50000], [1 << 22],
    [100] * 112, [100] * 113, [1025 * 16384 + 7, 3], [20000] * 599 + [1], [1] * 4200,
    [5] * 148, [70000, 1] * 148 + [3], [16384, 16385] * 74 + [40000],
    [70000, 3] * 112, [9000] * 225, [40000, 0, 8191, 8193] * 150,
    [4095, 4096, 4097, 8191, 8192, 8193], [4096] * 1030, [8200] * 1030,
]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{sum(s)}")
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16", "mixed"])
def test_clip(sizes, kind):
    import paper_1903_06934_amd as m
    g = gen(len(sizes), sum(sizes))
    types = {"f32": [F32], "bf16": [BF16], "f16": [F16], "mixed": [F32, BF16, F16]}[kind]
    grads = [(0.3 * randn(g, n)).to(types[i % len(types)]) for i, n in enumerate(sizes)]
    dev = [t.cuda() for t in grads]
    true, _ = ref.clip(grads, INF)
    for max_norm in (0.5 * true, 2 * true + 1, 0.0, INF):
        norm, want = ref.clip(grads, max_norm)
        keep = [t.clone() for t in dev]
        out = [torch.full_like(t, NAN) for t in dev]
        got = m.grad_clip(dev, max_norm, out=out)
        assert_close(got, torch.tensor([norm]), 2 * U * norm, "norm")
        for t, k in zip(dev, keep):
            assert torch.equal(t, k)
        for o, w, t in zip(out, want, grads):
            assert_close(o, w, 4 * U * w.abs() + half_ulp(w, t.dtype) * 1.01, "clipped")
        got2 = m.grad_clip(keep, max_norm)  # in place
        assert torch.equal(got, got2)
        for o, k in zip(out, keep):
            assert torch.equal(o, k)
        assert torch.equal(m.grad_norm(dev), got)


def test_clip_odd_places():
    """Gradients and outputs that begin at any element, and neighbours left alone."""
    import paper_1903_06934_amd as m
    for dtype in (F32, BF16):
        flat, dest = torch.randn(70000, device="cuda").to(dtype), torch.zeros(70000, device="cuda",
                                                                             dtype=dtype)
        cuts = [(1, 100), (103, 40001), (40104, 1), (40107, 16384)]
        grads = [flat[a:a + n] for a, n in cuts]
        outs = [dest[a + 5:a + 5 + n] for a, n in cuts]
        dest.fill_(7.0)
        m.grad_clip(grads, 1.0, out=outs)
        _, want = ref.clip([t.cpu() for t in grads], 1.0)
        inside = torch.zeros(70000, dtype=torch.bool)
        for (a, n), w, o in zip(cuts, want, outs):
            inside[a + 5:a + 5 + n] = True
            assert_close(o, w, 4 * U * w.abs() + half_ulp(w, dtype) * 1.01, "clipped")
        assert (dest.cpu()[~inside] == 7.0).all()


def test_clip_extremes():
    """Squares beyond 32 bits, infinities and NaN."""
    import paper_1903_06934_amd as m
    big = torch.tensor([3e30, -4e30, 1.0], device="cuda")
    norm = m.grad_clip([big], 5.0)
    assert abs(float(norm) / 5e30 - 1) < 1e-6
    assert abs(float(big[0]) - 3) < 1e-5 and abs(float(big[1]) + 4) < 1e-5
    small = torch.tensor([3e-30, 4e-30], device="cuda")
    assert abs(float(m.grad_norm([small])) / 5e-30 - 1) < 1e-6
    for bad in (INF, NAN):
        t = [torch.ones(40, device="cuda"), torch.full((20000,), 2.0, device="cuda")]
        t[1][777] = bad
        norm = float(m.grad_clip(t, 1.0))
        got = torch.cat(t).cpu()
        assert norm == INF if bad == INF else math.isnan(norm)
        odd = torch.zeros(20040, dtype=torch.bool)
        odd[817] = True
        assert torch.isnan(got[817])
        assert (got[~odd] == 0).all() if bad == INF else torch.isnan(got).all()


# ----------------------------------------------------------------- streams, graphs
def _step(m, d, out):
    """One call of each operator, into out's tensors."""
    m.layernorm_fwd(d["x"], d["w"], d["b"], y=out["y"], mean=out["mean"], rstd=out["rstd"],
                    ws=out["ws_f"])
    r = m.logprob_fwd(out["y"], d["t"], top=5, ws=out["ws_l"])
    out["logp"].copy_(r.logp)
    out["top"].copy_(r.top_index)
    m.logprob_bwd(out["y"], r.stats, d["t"], d["dlogp"], dlogits=out["dy"])
    m.layernorm_bwd(out["dy"], d["x"], out["mean"], out["rstd"], d["w"], dx=out["dx"],
                    dw=out["dw"], db=out["db"], ws=out["ws_b"])
    m.grad_clip([out["dw"], out["db"], out["dx"].view(-1)], 0.01, norm=out["norm"],
                ws=out["ws_c"])


def _data(m, rows, cols, xt, seed):
    g = gen(seed, rows, cols)
    d = {"x": randn(g, rows, cols).to(xt).cuda(), "w": randn(g, cols).cuda(),
         "b": randn(g, cols).cuda(), "t": torch.randint(cols, (rows,), generator=g).cuda(),
         "dlogp": randn(g, rows).cuda()}
    new = lambda *s, t=F32: torch.empty(s, dtype=t, device="cuda")
    out = {"y": new(rows, cols, t=xt), "dy": new(rows, cols, t=xt), "dx": new(rows, cols, t=xt),
           "mean": new(rows), "rstd": new(rows), "logp": new(rows), "dw": new(cols),
           "db": new(cols), "norm": new(1), "top": new(rows, 5, t=torch.int64)}
    ws = {"ws_f": m.layernorm_workspace(False, d["x"]), "ws_b": m.layernorm_workspace(True, d["x"]),
          "ws_l": m.logprob_workspace(d["x"], 5),
          "ws_c": m.grad_workspace([out["dw"], out["db"], out["dx"].view(-1)])}
    return d, {**out, **ws}


RESULTS = ["y", "dx", "mean", "rstd", "logp", "dw", "db", "norm", "top"]


@pytest.mark.parametrize("rows,cols,xt", [(300, 1000, BF16), (3, 60000, F32)])
def test_operators_replay_in_a_graph(rows, cols, xt):
    import paper_1903_06934_amd as m
    d, out = _data(m, rows, cols, xt, 1)
    _step(m, d, out)
    torch.cuda.synchronize()
    eager = {k: out[k].clone() for k in RESULTS}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _step(m, d, out)
    torch.cuda.synchronize()
    for rep in range(3):
        for k in RESULTS:
            out[k].fill_(7)
        junk = torch.randn(300, 300, device="cuda") @ torch.randn(300, 300, device="cuda")
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in RESULTS:
            assert torch.equal(out[k], eager[k]), (rep, k)
        del junk


def test_clip_of_many_tensors_in_a_graph():
    """Lists that go through a table: the graph holds their pointers."""
    import paper_1903_06934_amd as m
    g = gen(31)
    src = [randn(g, int(n)) for n in torch.randint(1, 9000, (250,), generator=g)]
    grads = [t.cuda() for t in src]
    out = [torch.empty_like(t) for t in grads]
    norm, ws = torch.empty(1, device="cuda"), m.grad_workspace(grads)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        m.grad_clip(grads, 3.0, out=out, norm=norm, ws=ws)
    for rep in range(3):
        for t, s in zip(grads, src):
            t.copy_(s * (rep + 1))
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        eager = [torch.empty_like(t) for t in grads]
        want = m.grad_clip(grads, 3.0, out=eager)
        assert torch.equal(norm, want)
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


def test_binding_refuses_on_the_gpu():
    """Types, layouts and sizes that the binding does not take."""
    import paper_1903_06934_amd as m
    x = torch.zeros(4, 8, device="cuda")
    w, f64 = torch.zeros(8, device="cuda"), torch.zeros(4, 8, device="cuda", dtype=torch.float64)
    lab = torch.zeros(4, dtype=torch.int64, device="cuda")
    y, mean, rstd = m.layernorm_fwd(x, w, w)
    st = m.logprob_fwd(x).stats
    bad = [
        lambda: m.layernorm_fwd(f64), lambda: m.layernorm_fwd(x, w[:7]),
        lambda: m.layernorm_fwd(x, w, w.half()), lambda: m.layernorm_fwd(x, w.cpu()),
        lambda: m.layernorm_fwd(x, y=y[:3]), lambda: m.layernorm_fwd(x, y=y.half()),
        lambda: m.layernorm_fwd(x.t()), lambda: m.layernorm_fwd(x, mean=mean[:3]),
        lambda: m.layernorm_bwd(x.half(), x, mean, rstd), lambda: m.layernorm_bwd(x, x, rstd[:2], rstd),
        lambda: m.layernorm_bwd(x[:1].expand(4, 8), x, mean, rstd),
        lambda: m.logprob_fwd(x, lab.int()), lambda: m.logprob_fwd(x, lab[:3]),
        lambda: m.logprob_bwd(x, st[:3], lab, mean), lambda: m.logprob_bwd(x, st, lab, mean.half()),
        lambda: m.logprob_bwd(x, st, lab, mean, dlogits=y.half()),
        lambda: m.grad_clip([x, w.double()], 1.0), lambda: m.grad_clip([x.t()], 1.0),
        lambda: m.grad_clip([x, "w"], 1.0), lambda: m.grad_clip([x], 1.0, out=[]),
        lambda: m.grad_clip([x], 1.0, out=[w]), lambda: m.grad_clip([x], 1.0, norm=mean),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    refused = [
        lambda: m.layernorm_fwd(x, y=x), lambda: m.layernorm_fwd(x, eps=-1.0),
        lambda: m.layernorm_fwd(x.bfloat16(), w.half(), w.half()),
        lambda: m.layernorm_fwd(x[:, :0]), lambda: m.logprob_fwd(x, scale=0.0),
        lambda: m.logprob_fwd(x, top=-1), lambda: m.logprob_fwd(torch.zeros(1, 99).cuda(), top=65),
        lambda: m.logprob_bwd(x, st), lambda: m.logprob_bwd(x, st, dlogp=mean),
        lambda: m.logprob_bwd(x[:, :7], st, lab, mean, dlogits=x[:, 1:]),
        lambda: m.grad_clip([w, w], 1.0), lambda: m.grad_clip([w], float("nan")),
        lambda: m.layernorm_bwd(x, x, mean, rstd, ws=torch.empty(0, device="cuda")),
    ]
    for call in refused:
        with pytest.raises((m.MiconvError, ValueError)):
            call()
    # Nothing was launched that left an error behind.
    torch.cuda.synchronize()
    assert torch.isfinite(m.layernorm_fwd(x + 1, w, w)[0]).all()


def test_operators_on_two_streams():
    import paper_1903_06934_amd as m
    data = [_data(m, 500, 900, BF16, 2), _data(m, 4, 50000, F32, 3)]
    want = []
    for d, out in data:
        _step(m, d, out)
        torch.cuda.synchronize()
        want.append({k: out[k].clone() for k in RESULTS})
        for k in RESULTS:
            out[k].fill_(7)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for (d, out), s in zip(data, streams):
        with torch.cuda.stream(s):
            _step(m, d, out)
    torch.cuda.synchronize()
    for (d, out), w in zip(data, want):
        for k in RESULTS:
            assert torch.equal(out[k], w[k]), k


def test_rows_past_32_bits():
    """A matrix whose last rows begin past 2^32 bytes and 2^31 elements."""
    import paper_1903_06934_amd as m
    rows, cols, ld = 5, 3000, 600000000  # f16: 2.4e9 elements, 4.8 GB
    wide = torch.empty(rows * ld, dtype=F16, device="cuda")
    x = wide.view(rows, ld)[:, :cols]
    src = randn(gen(8), rows, cols).to(F16)
    x.copy_(src)
    y, mean, rstd = m.layernorm_fwd(x)
    plain = m.layernorm_fwd(src.cuda())
    assert torch.equal(y, plain[0])
    t = torch.arange(rows, device="cuda")
    a, b = m.logprob_fwd(x, t, top=3), m.logprob_fwd(src.cuda(), t, top=3)
    for p, q in zip(a, b):
        assert torch.equal(p, q)
    dl = torch.ones(rows, device="cuda")
    want = m.logprob_bwd(src.cuda(), b.stats, t, dl)
    dx = m.layernorm_bwd(want, x, mean, rstd)[0]
    assert torch.equal(dx, m.layernorm_bwd(want, src.cuda(), mean, rstd)[0])
    m.logprob_bwd(x, a.stats, t, dl, dlogits=x)
    assert torch.equal(x.contiguous(), want)
