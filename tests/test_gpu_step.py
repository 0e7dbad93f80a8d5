"""Dropout, residual branches and the losses of fine-tuning on the GPU against their
plain 64-bit forms (step_ref.py), over types, sizes on both sides of every launch rule,
strides, alignments, masks and sequences that leave nothing.

Bounds, with u = 2^-24: those of step_ref.py, those of the layer norm's tests for what the
norm computes, and half a unit in a result's last place."""
import math

import pytest
import torch

import step_ref as ref
import train_ref
from test_gpu_train import norm_terms, gen, randn, strided, untouched
from train_ref import INF, U, assert_close, half_ulp

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAN = math.nan
SEED = 0xFEDCBA9876543210


def ulp(want, dtype):
    return half_ulp(want, dtype) * 1.01


# --------------------------------------------------------------------- dropout
@pytest.mark.parametrize("xt", [F32, BF16, F16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 7), (3, 8), (5, 3), (700, 1), (37, 13), (129, 64),
                                       (33, 513), (128, 1000), (2, 40001), (300, 4096)])
def test_dropout(rows, cols, xt):
    import paper_1903_06934_amd as m
    g = gen(rows, cols)
    x, res = randn(g, rows, cols).to(xt), 3 * randn(g, rows, cols).to(xt)
    for p, layer, step in ((0.1, 0, 0), (0.5, 7, 2 ** 32 - 1), (0.999, 2 ** 32 - 1, 5)):
        keep = ref.mask_of(rows, cols, p, SEED, layer, step)
        want, size = ref.dropout(x, keep, p)
        for gap, shift in ((0, 0), (0, 1), (5, 3)):
            xv, _ = strided(x, gap, shift)
            yv, wide = strided(torch.zeros(rows, cols, dtype=xt), gap, shift)
            y = m.dropout_fwd(xv, p, SEED, layer, step, y=yv)
            assert_close(y, want, U * size + ulp(want, xt), f"y {p} {gap}")
            assert bool((y.cpu()[~keep] == 0).all())
            untouched(yv, wide)
            dx = m.dropout_bwd(xv, p, SEED, layer, step)
            assert torch.equal(dx, y)
    rv, _ = strided(res, 2, 1)
    both, size = ref.dropout(x, keep, p, res)
    y = m.dropout_fwd(x.cuda(), p, SEED, layer, step, residual=rv)
    assert_close(y, both, U * size + ulp(both, xt), "residual")
    # In place, to x and to the residual.
    xc, rc = x.cuda(), res.cuda()
    assert m.dropout_fwd(xc, p, SEED, layer, step, residual=rv, y=xc) is xc and torch.equal(xc, y)
    m.dropout_fwd(x.cuda(), p, SEED, layer, step, residual=rc, y=rc)
    assert torch.equal(rc, y)
    xc = x.cuda()
    m.dropout_bwd(xc, p, SEED, layer, step, dx=xc)
    assert torch.equal(xc, dx)


@pytest.mark.parametrize("xt", [F32, BF16])
def test_dropout_borders(xt):
    """None and all dropped; what is dropped is 0 whatever it was; no rows."""
    import paper_1903_06934_amd as m
    x = torch.tensor([[INF, -INF, NAN, 1.0, -2.0, 0.0, 3.0, 4.0, 5.0]] * 50, dtype=xt, device="cuda")
    assert torch.equal(torch.nan_to_num(m.dropout_fwd(x, 0.0, 1), 9), torch.nan_to_num(x, 9))
    assert torch.equal(torch.nan_to_num(m.dropout_fwd(x, 2.0 ** -18, 1), 9), torch.nan_to_num(x, 9))
    assert bool((m.dropout_fwd(x, 1.0, 1) == 0).all())
    res = torch.full_like(x, 2.5)
    assert torch.equal(m.dropout_fwd(x, 1.0, 1, residual=res), res)
    keep = ref.mask_of(50, 9, 0.4, 1)
    y = m.dropout_fwd(x, 0.4, 1).cpu()
    assert bool((y[~keep] == 0).all())
    assert torch.equal(torch.isnan(y), torch.isnan(x.cpu()) & keep)
    assert torch.equal(torch.isinf(y), torch.isinf(x.cpu()) & keep)
    empty = torch.empty(0, 5, dtype=xt, device="cuda")
    assert m.dropout_fwd(empty, 0.1, 1).shape == (0, 5)


def test_dropout_numbers():
    """Seeds, layers and steps have masks of their own; the mask goes by the element's
    index, not by type, shape or strides; a step on the device is added."""
    import paper_1903_06934_amd as m
    x = torch.ones(64, 96, device="cuda")
    base = m.dropout_fwd(x, 0.5, 5, 1, 9)
    for other in ((6, 1, 9), (5 + 2 ** 32, 1, 9), (5, 2, 9), (5, 1, 10)):
        y = m.dropout_fwd(x, 0.5, *other)
        # Independent masks of a half agree in a half of the places.
        assert 0.4 < float((y == base).float().mean()) < 0.6
    assert torch.equal(m.dropout_fwd(x.view(3, 2, 1024), 0.5, 5, 1, 9).view(64, 96), base)
    assert torch.equal(m.dropout_fwd(x.bfloat16(), 0.5, 5, 1, 9).float(), base)
    at = torch.tensor([2 ** 32 * 3 + 9], device="cuda")
    assert torch.equal(m.dropout_fwd(x, 0.5, 5, 1, at), base)
    assert torch.equal(m.dropout_fwd(x, 0.5, 5, 1, 2 ** 32 + 9), base)
    with pytest.raises(ValueError):
        m.dropout_fwd(x, 0.5, 5, 1, at.int())
    with pytest.raises(ValueError):
        m.dropout_fwd(x, 0.5, 5, 1, at.cpu())


def test_dropout_share():
    """The share that is dropped, and every half word's: by five standard deviations."""
    import paper_1903_06934_amd as m
    n = 1 << 22
    y = m.dropout_fwd(torch.ones(n, device="cuda"), 0.25, 77)
    dropped = (y == 0).double()
    assert abs(float(dropped.mean()) - 0.25) < 5 * math.sqrt(0.1875 / n)
    each = dropped.view(-1, 8).mean(0)
    assert bool(((each - 0.25).abs() < 5 * math.sqrt(0.1875 / (n / 8))).all())
    assert abs(float(y.double().mean()) - 1) < 5 * math.sqrt(1 / 3 / n)


# ------------------------------------------------------------ residual branches
COLS = [1, 3, 7, 8, 24, 64, 100, 130, 197, 255, 512, 513, 1000, 1025, 2048, 2049, 4096, 5000, 8192,
        9001, 16385, 32768, 32771, 50000]


@pytest.mark.parametrize("xt,wt", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F16)])
@pytest.mark.parametrize("cols", COLS)
def test_residual_norm(cols, xt, wt):
    import paper_1903_06934_amd as m
    for rows, p in ((37 if cols <= 5000 else 5, 0.3), (600 if cols <= 513 else 70, 0.0)):
        check_residual_norm(m, rows, cols, xt, wt, p)


def check_residual_norm(m, rows, cols, xt, wt, p):
    g = gen(rows, cols)
    x, res = randn(g, rows, cols).to(xt), (randn(g, rows, cols) + randn(g, rows, 1)).to(xt)
    w, b = (1 + 0.3 * randn(g, cols)).to(wt), randn(g, cols).to(wt)
    num = dict(p=p, seed=SEED, layer=3, step=11)
    keep = ref.mask_of(rows, cols, p, SEED, 3, 11)
    gap, shift = (0, 0) if cols % 3 else (5, 3)
    xv, _ = strided(x, gap, shift)
    rv, _ = strided(res, gap + 2, 0)
    tv, wide_t = strided(torch.zeros(rows, cols, dtype=xt), gap, shift)
    yv, wide_y = strided(torch.zeros(rows, cols, dtype=xt), gap + 1, shift)
    out = m.residual_norm_fwd(xv, rv, w.cuda(), b.cuda(), 1e-5, **num, total=tv, y=yv)
    want, size = ref.dropout(x, keep, p, res)
    assert_close(out.total, want, U * size + ulp(want, xt), "total")
    total = out.total.cpu()
    ry, rmean, rrstd, nsize, msize = train_ref.layernorm_fwd(total, w, b)
    k = norm_terms(cols) * U
    assert_close(out.mean, rmean, k * msize, "mean")
    assert_close(out.rstd, rrstd, rrstd * (k + (k * msize * rrstd) ** 2), "rstd")
    assert_close(out.y, ry, 2 * k * nsize + ulp(ry, xt), "y")
    untouched(tv, wide_t)
    untouched(yv, wide_y)
    # In place to the residual: the same.
    rc = res.cuda()
    again = m.residual_norm_fwd(xv, rc, w.cuda(), b.cuda(), 1e-5, **num, total=rc)
    assert again.total is rc and torch.equal(rc, out.total) and torch.equal(again.y, out.y)

    dy, dt = randn(g, rows, cols).to(xt), randn(g, rows, cols).to(xt)
    dyv, _ = strided(dy, gap, shift)
    (dn, nsize), (rdw, sdw), (rdb, sdb) = train_ref.layernorm_bwd(dy, total, out.mean.cpu(),
                                                                  out.rstd.cpu(), w)
    for dtotal in (dt, None):
        rg = dn if dtotal is None else dn + dt.double()
        off = k * nsize + U * rg.abs()
        rx, _ = ref.dropout(rg, keep, p)
        drv, wide_r = strided(torch.zeros(rows, cols, dtype=xt), gap + 2, shift)
        dxv, wide_x = strided(torch.zeros(rows, cols, dtype=xt), gap, shift)
        dtv = None if dtotal is None else strided(dt, 1, 2)[0]
        dx, dr, dw, db = m.residual_norm_bwd(dyv, tv, out.mean, out.rstd, w.cuda(), dtv, **num,
                                             dx=dxv, dresidual=drv)
        assert_close(dr, rg, off + ulp(rg, xt), "dresidual")
        assert_close(dx, rx, off * ref.scale_of(p) + 2 * U * rx.abs() + ulp(rx, xt), "dx")
        assert bool((dx.cpu()[~keep] == 0).all())
        untouched(drv, wide_r)
        untouched(dxv, wide_x)
        for got, val, mag, name in ((dw, rdw, sdw, "dw"), (db, rdb, sdb, "db")):
            assert got.dtype == wt
            assert_close(got, val, 64 * U * mag + ulp(val, wt), name)
    # In place to dtotal, and in parts: the same bits.
    dtc = dt.cuda()
    full = m.residual_norm_bwd(dyv, tv, out.mean, out.rstd, w.cuda(), dt.cuda(), **num)
    part = m.residual_norm_bwd(dyv, tv, out.mean, out.rstd, w.cuda(), dtc, **num, dresidual=dtc,
                               with_weight=False, with_bias=False)
    assert part[1] is dtc and part[2] is None and part[3] is None
    assert torch.equal(dtc, full[1]) and torch.equal(part[0], full[0])
    if p == 0:
        assert full[0] is full[1]
    part = m.residual_norm_bwd(dyv, tv, out.mean, out.rstd, w.cuda(), dt.cuda(), **num,
                               with_input=False)
    assert part[0] is None and part[1] is None
    assert torch.equal(part[2], full[2]) and torch.equal(part[3], full[3])


@pytest.mark.parametrize("xt", [F32, BF16, F16])
@pytest.mark.parametrize("base", [40, 1200, 4352, 9000])
def test_residual_norm_short_vectors(base, xt):
    """Every number of elements that the row's end leaves of a vector, in every form; rows
    whose groups of random numbers begin at every place."""
    import paper_1903_06934_amd as m
    for cols in range(base, base + 8):
        check_residual_norm(m, 19, cols, xt, F32, 0.4)


@pytest.mark.parametrize("xt", [F32, BF16])
@pytest.mark.parametrize("cols", [9, 10, 33, 80, 130, 145, 257, 288, 513, 576, 1088, 2049, 4100])
def test_residual_norm_row_tails(cols, xt):
    """Many rows some elements longer than whole vectors of a wave or some waves."""
    import paper_1903_06934_amd as m
    check_many(m, 2100, cols, xt)


def check_many(m, rows, cols, xt):
    g = gen(rows, cols, 5)
    x, res, dy = (randn(g, rows, cols).to(xt) for _ in range(3))
    w, num = randn(g, cols), dict(p=0.2, seed=9, layer=1, step=2)
    keep = ref.mask_of(rows, cols, 0.2, 9, 1, 2)
    out = m.residual_norm_fwd(x.cuda(), res.cuda(), w.cuda(), **num)
    want, size = ref.dropout(x, keep, 0.2, res)
    assert_close(out.total, want, U * size + ulp(want, xt), "total")
    total = out.total.cpu()
    ry, _, _, nsize, _ = train_ref.layernorm_fwd(total, w)
    k = norm_terms(cols) * U
    assert_close(out.y, ry, 2 * k * nsize + ulp(ry, xt), "y")
    dx, dr, dw, db = m.residual_norm_bwd(dy.cuda(), out.total, out.mean, out.rstd, w.cuda(),
                                         res.cuda(), **num)
    (dn, nsize), (rdw, sdw), (rdb, sdb) = train_ref.layernorm_bwd(dy, total, out.mean.cpu(),
                                                                  out.rstd.cpu(), w)
    rg = dn + res.double()
    off = k * nsize + U * rg.abs()
    rx, _ = ref.dropout(rg, keep, 0.2)
    assert_close(dr, rg, off + ulp(rg, xt), "dresidual")
    assert_close(dx, rx, off * ref.scale_of(0.2) + 2 * U * rx.abs() + ulp(rx, xt), "dx")
    for got, val, mag, name in ((dw, rdw, sdw, "dw"), (db, rdb, sdb, "db")):
        assert_close(got, val, (300 + rows / 256) * U * mag, name)


@pytest.mark.parametrize("rows", [0, 1, 2, 255, 1023])
@pytest.mark.parametrize("cols,xt", [(48, BF16), (513, F32), (3000, BF16), (9000, F32),
                                     (40000, BF16)])
def test_residual_norm_rows(rows, cols, xt):
    import paper_1903_06934_amd as m
    if rows:
        check_many(m, rows if cols < 9000 else min(rows, 67), cols, xt)
        return
    x = torch.empty(0, cols, dtype=xt, device="cuda")
    out = m.residual_norm_fwd(x, x, p=0.5, seed=1)
    dx, dr, dw, db = m.residual_norm_bwd(x, x, out.mean, out.rstd, p=0.5, seed=1)
    assert dx.shape == dr.shape == (0, cols) and not dw.any() and not db.any()


def test_residual_norm_special_rows():
    """Rows of equal or neighbouring elements after the sum (they are read again where they
    were written), infinities and NaN in theirs; a dropped NaN is none."""
    import paper_1903_06934_amd as m
    for cols in (20, 700, 5000, 40000):
        for xt in (F32, BF16):
            res = torch.full((8, cols), 100.25, dtype=xt)
            x = torch.zeros(8, cols, dtype=xt)
            x[1] = 0.5
            x[2, ::2] = 1.0
            x[3, 3], x[4, cols - 1] = INF, NAN
            keep = ref.mask_of(8, cols, 0.5, 4)
            x[5] = torch.where(keep[5], torch.zeros(()), torch.tensor(NAN)).to(xt)
            for p, total in ((0.0, None), (0.0, "res"), (0.5, None)):
                rc = res.cuda()
                out = m.residual_norm_fwd(x.cuda(), rc, p=p, seed=4,
                                          total=rc if total else None)
                t = out.total.cpu()
                ry, rmean, _, nsize, msize = train_ref.layernorm_fwd(t)
                k = norm_terms(cols) * U
                fine = torch.isfinite(t.double()).all(1)
                assert fine[[0, 1, 2, 6, 7]].all() and bool(fine[5]) == (p == 0.5)
                assert_close(out.mean[fine.cuda()], rmean[fine], (k * msize)[fine], "mean")
                assert_close(out.y[fine.cuda()], ry[fine], (2 * k * nsize)[fine] +
                             ulp(ry[fine], xt), "y")
                equal = (t == t[:, :1]).all(1) & fine
                assert bool((out.y.cpu()[equal] == 0).all())
                assert torch.isnan(out.y.cpu()[~fine]).all()


# ---------------------------------------------------------------------- losses
def make_starts(g, tokens, seqs, tail=0):
    cuts = torch.randint(max(1, tokens - tail + 1), (seqs + 1,), generator=g)
    if seqs:
        cuts[0] = 0
    cuts[-1] = max(0, tokens - tail)
    return torch.sort(cuts)[0]


def make_policy(g, n, seqs, tail=0, masked=0.0):
    lp = -2 * randn(g, n).abs()
    d = {"logp": lp, "old": lp - 0.3 * randn(g, n), "ref": lp + 0.5 * randn(g, n),
         "entropy": 3 * torch.rand(n, generator=g), "starts": make_starts(g, n, seqs, tail),
         "adv": randn(g, n), "seq_adv": randn(g, seqs)}
    if masked:
        d["mask"] = torch.rand(n, generator=g) >= masked
        if seqs > 1:
            d["mask"][:d["starts"][1]] = False
        for i, k in enumerate(("logp", "old", "ref", "entropy", "adv")):
            d[k] = torch.where(d["mask"], d[k], torch.tensor([NAN, INF, -INF])[i % 3])
    return d


def call_policy(m, d, by, kl, entropy, mean, dual=INF, scale=1.0, kl_weight=0.07, **more):
    c = lambda k: d[k].cuda() if k in d and d[k] is not None else None
    return m.policy_loss(c("logp"), c("old"), c("seq_adv") if by else c("adv"), by_sequence=by,
                         ref_logp=c("ref") if kl else None, entropy=c("entropy") if entropy else None,
                         mask=c("mask"), starts=c("starts"), clip_low=0.2, clip_high=0.3,
                         dual_clip=dual, kl=kl or "low", kl_weight=kl_weight if kl else 0.0,
                         entropy_weight=0.02 if entropy else 0.0, mean=mean, scale=scale, **more)


def want_policy(d, by, kl, entropy, mean, dual=INF, scale=1.0, kl_weight=0.07):
    return ref.policy(d["logp"], d["old"], d["seq_adv"] if by else d["adv"], by,
                      d["ref"] if kl else None, d["entropy"] if entropy else None, d.get("mask"),
                      d["starts"], 0.2, 0.3, dual, kl or "low", kl_weight if kl else 0.0,
                      0.02 if entropy else 0.0, mean, scale)


def check_policy(m, d, *args, **kw):
    out = call_policy(m, d, *args, **kw)
    (stats, sb), (g, gb), (gh, hb) = want_policy(d, *args, **kw)
    assert_close(out.dlogp, g, gb, f"dlogp {args}")
    if args[2]:
        assert_close(out.dentropy, gh, hb, f"dentropy {args}")
    else:
        assert out.dentropy is None
    assert_close(out.stats, stats, sb, f"stats {args}")
    again = call_policy(m, d, *args, **kw)
    assert torch.equal(out.stats, again.stats) and torch.equal(out.dlogp, again.dlogp)
    only = call_policy(m, d, *args, **kw, with_grad=False)
    assert only.dlogp is None and only.dentropy is None and torch.equal(only.stats, out.stats)


@pytest.mark.parametrize("masked", [0.0, 0.4])
@pytest.mark.parametrize("tokens,seqs,tail", [
    (1, 1, 0), (2, 5, 0), (5, 1, 2), (63, 3, 0), (1000, 7, 13), (4096, 4096, 0), (4097, 5, 0),
    (4099, 300, 0), (8192, 1, 0), (8192, 8192, 0), (8193, 1, 0), (8193, 40, 5), (300, 9000, 7), (20001, 3, 0), (50003, 600, 77),
    (70000, 20000, 1)])
def test_policy(tokens, seqs, tail, masked):
    """Both means, both kinds of advantage, all forms, with and without each part."""
    import paper_1903_06934_amd as m
    d = make_policy(gen(tokens, seqs, 1), tokens, seqs, tail, masked)
    check_policy(m, d, False, "low", True, "tokens")
    check_policy(m, d, True, "linear", False, "sequences", 3.0)
    check_policy(m, d, False, "square", True, "sequences", 1.5, -2.5)
    check_policy(m, d, True, "", False, "tokens", 1.2)
    check_policy(m, d, False, "", False, 1000.0, scale=1024.0)
    check_policy(m, d, True, "low", True, 3.0, kl_weight=0.0)


@pytest.mark.parametrize("tokens", [0, 1, 700, 9000])
def test_policy_nothing_counts(tokens):
    """No token, no sequence, sequences of none, a mask that leaves nothing."""
    import paper_1903_06934_amd as m
    d = make_policy(gen(tokens), tokens, 3)
    nothing = torch.zeros(tokens, dtype=torch.bool)
    z = lambda *v: torch.tensor(v, dtype=torch.int64)
    for starts, mask in ((d["starts"], nothing), (z(0, 0, 0, 0), None), (z(tokens), None),
                         (z(tokens, tokens), None), (z(5, 5), None)):
        d["starts"], d["mask"] = starts, mask
        d["seq_adv"] = torch.ones(len(starts) - 1)
        for by, mean in ((False, "tokens"), (True, "sequences"), (True, 2.0)):
            out = call_policy(m, d, by, "low", True, mean, dlogp=torch.full((tokens,), NAN).cuda())
            assert not out.stats.any() and not out.dlogp.any() and not out.dentropy.any()


@pytest.mark.parametrize("tokens", [500, 20000])
def test_policy_of_no_sequences(tokens):
    """starts left out: all tokens are one sequence; masks of uint8, any byte but 0."""
    import paper_1903_06934_amd as m
    d = make_policy(gen(tokens, 3), tokens, 1, 0, 0.3)
    one = call_policy(m, d, False, "low", True, "tokens")
    d["starts"] = None
    mask = d["mask"]
    d["mask"] = mask.to(torch.uint8) * 128
    out = call_policy(m, d, False, "low", True, "tokens")
    assert torch.equal(out.stats, one.stats) and torch.equal(out.dlogp, one.dlogp)
    for by, mean in ((True, "tokens"), (False, "sequences")):
        with pytest.raises((ValueError, m.MiconvError)):
            call_policy(m, d, by, "low", True, mean)


@pytest.mark.parametrize("tokens", [600, 30000])
def test_policy_starts_past_the_tokens(tokens):
    """Starts below 0 and past the tokens are cut to them; tokens in no sequence have no
    gradient."""
    import paper_1903_06934_amd as m
    d = make_policy(gen(tokens, 4), tokens, 4)
    for starts in ([-7, 100, 300, 2 ** 40, 2 ** 41], [-2 ** 62, -1, 0, 17, 2 ** 62],
                   [200, 250, 250, 400, 500]):
        d["starts"] = torch.tensor(starts)
        for by in (False, True):
            check_policy(m, d, by, "low", False, "sequences")
            check_policy(m, d, by, "low", False, "tokens")


def test_policy_falling_starts_stay_inside():
    """Starts that fall: the results are unspecified, but nothing else is written."""
    import paper_1903_06934_amd as m
    for tokens in (700, 30000):
        d = make_policy(gen(tokens, 6), tokens, 6, 0, 0.2)
        wide = torch.full((tokens + 64,), 7.0, device="cuda")
        for starts in ([tokens, 3, 600, 2, 1, 0, 5], [5, 4, 3, 2, 1, 0, -9],
                       [0, tokens, 0, tokens, 0, tokens, 0]):
            d["starts"] = torch.tensor(starts)
            for mean in ("tokens", "sequences"):
                call_policy(m, d, True, "low", False, mean, dlogp=wide[32:32 + tokens])
            r = torch.full((70,), 7.0, device="cuda")
            m.preference_loss(torch.zeros(tokens, device="cuda"), None, d["starts"].cuda(), 0.1,
                              rewards=r[32:38], dlogp=wide[32:32 + tokens])
            assert bool((r[:32] == 7).all()) and bool((r[38:] == 7).all())
        assert bool((wide[:32] == 7).all()) and bool((wide[32 + tokens:] == 7).all())


@pytest.mark.parametrize("tokens", [64, 9000])
def test_policy_special_tokens(tokens):
    """A token without a probability, then or now; NaN only reaches its own gradient."""
    import paper_1903_06934_amd as m
    d = make_policy(gen(tokens, 5), tokens, 1)
    d["adv"] = torch.ones(tokens)
    d["logp"][3], d["old"][5] = -INF, -INF  # ratio 0, and infinite: clipped
    out = call_policy(m, d, False, "", False, "tokens")
    assert out.dlogp[3] == 0 and out.dlogp[5] == 0
    assert torch.isfinite(out.stats[:2]).all() and out.ratio == INF
    d["logp"][40] = NAN
    out = call_policy(m, d, False, "low", False, "tokens")
    assert torch.isnan(out.loss) and torch.isnan(out.dlogp[40])
    assert int(torch.isnan(out.dlogp).sum()) == 1


def test_policy_border():
    """Log ratios at the clip's border and the next numbers above and below it."""
    import paper_1903_06934_amd as m
    hi, lo = math.log1p(0.3), math.log1p(-0.2)
    near = []
    for v in (hi, lo):
        f = torch.tensor(v, dtype=F32)
        near += [f, torch.nextafter(f, torch.tensor(9.0)), torch.nextafter(f, torch.tensor(-9.0))]
    lp = torch.stack(near * 2)
    adv = torch.tensor([1.0] * 6 + [-1.0] * 6)
    d = {"logp": lp, "old": torch.zeros(12), "adv": adv, "starts": None}
    out = call_policy(m, d, False, "", False, 1.0)
    for i in range(12):
        v = float(lp[i])
        clipped = v > hi if adv[i] > 0 else v < lo
        assert (float(out.dlogp[i]) == 0) == clipped, i


def test_policy_gradient_by_differences():
    import paper_1903_06934_amd as m
    d = make_policy(gen(8), 3000, 5, 11, 0.3)
    out = call_policy(m, d, True, "low", True, "sequences", 2.0)
    g, h = gen(9), 1e-5
    v = torch.where(d["mask"], randn(g, 3000), torch.zeros(())).double()
    for key, grad in (("logp", out.dlogp), ("entropy", out.dentropy)):
        loss = []
        for sign in (1, -1):
            e = {k: t.double() if torch.is_tensor(t) and t.is_floating_point() else t
                 for k, t in d.items()}
            e[key] = torch.where(d["mask"], e[key] + sign * h * v, e[key])
            loss.append(float(want_policy(e, True, "low", True, "sequences", 2.0)[0][0][0]))
        diff, got = (loss[0] - loss[1]) / (2 * h), float((grad.cpu().double() * v).sum())
        # A token within 1e-5 of the clip's border moves the difference by its share.
        assert abs(diff - got) < 1e-3 * (1e-2 + abs(diff))


def make_pairs(g, n, pairs, tail=0, masked=0.0):
    lp = -2 * randn(g, n).abs()
    d = {"logp": lp, "ref": lp + 0.2 * randn(g, n), "starts": make_starts(g, n, 2 * pairs, tail)}
    if masked:
        d["mask"] = torch.rand(n, generator=g) >= masked
        if pairs:
            d["mask"][:d["starts"][1]] = False
        d["logp"] = torch.where(d["mask"], lp, torch.tensor(NAN))
        d["ref"] = torch.where(d["mask"], d["ref"], torch.tensor(-INF))
    return d


def check_pairs(m, d, use_ref=True, **kw):
    c = lambda k: d[k].cuda() if d.get(k) is not None else None
    ref_logp = c("ref") if use_ref else None
    out = m.preference_loss(c("logp"), ref_logp, c("starts"), mask=c("mask"), **kw)
    (stats, sb), (r, rb), (g, gb) = ref.preference(d["logp"], d["ref"] if use_ref else None,
                                                   d["starts"], mask=d.get("mask"), **kw)
    assert_close(out.rewards, r, rb, f"rewards {kw}")
    assert_close(out.dlogp, g, gb, f"dlogp {kw}")
    assert_close(out.stats, stats, sb, f"stats {kw}")
    again = m.preference_loss(c("logp"), ref_logp, c("starts"), mask=c("mask"), **kw)
    for a, b in zip(out, again):
        assert torch.equal(a, b)
    only = m.preference_loss(c("logp"), ref_logp, c("starts"), mask=c("mask"), with_grad=False, **kw)
    assert only.dlogp is None and torch.equal(only.stats, out.stats)


@pytest.mark.parametrize("masked", [0.0, 0.4])
@pytest.mark.parametrize("tokens,pairs,tail", [
    (1, 1, 0), (2, 4, 0), (7, 2, 3), (100, 1, 0), (1000, 7, 13), (4096, 512, 0), (900, 513, 0),
    (4097, 5, 0), (4099, 150, 0), (8192, 1, 0), (8192, 1024, 0), (8193, 1, 0), (8193, 20, 5), (300, 1500, 7), (20001, 2, 0), (50003, 300, 77),
    (70000, 10000, 1)])
def test_preference(tokens, pairs, tail, masked):
    import paper_1903_06934_amd as m
    d = make_pairs(gen(tokens, pairs, 2), tokens, pairs, tail, masked)
    check_pairs(m, d, beta=0.1)
    check_pairs(m, d, beta=0.5, smoothing=0.2, margin=0.3, length_mean=True, scale=-3.0)
    check_pairs(m, d, beta=0.05, form="squared")
    check_pairs(m, d, beta=2.0, form="squared", length_mean=True, margin=-1.0)
    # No gap is at the hinge: an odd margin.
    check_pairs(m, d, beta=0.3, form="hinge", margin=0.12345)
    check_pairs(m, d, use_ref=False, beta=1.0, smoothing=1.0, length_mean=True)


@pytest.mark.parametrize("lengths", [
    [75001, 0, 75000, 64, 2047, 2048], [250000] + 41 * [1000], 150 * [7] + [250001] + 149 * [300],
    [8192] * 40, [1, 300000]], ids=lambda v: f"{len(v)}x{max(v)}")
def test_long_sequences(lengths):
    """Sequences of many chunks of tokens, alone and among short ones."""
    import paper_1903_06934_amd as m
    n, seqs = sum(lengths), len(lengths)
    starts = torch.tensor([0] + lengths).cumsum(0)
    d = dict(make_policy(gen(n, seqs, 3), n, seqs, 0, 0.2), starts=starts)
    check_policy(m, d, True, "low", True, "sequences")
    d = dict(make_pairs(gen(n, seqs, 4), n, seqs // 2, 0, 0.2), starts=starts)
    check_pairs(m, d, beta=0.1, smoothing=0.1, length_mean=True)
    d.pop("mask")
    d["logp"], d["ref"] = d["logp"].nan_to_num(-1.0), d["ref"].nan_to_num(0, 0, -0.5)
    check_pairs(m, d, beta=0.002, form="squared")


@pytest.mark.parametrize("tokens", [0, 1, 700, 9000])
def test_preference_nothing_counts(tokens):
    import paper_1903_06934_amd as m
    lp = torch.full((tokens,), NAN, device="cuda")
    z = lambda *v: torch.tensor(v, dtype=torch.int64, device="cuda")
    none = torch.zeros(tokens, dtype=torch.bool, device="cuda")
    for starts, mask in ((z(0, 0, 0), None), (z(0, tokens // 2, tokens), none), (z(0), None),
                         (z(tokens, tokens, tokens, tokens, tokens), None)):
        out = m.preference_loss(lp, None, starts, 0.1, mask=mask,
                                dlogp=torch.full((tokens,), NAN, device="cuda"))
        assert not out.stats.any() and not out.rewards.any() and not out.dlogp.any()
    with pytest.raises(ValueError):
        m.preference_loss(lp, None, z(0, tokens), 0.1)


@pytest.mark.parametrize("tokens", [400, 30000])
def test_preference_special_pairs(tokens):
    """A pair of two empty sequences does not count; an infinity or NaN stays in its pair's
    gradients and rewards; far gaps neither overflow nor lose their loss."""
    import paper_1903_06934_amd as m
    lp = randn(gen(tokens, 7), tokens)
    q = tokens // 8
    starts = torch.tensor([0, q, 2 * q, 2 * q, 4 * q, 5 * q, 6 * q, 6 * q, 8 * q])
    lp[10], lp[q + 10] = -INF, NAN
    lp[4 * q:5 * q] = -1e5
    out = m.preference_loss(lp.cuda(), None, starts.cuda(), 1.0)
    r, g = out.rewards.cpu(), out.dlogp.cpu()
    assert r[0] == -INF and torch.isnan(r[1]) and r[2] == 0 and torch.isfinite(r[3:]).all()
    assert torch.isnan(g[q:2 * q]).all() and torch.isnan(g[5 * q:6 * q]).all()
    assert torch.isfinite(g[2 * q:5 * q]).all() and torch.isfinite(g[6 * q:]).all()
    # Pair 0: the gap is -inf + large, its slope -1 / 3 pairs (sequences 2 and 6, which
    # are pair 2, have no token).
    third = torch.tensor(1 / 3)
    assert bool((g[:q] == -third).all()) and bool((g[4 * q:5 * q] == third).all())
    d = {"logp": torch.tensor([-2e4, 3.0, 0.0, 2e4]), "starts": torch.arange(5)}
    check_pairs(m, d, use_ref=False, beta=1.0)


def test_losses_in_strided_and_shaped_tensors():
    """Contiguous tensors of any shape; others are refused."""
    import paper_1903_06934_amd as m
    d = make_policy(gen(3), 96, 2)
    lp, old, adv = (d[k].cuda() for k in ("logp", "old", "adv"))
    a = m.policy_loss(lp, old, adv)
    b = m.policy_loss(lp.view(8, 12), old.view(8, 12), adv)
    assert b.dlogp.shape == (8, 12) and torch.equal(a.dlogp, b.dlogp.view(-1))
    for bad in (lp.view(8, 12).t(), lp.double(), lp[:95]):
        with pytest.raises(ValueError):
            m.policy_loss(lp, bad, adv)
    with pytest.raises(ValueError):
        m.policy_loss(lp, old, adv, starts=torch.zeros(0, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        m.policy_loss(lp, old, adv, starts=torch.tensor([0, 96], device="cuda", dtype=torch.int32))
