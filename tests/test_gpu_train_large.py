"""The training step's operators at the sizes where launches are cut or indices
grow: millions of short rows, more rows than a grid's second dimension, single
very long rows, tensors past 2^31 elements.  References in 64 bits on sampled
rows, by torch on the GPU; bounds as in test_gpu_train.py."""
import math

import pytest
import torch

from train_ref import U, half_ulp, assert_close
import train_ref as ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _cuda(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(n, *more):
    return torch.tensor(sorted({r for r in (0, 1, n // 2, n - 2, n - 1, *more) if 0 <= r < n}))


@pytest.mark.parametrize("rows,vocab,xt,top", [
    (9_000_001, 3, F16, 2),      # several launches of waves and of small groups
    (70_001, 4097, F16, 3),      # more rows than one launch of pieces backward
])
def test_many_rows_of_logits(rows, vocab, xt, top):
    import paper_1903_06934_amd as m
    z = (2 * torch.randn(rows, vocab, generator=_cuda(1), device="cuda")).to(xt)
    t = torch.randint(vocab, (rows,), generator=_cuda(2), device="cuda")
    dl = torch.randn(rows, generator=_cuda(3), device="cuda")
    out = m.logprob_fwd(z, t, top=top)
    dz = m.logprob_bwd(z, out.stats, t, dl)
    some = _rows(rows, 65534, 65535, 65536, (1 << 21) - 1, 1 << 21, (1 << 23) - 1, 1 << 23)
    at = some.cuda()
    want = ref.logprob_fwd(z[at].cpu(), t[at].cpu(), top)
    base = 64 * U * (3 + math.log(vocab))
    assert_close(out.lse[at], want["lse"], base + 4 * U * want["lse"].abs(), "lse")
    assert_close(out.logp[at], want["logp"], base + 4 * U * want["logp"].abs(), "logp")
    assert torch.equal(out.top_index[at].cpu(), want["top_index"])
    rz, size = ref.logprob_bwd(z[at].cpu(), t[at].cpu(), 1.0, out.stats[at].cpu(), dl[at].cpu())
    assert_close(dz[at], rz, 8 * U * size + half_ulp(rz, xt) * 1.01 + 1e-37, "dlogits")
    # All rows: the gradient of a row sums to 0 up to its elements' roundings.
    total = dz.double().sum(1).abs()
    assert bool((total <= vocab * 2.0 ** -11 * dl.abs().double() + 1e-6).all())


def test_many_short_rows():
    import paper_1903_06934_amd as m
    rows, cols = 5_000_003, 9
    x = torch.randn(rows, cols, generator=_cuda(4), device="cuda").to(BF16)
    dy = torch.randn(rows, cols, generator=_cuda(5), device="cuda").to(BF16)
    y, mean, rstd = m.layernorm_fwd(x)
    dx, dw, db = m.layernorm_bwd(dy, x, mean, rstd)
    some = _rows(rows, 1 << 20, 1 << 22)
    at = some.cuda()
    ry, rmean, rrstd, size, msize = ref.layernorm_fwd(x[at].cpu())
    assert_close(mean[at], rmean, 48 * U * msize, "mean")
    assert_close(y[at], ry, 96 * U * size + half_ulp(ry, BF16) * 1.01, "y")
    want = ref.layernorm_bwd(dy[at].cpu(), x[at].cpu(), mean[at].cpu(), rstd[at].cpu())
    assert_close(dx[at], want[0][0], 48 * U * want[0][1] + half_ulp(want[0][0], BF16) * 1.01, "dx")
    d, u = dy.double(), (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    for got, terms, name in ((dw, d * u, "dw"), (db, d, "db")):
        # Rows are added in runs of at most rows / 32768, their sums by 512 and less.
        bound = (600 + rows / 32768) * U * terms.abs().sum(0)
        assert_close(got, terms.sum(0).cpu(), bound.cpu(), name)


@pytest.mark.parametrize("xt", [F32, F16])
def test_one_very_long_row(xt):
    import paper_1903_06934_amd as m
    n = 50_000_001
    x = (1 + torch.randn(1, n, generator=_cuda(6), device="cuda")).to(xt)
    f = x.double()
    y, mean, rstd = m.layernorm_fwd(x)
    rmean = f.mean()
    rvar = ((f - rmean) ** 2).mean()
    rrstd = 1 / torch.sqrt(rvar + 1e-5)
    # A thread merges up to n / 64 / 1024 packs one by one.
    k = (64 + 4 * n / 65536) * U
    size = float(f.abs().mean())
    assert abs(float(mean - rmean)) <= k * size
    assert abs(float(rstd - rrstd)) <= float(rrstd) * (k + (k * size * float(rrstd)) ** 2)
    ry = (f - mean.double()) * rstd.double()
    bound = 4 * U * (ry.abs() + float(rstd) * f.abs()) + half_ulp(ry, xt) * 1.01
    assert bool(((y.double() - ry).abs() <= bound).all())
    dx, dw, db = m.layernorm_bwd(y, x, mean, rstd)
    assert torch.equal(db, y.float()[0])
    g, u = y.double(), ry
    s1, s2 = g.mean(), (g * u).mean()
    rdx = float(rstd) * (g - s1 - u * s2)
    bound = k * float(rstd) * (g.abs() + 1 + u.abs()) + half_ulp(rdx, xt) * 1.01
    assert bool(((dx.double() - rdx).abs() <= bound).all())

    t = torch.tensor([n - 1], device="cuda")
    out = m.logprob_fwd(x, t, top=10)
    lse = torch.logsumexp(f[0], 0)
    tol = (64 + n / 65536 / 4) * U * (3 + math.log(n))
    assert abs(float(out.lse - lse)) <= tol
    assert abs(float(out.logp - (f[0, n - 1] - lse))) <= tol
    order = torch.sort(f[0], descending=True, stable=True).indices[:10]
    assert torch.equal(out.top_index[0], order)
    dz = m.logprob_bwd(x, out.stats, t, torch.ones(1, device="cuda"))
    rz = -torch.exp(f - out.stats[0, 0].double() - out.stats[0, 1].double())
    rz[0, n - 1] += 1
    bound = 200 * U * rz.abs() + half_ulp(rz, xt) * 1.01 + 1e-37
    assert bool(((dz.double() - rz).abs() <= bound).all())


def test_clip_past_31_bits():
    import paper_1903_06934_amd as m
    n = (1 << 31) + 12345
    g = torch.full((n,), 0.5, dtype=F16, device="cuda")
    g[-3:] = 4.0
    norm = m.grad_clip([g], 100.0)
    want = math.sqrt(0.25 * (n - 3) + 48)
    assert abs(float(norm) / want - 1) < 1e-6
    f = 100.0 / want
    for at, v in ((0, 0.5), (1 << 30, 0.5), (n - 4, 0.5), (n - 1, 4.0)):
        assert abs(float(g[at]) - v * f) <= 2.0 ** -11 * v * f + 2.0 ** -25
    assert float(g[:n - 3].min()) == float(g[:n - 3].max())
