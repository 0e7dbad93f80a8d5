"""Launch rules of include/mistep.h's calls that only large ones reach, each against its
other side and the plain 64-bit forms (step_ref.py): loads that leave nothing in the caches
(more than 100 MB of whole cache lines), and sequences of many chunks that are joined by
several lanes in a launch of their own."""
import pytest
import torch

import step_ref as ref
import train_ref
from test_gpu_step import SEED, check_pairs, check_policy, gen, make_pairs, make_policy, ulp
from test_gpu_train import norm_terms
from train_ref import U, assert_close

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NUM = dict(p=0.3, seed=SEED, layer=2, step=5)


def rand(g, rows, cols, xt, gap=0):
    """Rows inside wider ones where there is a gap."""
    wide = torch.randn(rows, cols + gap, generator=g, device="cuda", dtype=torch.float32).to(xt)
    return wide[:, :cols]


def apart(t):
    """A copy whose rows share cache lines."""
    wide = torch.zeros(t.shape[0], t.shape[1] + 1, dtype=t.dtype, device="cuda")
    v = wide[:, :-1]
    v.copy_(t)
    return v


def samples(rows, cols):
    for r in (0, 1, rows // 2, rows - 1):
        yield r, ref.kept(range(r * cols, (r + 1) * cols), 0.3, SEED, 2, 5)[None]


@pytest.mark.parametrize("gap", [0, 64])
@pytest.mark.parametrize("rows,cols,xt,residual", [
    (13001, 4096, BF16, False), (6601, 4096, F16, True), (6601, 4096, F32, False),
    (1701, 8000, F32, True)])
def test_streamed_dropout(rows, cols, xt, residual, gap):
    import paper_1903_06934_amd as m
    assert rows * cols * xt.itemsize * (1 + residual) > 100 << 20
    g = torch.Generator(device="cuda").manual_seed(rows)
    x = rand(g, rows, cols, xt, gap)
    res = rand(g, rows, cols, xt) if residual else None
    assert x.data_ptr() % 128 == 0 and x.stride(0) * xt.itemsize % 128 == 0
    y = m.dropout_fwd(x, residual=res, **NUM)
    assert torch.equal(y, m.dropout_fwd(apart(x), residual=res, **NUM))
    for r, keep in samples(rows, cols):
        want, size = ref.dropout(x[r:r + 1].cpu(), keep, 0.3,
                                 res[r:r + 1].cpu() if residual else None)
        assert_close(y[r:r + 1], want, U * size + ulp(want, xt), r)
    if residual:
        assert m.dropout_fwd(x, residual=res, y=res, **NUM) is res and torch.equal(res, y)
    else:
        assert torch.equal(m.dropout_bwd(x, **NUM), y)


@pytest.mark.parametrize("rows,cols,xt", [(13001, 4096, BF16), (6601, 4096, F32), (53001, 1024, F16),
                                          (27001, 2048, BF16), (6701, 8192, F16)])
def test_streamed_residual_norm(rows, cols, xt):
    import paper_1903_06934_amd as m
    assert rows * cols * xt.itemsize > 100 << 20
    g = torch.Generator(device="cuda").manual_seed(cols)
    x, res, dy, dt = (rand(g, rows, cols, xt) for _ in range(4))
    w, b = 1 + 0.3 * rand(g, 1, cols, F32)[0], rand(g, 1, cols, F32)[0]
    keep_res = res.clone()
    out = m.residual_norm_fwd(x, res, w, b, total=res, **NUM)
    other = m.residual_norm_fwd(apart(x), keep_res, w, b, **NUM)
    for p, q in zip(out, other):
        assert torch.equal(p, q)
    back = m.residual_norm_bwd(dy, out.total, out.mean, out.rstd, w, dt, **NUM)
    other = m.residual_norm_bwd(apart(dy), out.total, out.mean, out.rstd, w, dt, **NUM)
    for p, q in zip(back, other):
        assert torch.equal(p, q)
    k = norm_terms(cols) * U
    for r, keep in samples(rows, cols):
        at = lambda t: t[r:r + 1].cpu()
        want, size = ref.dropout(at(x), keep, 0.3, at(keep_res))
        assert_close(at(out.total), want, U * size + ulp(want, xt), f"total {r}")
        ry, rmean, _, nsize, msize = train_ref.layernorm_fwd(at(out.total), w.cpu(), b.cpu())
        assert_close(at(out.mean), rmean, k * msize, f"mean {r}")
        assert_close(at(out.y), ry, 2 * k * nsize + ulp(ry, xt), f"y {r}")
        (dn, nsize), _, _ = train_ref.layernorm_bwd(at(dy), at(out.total), at(out.mean),
                                                    at(out.rstd), w.cpu())
        rg = dn + at(dt).double()
        off = k * nsize + U * rg.abs()
        rx, _ = ref.dropout(rg, keep, 0.3)
        assert_close(at(back[1]), rg, off + ulp(rg, xt), f"dresidual {r}")
        assert_close(at(back[0]), rx, off * ref.scale_of(0.3) + 2 * U * rx.abs() + ulp(rx, xt),
                     f"dx {r}")


@pytest.mark.parametrize("pairs,length", [(33, 8300), (79, 15800)])
@pytest.mark.parametrize("masked", [0.0, 0.2])
def test_pairs_of_many_chunks(pairs, length, masked):
    """Sixteen lanes a pair in the launch over the pairs, one short sequence among them."""
    import paper_1903_06934_amd as m
    lengths = torch.full((2 * pairs,), length) + torch.arange(2 * pairs) % 7
    lengths[pairs // 2], lengths[pairs] = 3, 0
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)])
    n = int(starts[-1])
    d = dict(make_pairs(gen(n, 5), n, pairs, 0, masked), starts=starts)
    check_pairs(m, d, beta=0.1, smoothing=0.1, length_mean=True)
    if length < 10000:
        check_pairs(m, d, beta=0.002, form="squared")
        d = dict(make_policy(gen(n, 6), n, 2 * pairs, 0, 0.2), starts=starts)
        check_policy(m, d, True, "low", True, "sequences")
