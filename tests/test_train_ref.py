"""Pins of the plain 64-bit operators of train_ref.py: gradients against central
differences, closed forms and special rows."""
import math

import pytest
import torch

import train_ref as ref

INF = math.inf


def _rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def test_layernorm_closed_forms():
    y, mean, rstd, _, _ = ref.layernorm_fwd(torch.tensor([[1.0, 3.0], [-2.0, -2.0]]), eps=0.25)
    assert mean.tolist() == [2.0, -2.0]
    assert rstd.tolist() == [1 / math.sqrt(1.25), 2.0]
    assert torch.allclose(y[0], torch.tensor([-1.0, 1.0], dtype=torch.float64) / math.sqrt(1.25))
    assert y[1].tolist() == [0.0, 0.0]
    x, w, b = _rand(1, 3, 7), _rand(2, 7), _rand(3, 7)
    y = ref.layernorm_fwd(x, w, b)[0]
    assert torch.allclose(y, torch.nn.functional.layer_norm(x, (7,), w, b, 1e-5), atol=1e-13)


def test_layernorm_gradient_by_differences():
    rows, cols, h = 3, 5, 1e-5
    x, dy, w, b = _rand(4, rows, cols), _rand(5, rows, cols), _rand(6, cols), _rand(7, cols)
    _, mean, rstd, _, _ = ref.layernorm_fwd(x, w, b)
    (dx, _), (dw, _), (db, _) = ref.layernorm_bwd(dy, x, mean, rstd, w)

    def loss():
        return float((ref.layernorm_fwd(x, w, b)[0] * dy).sum())

    for t, grad in ((x, dx), (w, dw), (b, db)):
        flat, g = t.view(-1), grad.reshape(-1)
        for i in range(flat.numel()):
            keep = float(flat[i])
            flat[i] = keep + h
            up = loss()
            flat[i] = keep - h
            down = loss()
            flat[i] = keep
            assert abs((up - down) / (2 * h) - float(g[i])) < 1e-8


@pytest.mark.parametrize("scale", [1.0, 0.5])
def test_logprob_gradient_by_differences(scale):
    rows, vocab, h = 4, 6, 1e-5
    z = _rand(8, rows, vocab) * 2
    z[1, 3] = -INF
    targets = torch.tensor([2, 0, -1, 5])
    dlogp, dent = _rand(9, rows), _rand(10, rows)
    out = ref.logprob_fwd(z, targets, scale=scale)
    dz, _ = ref.logprob_bwd(z, targets, scale, out["stats"], dlogp, out["entropy"], dent)

    def loss():
        o = ref.logprob_fwd(z, targets, scale=scale)
        return float((o["logp"] * dlogp + o["entropy"] * dent).sum())

    for r in range(rows):
        for j in range(vocab):
            if z[r, j] == -INF:
                assert dz[r, j] == 0
                continue
            keep = float(z[r, j])
            z[r, j] = keep + h
            up = loss()
            z[r, j] = keep - h
            down = loss()
            z[r, j] = keep
            assert abs((up - down) / (2 * h) - float(dz[r, j])) < 1e-8


def test_logprob_special_rows():
    z = torch.tensor([[-INF, -INF, -INF], [0.0, -INF, 0.0], [math.nan, 1.0, 2.0],
                      [INF, 0.0, 1.0], [3.0, 3.0, 3.0]])
    t = torch.tensor([1, 2, 1, 1, 7])
    out = ref.logprob_fwd(z, t, top=2)
    assert out["lse"][0] == -INF and out["logp"][0] == -INF and out["entropy"][0] == 0
    assert out["top_index"].tolist() == [[0, 1], [0, 2], [2, 1], [0, 2], [0, 1]]
    assert abs(float(out["entropy"][1]) - math.log(2)) < 1e-15
    for r in (2, 3):
        for k in ("lse", "logp", "entropy"):
            assert torch.isnan(out[k][r])
    assert torch.isnan(out["logp"][4])
    dz, _ = ref.logprob_bwd(z, t, 1.0, out["stats"], torch.ones(5))
    assert dz[0].tolist() == [0, 0, 0] and torch.isnan(dz[2:]).all()


def test_clip_closed_forms():
    norm, out = ref.clip([torch.tensor([3.0]), torch.tensor([0.0, 4.0])], 1.0)
    assert norm == 5.0
    assert torch.allclose(out[1], torch.tensor([0.0, 0.8], dtype=torch.float64))
    assert ref.clip([torch.tensor([3.0])], 3.0)[1][0].tolist() == [3.0]
    assert ref.clip([], 1.0) == (0.0, [])


def test_half_ulp():
    v = torch.tensor([1.0, 1.5, 2.0, 0.0])
    assert ref.half_ulp(v, torch.float32).tolist() == [2.0 ** -24] * 2 + [2.0 ** -23, 2.0 ** -150]
    assert ref.half_ulp(v, torch.bfloat16)[0] == 2.0 ** -8
    assert ref.half_ulp(v, torch.float16)[0] == 2.0 ** -11
