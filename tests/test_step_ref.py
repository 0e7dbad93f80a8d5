"""Pins of the plain 64-bit operators of step_ref.py: the generator's published
vectors, closed forms, gradients against central differences."""
import math

import numpy as np
import pytest
import torch

import step_ref as ref

F = 0xFFFFFFFF


def _rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
    ((F, F, F, F), (F, F), (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
    ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
     (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))])
def test_generator_known_answers(counter, key, want):
    """The known answers that the generator's authors publish for ten rounds."""
    assert tuple(ref.philox(counter, key)) == want


def test_kept_is_the_generator():
    seed, layer, step, p = (7 << 40) + 12345, 3, (1 << 32) + 9, 0.3
    e = np.array([0, 1, 7, 8, 13, 1 << 33, (1 << 36) + 5])
    got = ref.kept(e, p, seed, layer, step)
    for i, v in enumerate(e.tolist()):
        g = v >> 3
        w = ref.philox((g & F, g >> 32, 9, layer), (seed & F, seed >> 32))
        bits = w[(v & 7) // 2] >> 16 * (v & 1) & 0xFFFF
        assert bool(got[i]) == (bits >= 19661)


def test_dropout_closed_forms():
    assert ref.threshold(0.1) == 6554 and ref.threshold(2.0 ** -17) == 0
    assert ref.threshold(1.0) == 65536 and ref.scale_of(0.5) == 2.0
    share = float(ref.mask_of(300, 401, 0.3, 99).double().mean())
    # 120300 trials: five standard deviations.
    assert abs(share - (1 - 19661 / 65536)) < 5 * math.sqrt(0.21 / 120300)
    a, b = ref.mask_of(50, 64, 0.5, 1), ref.mask_of(50, 64, 0.5, 1, layer=1)
    assert not torch.equal(a, b) and torch.equal(a, ref.mask_of(25, 128, 0.5, 1).view(50, 64))


def test_policy_closed_forms():
    lp = torch.log(torch.tensor([1.5, 0.5, 1.0, 4.0, 0.5], dtype=torch.float64))
    old = torch.zeros(5)
    a = torch.tensor([2.0, -1.0, 3.0, -1.0, 1.0])
    (s, _), (g, _), _ = ref.policy(lp, old, a, dual=3.0, mean=1.0)
    # Clipped at 1.2, at 0.8, not, at the dual border, not.
    assert torch.allclose(s[1], torch.tensor(-2.4 + 0.8 - 3.0 + 3.0 - 0.5, dtype=torch.float64))
    assert g.tolist()[:2] == [0, 0] and g[3] == 0
    assert torch.allclose(g[[2, 4]], torch.tensor([-3.0, -0.5], dtype=torch.float64))
    assert s[5] == 3
    mask = torch.tensor([1, 0, 1, 1, 1])
    (s, _), _, _ = ref.policy(lp, old, a, mask=mask, starts=[0, 2, 2, 3, 4], mean="sequences")
    # Three sequences with one token each that counts; the last token is in none.
    assert torch.allclose(s[4], torch.tensor((1.5 + 1.0 + 4.0) / 3, dtype=torch.float64))


@pytest.mark.parametrize("kl", ["linear", "square", "low"])
@pytest.mark.parametrize("mean", ["tokens", "sequences", 7.0])
def test_policy_gradient_by_differences(kl, mean):
    n, h = 12, 1e-6
    lp, old, rf, ent = _rand(1, n) - 2, _rand(2, n) * 0.4, _rand(3, n) * 0.4, _rand(4, n).abs()
    old, rf = lp + old, lp + rf
    adv = _rand(5, 3)
    mask = torch.ones(n, dtype=torch.bool)
    mask[[0, 7]] = False
    args = dict(by_sequence=True, ref=rf, entropy=ent, mask=mask, starts=[0, 4, 5, 11], dual=2.0,
                kl=kl, kl_weight=0.3, entropy_weight=0.2, mean=mean)
    loss = lambda: float(ref.policy(lp, old, adv, **args)[0][0][0])
    _, (g, _), (gh, _) = ref.policy(lp, old, adv, **args)
    for t, grad in ((lp, g), (ent, gh)):
        for i in range(n):
            keep = float(t[i])
            t[i] = keep + h
            up = loss()
            t[i] = keep - h
            down = loss()
            t[i] = keep
            assert abs((up - down) / (2 * h) - float(grad[i])) < 1e-7


def test_preference_closed_forms():
    lp = torch.tensor([1.0, 2.0, 0.5, 0.5])
    (s, _), (r, _), (g, _) = ref.preference(lp, None, [0, 2, 4], 0.5)
    assert r.tolist() == [1.5, 0.5]
    assert abs(float(s[0]) - math.log1p(math.exp(-1))) < 1e-12
    assert torch.allclose(g, 0.5 / (1 + math.e) * torch.tensor([-1, -1, 1, 1], dtype=torch.float64))
    (s, _), (r, _), _ = ref.preference(lp, None, [0, 2, 2, 4, 4], 0.5, mask=torch.zeros(4))
    assert s.tolist() == [0] * 5 and r.tolist() == [0] * 4


@pytest.mark.parametrize("form", ["sigmoid", "hinge", "squared"])
@pytest.mark.parametrize("length_mean", [False, True])
def test_preference_gradient_by_differences(form, length_mean):
    n, h = 15, 1e-6
    lp, rf = _rand(6, n) - 1, _rand(7, n) - 1
    mask = torch.ones(n, dtype=torch.bool)
    mask[[1, 9, 10]] = False
    args = dict(form=form, smoothing=0.1, margin=0.2, length_mean=length_mean, mask=mask)
    starts = [0, 3, 6, 9, 11, 11, 14]  # the second of the second pair is empty
    loss = lambda: float(ref.preference(lp, rf, starts, 0.7, **args)[0][0][0])
    _, _, (g, _) = ref.preference(lp, rf, starts, 0.7, **args)
    for i in range(n):
        keep = float(lp[i])
        lp[i] = keep + h
        up = loss()
        lp[i] = keep - h
        down = loss()
        lp[i] = keep
        assert abs((up - down) / (2 * h) - float(g[i])) < 1e-7
