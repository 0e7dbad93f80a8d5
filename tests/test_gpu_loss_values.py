"""The losses of fine-tuning on the GPU at values where 32 bits end or lose what matters,
against their plain 64-bit forms (step_ref.py).  Calls of one workgroup, and of chunks."""
import math

import pytest
import torch

import step_ref as ref
from test_gpu_step import call_policy, gen, make_policy, want_policy
from train_ref import INF, assert_close

pytestmark = pytest.mark.gpu

# 32 bits end between exp(88.72) and exp(88.73).
FAR = [88.7, 88.73, 89.0, 90.0, 95.0, 100.0, 138.0, 139.0, 1000.0, 1e38]


def one_far(tokens, key, value, adv):
    """Ordinary tokens, of which one has value as its log ratio (key "old") or as ref - logp
    (key "ref"), and the advantage adv."""
    d = make_policy(gen(tokens, 12), tokens, 2)
    i = tokens // 2 + 1
    d["logp"][i] = d["old"][i] = d["ref"][i] = 0.0
    d[key][i] = -value if key == "old" else value
    d["adv"][i] = adv
    return d, i


def assert_same(got, want, bound, what):
    """Within its bound where what is wanted is in 32 bits, else infinite."""
    got, want = got.double().cpu(), want.double()
    far = want.abs() > 2.0 ** 128
    assert torch.equal(got[far], want[far].sign() * INF), (what, got[far], want[far])
    assert_close(got[~far], want[~far], bound[~far], what)


@pytest.mark.parametrize("tokens", [64, 9000])
@pytest.mark.parametrize("value", FAR)
def test_ratios_past_32_bits(tokens, value):
    """Those of a gain are clipped, those of a loss infinite; none is NaN."""
    import paper_1903_06934_amd as m
    for adv in (1.0, -1.0):
        d, _ = one_far(tokens, "old", value, adv)
        out = call_policy(m, d, False, "", False, 1.0)
        (stats, sb), (g, gb), _ = want_policy(d, False, "", False, 1.0)
        assert_same(out.stats, stats, sb, f"stats {adv}")
        assert_same(out.dlogp, g, gb, f"dlogp {adv}")


@pytest.mark.parametrize("tokens", [64, 9000])
@pytest.mark.parametrize("value", FAR)
def test_divergences_past_32_bits(tokens, value):
    import paper_1903_06934_amd as m
    d, _ = one_far(tokens, "ref", value, 0.5)
    out = call_policy(m, d, False, "low", False, 1.0, kl_weight=1.0)
    (stats, sb), (g, gb), _ = want_policy(d, False, "low", False, 1.0, kl_weight=1.0)
    assert_same(out.stats, stats, sb, "stats")
    assert_same(out.dlogp, g, gb, "dlogp")
