"""The losses of fine-tuning on the GPU at values where 32 bits end or lose what matters,
against their plain 64-bit forms (step_ref.py).  Calls of one workgroup, and of chunks."""
import math

import pytest
import torch

import step_ref as ref
from test_gpu_step import call_policy, gen, make_policy, want_policy
from train_ref import INF, U, assert_close, half_ulp

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


@pytest.mark.parametrize("tokens", [64, 9000])
@pytest.mark.parametrize("value", [0.5, 100.0, INF])
def test_no_advantage(tokens, value):
    """An advantage of 0, of a token or of its whole sequence, gives 0 to the loss and its
    gradient however large the ratio is."""
    import paper_1903_06934_amd as m
    for by, high in ((False, 0.3), (True, 0.3), (True, INF)):
        d, i = one_far(tokens, "old", value, 0.0)
        d["adv"][:5], d["seq_adv"][int(i >= d["starts"][1])] = 0.0, 0.0
        zero = d["adv"] == 0
        if by:
            s = int(i >= d["starts"][1])
            zero = torch.arange(tokens) >= d["starts"][1] if s else torch.arange(tokens) < d["starts"][1]
        out = m.policy_loss(d["logp"].cuda(), d["old"].cuda(), d["seq_adv" if by else "adv"].cuda(),
                            by_sequence=by, starts=d["starts"].cuda(), clip_high=high)
        # By the definition, with a ratio that the 64-bit form can multiply by 0.
        d["old"][i] = max(float(d["old"][i]), -100.0)
        (stats, sb), (g, gb), _ = ref.policy(d["logp"], d["old"], d["seq_adv" if by else "adv"], by,
                                             starts=d["starts"], high=high)
        assert_same(out.stats, stats, sb, "stats")
        assert_same(out.dlogp, g, gb, "dlogp")
        assert bool((out.dlogp.cpu()[zero] == 0).all())


def test_no_advantage_and_no_number():
    import paper_1903_06934_amd as m
    lp = torch.tensor([0.0, math.nan, -1.0], device="cuda")
    out = m.policy_loss(lp, torch.zeros(3, device="cuda"), torch.zeros(3, device="cuda"))
    assert torch.isnan(out.dlogp).tolist() == [False, True, False] and torch.isnan(out.loss)


@pytest.mark.parametrize("tokens", [64, 9000])
@pytest.mark.parametrize("kl", ["linear", "square", "low"])
def test_divergence_of_an_impossible_token(tokens, kl):
    """A token that has no probability now, or none under the reference: the limits of the
    divergence and of its slope."""
    import paper_1903_06934_amd as m
    for now in (True, False):
        d, i = one_far(tokens, "ref", 0.0, 1.0)
        d["logp" if now else "ref"][i] = -INF  # x is +inf, or -inf
        out = call_policy(m, d, False, kl, False, 1.0, kl_weight=1.0)
        assert out.kl == (INF if kl != "linear" or not now else -INF)
        assert out.loss == out.kl
        want = {"linear": 1.0, "square": -INF if now else INF, "low": -INF if now else 1.0}[kl]
        # Beside it the surrogate's slope: 0 of a ratio of 0, -1 of a ratio of 1.
        assert float(out.dlogp[i]) == want - (0.0 if now else 1.0)
        assert int(torch.isfinite(out.dlogp).sum()) >= tokens - 1


def test_results_of_one_workgroup_together():
    """The loss is that of the same call's sums, call after call on changing tokens."""
    import paper_1903_06934_amd as m
    sets = [make_policy(gen(n, 14), n, 3) for n in (5, 300, 4096, 8192)]
    for _ in range(20):
        for d in sets:
            s = call_policy(m, d, True, "low", True, "sequences").stats.double().tolist()
            size = abs(s[1]) + 0.07 * abs(s[2]) + 0.02 * abs(s[3])
            # Each statistic and the two weights are rounded once, the loss too.
            assert abs(s[0] - (s[1] + 0.07 * s[2] - 0.02 * s[3])) <= 3 * U * size


def policy_of(adv, **kw):
    """The call on tokens whose ratio is 1: their surrogates are -adv."""
    import paper_1903_06934_amd as m
    lp = torch.zeros(len(adv), device="cuda")
    return m.policy_loss(lp, lp, adv.cuda(), **kw)


@pytest.mark.parametrize("tokens", [8, 4000, 8000, 9000])
def test_sums_hold_what_32_bits_lose(tokens):
    """Neighbours that cancel each other leave what lies between them; sums past 32 bits
    whose mean is within them."""
    adv = torch.zeros(tokens)
    adv[:3] = torch.tensor([1.0, 2.0 ** -30, -1.0])
    adv[4:7] = torch.tensor([-1.0, 2.0 ** -31, 1.0])
    out = policy_of(adv, mean=1.0)
    assert float(out.loss) == float(out.surrogate) == -(2.0 ** -30 + 2.0 ** -31)
    big = torch.full((tokens,), 3e38)
    for kw in ({}, {"starts": torch.tensor([0, tokens // 3, tokens]).cuda(), "mean": "sequences"}):
        out = policy_of(big, **kw)
        # The sum's mean in 64 bits, rounded.
        want = -big[:1].double()
        assert_close(out.stats[:2], want.expand(2), U * want.abs(), "stats")
    e = torch.tensor([1.0, 2.0 ** -30, -1.0, 0.0]).repeat(tokens // 4).cuda()
    out = policy_of(torch.zeros(tokens), entropy=e, mean=float(tokens // 4))
    assert float(out.entropy) == 2.0 ** -30


@pytest.mark.parametrize("tokens,seqs", [(4000, 40), (8000, 33), (50000, 300), (200000, 7)])
def test_gradients_are_rounded_once(tokens, seqs):
    """Of slopes that 32 bits hold: at the nearest number of 32 bits, but for what the
    weights' 64 bits decide."""
    import paper_1903_06934_amd as m
    d = make_policy(gen(tokens, 15), tokens, seqs)
    lp, ent, starts = torch.zeros(tokens), d["entropy"], d["starts"]
    length = (starts[1:] - starts[:-1]).double()
    seq = torch.searchsorted(starts[1:].contiguous(), torch.arange(tokens), right=True)
    each = {"sequences": 1 / length[seq] / (length > 0).sum(), "tokens": 1 / lp.new_full((1,), tokens,
            dtype=torch.float64).expand(tokens)}
    for mean, by in (("sequences", False), ("sequences", True), ("tokens", True)):
        adv = d["seq_adv" if by else "adv"]
        out = m.policy_loss(lp.cuda(), lp.cuda(), adv.cuda(), by_sequence=by, entropy=ent.cuda(),
                            starts=starts.cuda(), entropy_weight=0.25, mean=mean, scale=3.0)
        g = -3 * (adv[seq] if by else adv).double() * each[mean]
        for got, want in ((out.dlogp, g), (out.dentropy, -0.75 * each[mean])):
            # Some five roundings of 64 bits.
            bound = half_ulp(want, torch.float32) + 2.0 ** -50 * want.abs()
            assert_close(got, want, bound, f"{mean} {by}")


@pytest.mark.parametrize("tokens", [8, 4000, 8000, 9000, 300000])
def test_log_ratios_hold_what_32_bits_lose(tokens):
    """Differences of log probabilities that 32 bits cannot hold, which cancel in the sum."""
    import paper_1903_06934_amd as m
    lp, lr = torch.zeros(tokens), torch.zeros(tokens)
    half = tokens // 2
    lp[:2], lr[0] = torch.tensor([1.0, -1.0]), 2.0 ** -30
    lp[half:half + 2], lr[half + 1] = torch.tensor([-1.0, 1.0]), -2.0 ** -28
    starts = torch.tensor([0, half, tokens])
    out = m.preference_loss(lp.cuda(), lr.cuda(), starts.cuda(), 1.0)
    assert out.rewards.tolist() == [-2.0 ** -30, 2.0 ** -28]
    assert float(out.gap) == -2.0 ** -30 - 2.0 ** -28
