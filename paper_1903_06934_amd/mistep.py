"""Python binding of more of the training step's operators (include/mistep.h):
dropout, the end of a residual branch, and the losses of fine-tuning by sampled
answers and by preferences, with their gradients.

Argument marshalling only, in the manner of mitrain.py: torch's current stream
and device, tensors of rows, outputs and workspaces allocated where they are left
out, ValueError and MiconvError, no autograd history.

Dropout's mask is a function of an element's index in the tensor, the seed (64
bits), the layer (32 bits: which of a program's dropouts) and the step (modulo
2^32), and is the same forward and backward, in any type and for any strides.  step
is a number, or a device tensor of one int64, which is read as the kernels run:
a captured graph's replays then see the numbers that the program writes there.
"""
from __future__ import annotations

import ctypes
import math
from typing import NamedTuple, Optional

from . import miconv, mitrain

_FUNCTIONS = ("dropout_fwd", "dropout_bwd", "residual_norm_fwd_workspace_size",
              "residual_norm_bwd_workspace_size", "residual_norm_fwd", "residual_norm_bwd",
              "policy_loss_workspace_size", "policy_loss", "preference_loss_workspace_size",
              "preference_loss")

_ext = None


def _binding():
    """The compiled binding, with the library's functions handed to it (raises if
    either has not been built)."""
    global _ext
    if _ext is None:
        ext = mitrain._binding()
        L = miconv.lib()
        ext.load_step([ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in _FUNCTIONS])
        _ext = ext
    return _ext


# -------------------------------------------------------------------- dropout
def dropout_fwd(x, p, seed, layer=0, step=0, residual=None, y=None):
    """y = residual + dropout(x) of x's type [..., cols] (residual None: 0): elements
    are dropped with probability p, to a multiple of 2^-16, and the others scaled so
    that the mean is kept.  y may be x or residual."""
    return _binding().dropout_fwd(x, p, seed, layer, step, residual, y)


def dropout_bwd(dy, p, seed, layer=0, step=0, dx=None):
    """dx from dy [..., cols], by the forward's p, seed, layer and step.  dx may be dy."""
    return _binding().dropout_bwd(dy, p, seed, layer, step, dx)


# ----------------------------------------------------------- residual branches
class ResidualNorm(NamedTuple):
    """residual_norm_fwd's results: total and y like the branch, mean and rstd [rows]."""
    total: object
    y: object
    mean: object
    rstd: object


def residual_norm_workspace(backward, x):
    """A workspace for residual_norm_bwd (backward true) or residual_norm_fwd on x, or
    None where none is needed."""
    return _binding().residual_norm_workspace(backward, x)


def residual_norm_fwd(x, residual, w=None, b=None, eps=1e-5, p=0.0, seed=0, layer=0, step=0,
                      total=None, y=None, mean=None, rstd=None, ws=None):
    """ResidualNorm of a branch's output x [..., cols] and the residual stream: total =
    residual + dropout(x), and the layer norm of total's rows, as layernorm_fwd
    gives it.  total may be residual."""
    return ResidualNorm(*_binding().residual_norm_fwd(x, residual, w, b, eps, p, seed, layer, step,
                                                      total, y, mean, rstd, ws))


def residual_norm_bwd(dy, total, mean, rstd, w=None, dtotal=None, p=0.0, seed=0, layer=0, step=0,
                      dx=None, dresidual=None, dw=None, db=None, with_input=True, with_weight=True,
                      with_bias=True, ws=None):
    """(dx, dresidual, dw, db) from dy [..., cols], the forward's total, mean and rstd,
    w, and what reaches total beside the norm (dtotal; None: nothing).  Where nothing is
    dropped and no dx is given, dx is dresidual.  dresidual may be dtotal; those
    switched off (with_input: dx and dresidual) are None."""
    return _binding().residual_norm_bwd(dy, total, mean, rstd, w, dtotal, p, seed, layer, step, dx,
                                        dresidual, dw, db, with_input, with_weight, with_bias, ws)


# --------------------------------------------------------------------- losses
_KL = {"linear": 0, "square": 1, "low": 2}
_MEAN = {"tokens": 0, "sequences": 1}
_FORM = {"sigmoid": 0, "hinge": 1, "squared": 2}


def _choice(value, choices, name):
    try:
        return choices[value]
    except (KeyError, TypeError):
        raise ValueError(f"{name} must be one of {', '.join(choices)}") from None


class PolicyLoss(NamedTuple):
    """policy_loss's results: stats [6] and the gradients, like logp (None where not asked
    for).  The properties are views of stats' elements."""
    stats: object
    dlogp: Optional[object]
    dentropy: Optional[object]

    loss = property(lambda self: self.stats[0])
    surrogate = property(lambda self: self.stats[1])
    kl = property(lambda self: self.stats[2])
    entropy = property(lambda self: self.stats[3])
    ratio = property(lambda self: self.stats[4])
    clipped = property(lambda self: self.stats[5])


def policy_workspace(logp, starts=None):
    """A workspace for policy_loss on these tokens, or None where none is needed."""
    return _binding().policy_workspace(logp, starts)


def policy_loss(logp, old_logp, advantages, by_sequence=False, ref_logp=None, entropy=None,
                mask=None, starts=None, clip_low=0.2, clip_high=0.2, dual_clip=math.inf, kl="low",
                kl_weight=0.0, entropy_weight=0.0, mean="tokens", scale=1.0, with_grad=True,
                stats=None, dlogp=None, dentropy=None, ws=None):
    """PolicyLoss of sampled tokens: the clipped policy loss, plus kl_weight times the
    divergence from ref_logp (kl: linear, square or low), minus entropy_weight times the
    entropy.  logp, old_logp, ref_logp and entropy are float32 tensors of as many elements,
    sequence after sequence; starts [sequences + 1] (int64; None: one sequence) says where
    each begins and the last one ends; advantages are of the tokens, or (by_sequence) of
    the sequences; tokens whose mask (bool or uint8) is 0, or that no sequence has, do not
    count.  mean: over the tokens, or over the sequences' means, or a number that the
    tokens' sum is divided by.  The gradients, of loss times scale, are what logprob_bwd
    takes; dentropy where entropy is given."""
    if isinstance(mean, str):
        form, count = _choice(mean, _MEAN, "mean"), 1.0
    else:
        form, count = 2, float(mean)
    return PolicyLoss(*_binding().policy_loss(
        logp, old_logp, advantages, by_sequence, ref_logp, entropy, mask, starts, clip_low,
        clip_high, dual_clip, _choice(kl, _KL, "kl"), kl_weight, entropy_weight, form, count, scale,
        with_grad, stats, dlogp, dentropy, ws))


class PreferenceLoss(NamedTuple):
    """preference_loss's results: stats [5], the sequences' rewards [2 pairs], and the
    gradient, like logp (None where not asked for).  The properties are views of stats'
    elements: means over the pairs."""
    stats: object
    rewards: object
    dlogp: Optional[object]

    loss = property(lambda self: self.stats[0])
    gap = property(lambda self: self.stats[1])
    accuracy = property(lambda self: self.stats[2])
    chosen_reward = property(lambda self: self.stats[3])
    rejected_reward = property(lambda self: self.stats[4])


def preference_workspace(logp, starts):
    """A workspace for preference_loss on these tokens, or None where none is needed."""
    return _binding().preference_workspace(logp, starts)


def preference_loss(logp, ref_logp, starts, beta, form="sigmoid", smoothing=0.0, margin=0.0,
                    length_mean=False, mask=None, scale=1.0, with_grad=True, stats=None,
                    rewards=None, dlogp=None, ws=None):
    """PreferenceLoss of pairs of sequences: of 2 pairs sequences the first half are
    preferred to the second, one by one.  logp and ref_logp (float32; ref_logp may be
    None), starts [2 pairs + 1] and mask are as for policy_loss.  A sequence's reward is
    beta times the sum (length_mean: the mean) of logp - ref_logp; form: sigmoid (with
    label smoothing), hinge or squared, of the rewards' gap less margin.  dlogp is the
    gradient of the mean loss times scale."""
    return PreferenceLoss(*_binding().preference_loss(
        logp, ref_logp, starts, beta, _choice(form, _FORM, "form"), smoothing, margin, length_mean,
        mask, scale, with_grad, stats, rewards, dlogp, ws))
