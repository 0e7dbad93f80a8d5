"""Python binding of the training step's operators (include/mitrain.h): layer
norm, log probabilities of given tokens, the gradients' norm and clipping.

Argument marshalling only (in csrc/binding.cpp): kernels are enqueued on
torch's current stream, of the current HIP device.  Tensors are float32,
bfloat16 or float16 tensors on that device.  A tensor of rows has its rows'
elements in the last dimension, side by side; the dimensions before it may have
any strides that one row stride covers (a slice of a wider matrix's columns or
rows, say).  What is left out of the output and workspace arguments is
allocated.  ValueError: a tensor of another type, layout, size or device;
MiconvError: what the library refuses.

Autograd does not record the calls: results have no history, whether or not an
input requires a gradient.  A given tensor that a call writes counts as changed
in place, so that torch reports a backward pass that had saved it.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
from typing import NamedTuple, Optional

from . import miconv

BINDING = os.path.join(miconv.PKG, "_mitrain.so")
_FUNCTIONS = ("layernorm_fwd_workspace_size", "layernorm_bwd_workspace_size", "layernorm_fwd",
              "layernorm_bwd", "logprob_fwd_workspace_size", "logprob_fwd", "logprob_bwd",
              "grad_workspace_size", "grad_norm", "grad_clip")

_ext = None


def _raise(status, name):
    raise miconv.MiconvError(status, name)


def _binding():
    """The compiled binding, with the library's functions handed to it (raises if
    either has not been built)."""
    global _ext
    if _ext is None:
        L = miconv.lib()
        if not os.path.exists(BINDING):
            raise RuntimeError(f"{BINDING} is not built; run paper_1903_06934_amd.build.build()")
        spec = importlib.util.spec_from_file_location("_mitrain", BINDING)
        ext = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(ext)
        ext.load([ctypes.cast(getattr(L, n), ctypes.c_void_p).value for n in _FUNCTIONS], _raise)
        _ext = ext
    return _ext


# ---------------------------------------------------------------- layer norm
def layernorm_workspace(backward, x):
    """A workspace for layernorm_bwd (backward true) or layernorm_fwd on x, or
    None where none is needed."""
    return _binding().layernorm_workspace(backward, x)


def layernorm_fwd(x, w=None, b=None, eps=1e-5, y=None, mean=None, rstd=None, ws=None):
    """(y, mean, rstd): the layer norm of x's rows [..., cols], times w [cols], plus
    b [cols] (each may be None; of x's type, or float32), and the float32
    statistics [rows] that layernorm_bwd takes."""
    return _binding().layernorm_fwd(x, w, b, eps, y, mean, rstd, ws)


def layernorm_bwd(dy, x, mean, rstd, w=None, dx=None, dw=None, db=None, with_input=True,
                  with_weight=True, with_bias=True, ws=None):
    """(dx, dw, db) from dy and x [..., cols], the forward's mean and rstd [rows] and
    w [cols] (None: 1).  dw and db [cols] are of w's type (without w of dw's or
    db's, or float32); those switched off are None."""
    return _binding().layernorm_bwd(dy, x, mean, rstd, w, dx, dw, db, with_input, with_weight,
                                    with_bias, ws)


# --------------------------------------------------------- log probabilities
class LogProbs(NamedTuple):
    """logprob_fwd's results: float32 tensors of the rows' shape (stats [..., 2],
    top_logp [..., top], top_index the same in int64); None where not asked for."""
    logp: Optional[object]
    lse: object
    entropy: object
    stats: object
    top_logp: Optional[object]
    top_index: Optional[object]


def logprob_workspace(logits, top=0):
    """A workspace for logprob_fwd, or None where none is needed."""
    return _binding().logprob_workspace(logits, top)


def logprob_fwd(logits, targets=None, top=0, scale=1.0, ws=None, logp=None, lse=None,
                entropy=None, stats=None, top_logp=None, top_index=None):
    """LogProbs of the rows of logits [..., vocab] under softmax(scale * logits):
    the log probabilities of targets [...] (int64; negative: none given), the
    log of the softmax's sum, its entropy, the top (at most 64, or vocab where that
    is fewer) likeliest tokens, and the statistics that logprob_bwd takes.  Given
    results have as many elements as LogProbs states, side by side."""
    return LogProbs(*_binding().logprob_fwd(logits, targets, top, scale, logp, lse, entropy, stats,
                                            top_logp, top_index, ws))


def logprob_bwd(logits, stats, targets=None, dlogp=None, entropy=None, dentropy=None, scale=1.0,
                dlogits=None):
    """The gradient in the logits of (dlogp * logp + dentropy * entropy).sum(): from
    the forward's stats [..., 2] (and entropy, for dentropy), targets and dlogp
    [...], dentropy [...]; one of the two may be None.  dlogits may be logits."""
    return _binding().logprob_bwd(logits, stats, targets, dlogp, entropy, dentropy, scale, dlogits)


# ------------------------------------------------------------------ clipping
def grad_workspace(grads):
    """A workspace for grad_norm and grad_clip on gradients of these sizes, or None."""
    return _binding().grad_workspace(grads)


def grad_norm(grads, norm=None, ws=None):
    """norm [1] float32: the root of the sum of the squares of all gradients."""
    return _binding().grad_norm(grads, norm, ws)


def grad_clip(grads, max_norm, out=None, norm=None, ws=None):
    """Scales the gradients to a global norm of at most max_norm, in place or to
    the tensors of out; returns their norm before that, [1] float32."""
    return _binding().grad_clip(grads, max_norm, out, norm, ws)
