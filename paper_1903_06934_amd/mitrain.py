"""ctypes binding of the training step's operators (include/mitrain.h): layer
norm, log probabilities of given tokens, the gradients' norm and clipping.

Argument marshalling only, as in miconv.py: kernels are enqueued on torch's
current stream, of the current HIP device.  Tensors are float32, bfloat16 or
float16 device tensors.  A tensor of rows has its rows' elements in the last
dimension, side by side; the dimensions before it may have any strides that
one row stride covers (a slice of a wider matrix's columns or rows, say).
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

from .miconv import _call, _ptr, _stream, _workspace, lib

_types = {}


def _type(t, name):
    if not _types:
        import torch
        _types.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    if t.dtype not in _types or t.device.type != "cuda":
        raise ValueError(f"{name} must be a float32, bfloat16 or float16 device tensor")
    return _types[t.dtype]


def _rows(t, name):
    """(rows, columns, row stride) of a tensor of rows."""
    shape, strides = t.shape, t.stride()
    if not shape:
        raise ValueError(f"{name} must have at least one dimension")
    cols = shape[-1]
    rows = 1
    for n in shape[:-1]:
        rows *= n
    if cols > 1 and strides[-1] != 1:
        raise ValueError(f"the elements of {name}'s rows must lie side by side")
    ld, span = cols, None  # span: the stride that the next outer dimension needs
    if rows > 1:
        for n, st in zip(reversed(shape[:-1]), reversed(strides[:-1])):
            if n == 1:
                continue
            if span is None:
                ld = span = st
            elif st != span:
                raise ValueError(f"one stride must cover {name}'s rows")
            span *= n
        if ld < cols:
            raise ValueError(f"{name}'s rows must not overlap")
    return rows, cols, ld


def _vector(t, name, n, dtype=None):
    """Checks a contiguous device vector of n elements (of dtype)."""
    if t is None:
        return
    if (t.numel() != n or not t.is_contiguous() or t.device.type != "cuda"
            or (dtype is not None and t.dtype != dtype)):
        raise ValueError(f"{name} must be a contiguous device tensor of {n} elements"
                         + (f" of {dtype}" if dtype is not None else ""))


def _like(t, name, x, rows, cols):
    """The row stride of t, which has x's type, rows and columns."""
    r, c, ld = _rows(t, name)
    if t.dtype != x.dtype or t.device.type != "cuda" or (r, c) != (rows, cols):
        raise ValueError(f"{name} must be a device tensor of {rows} x {cols} elements of {x.dtype}")
    return ld


def _size(ws):
    return 0 if ws is None else ws.numel() * ws.element_size()


# ---------------------------------------------------------------- layer norm
def layernorm_workspace(backward, x):
    """A workspace for layernorm_bwd (backward true) or layernorm_fwd on x, or
    None where none is needed."""
    rows, cols, _ = _rows(x, "x")
    L = lib()
    size = L.layernorm_bwd_workspace_size if backward else L.layernorm_fwd_workspace_size
    return _workspace(int(size(_type(x, "x"), rows, cols)), x.device)


def layernorm_fwd(x, w=None, b=None, eps=1e-5, y=None, mean=None, rstd=None, ws=None):
    """(y, mean, rstd): the layer norm of x's rows [..., cols], times w [cols], plus
    b [cols] (each may be None; of x's type, or float32), and the float32
    statistics [rows] that layernorm_bwd takes."""
    import torch
    rows, cols, ldx = _rows(x, "x")
    xtype = _type(x, "x")
    wtype = xtype
    for t, n in ((w, "w"), (b, "b")):
        if t is not None:
            _vector(t, n, cols)
            wtype = _type(t, n)
    if w is not None and b is not None and w.dtype != b.dtype:
        raise ValueError("w and b must be of one type")
    if y is None:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    ldy = _like(y, "y", x, rows, cols)
    if mean is None:
        mean = torch.empty(rows, dtype=torch.float32, device=x.device)
    if rstd is None:
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
    _vector(mean, "mean", rows, torch.float32)
    _vector(rstd, "rstd", rows, torch.float32)
    L = lib()
    if ws is None:
        ws = _workspace(int(L.layernorm_fwd_workspace_size(xtype, rows, cols)), x.device)
    _call(L.layernorm_fwd, "layernorm_fwd", xtype, wtype, rows, cols, _ptr(x), ldx, _ptr(w),
          _ptr(b), eps, _ptr(y), ldy, _ptr(mean), _ptr(rstd), _ptr(ws), _size(ws), _stream())
    return y, mean, rstd


def layernorm_bwd(dy, x, mean, rstd, w=None, dx=None, dw=None, db=None, with_input=True,
                  with_weight=True, with_bias=True, ws=None):
    """(dx, dw, db) from dy and x [..., cols], the forward's mean and rstd [rows] and
    w [cols] (None: 1).  dw and db [cols] are of w's type (without w of dw's or
    db's, or float32); those switched off are None."""
    import torch
    rows, cols, ldx = _rows(x, "x")
    xtype = _type(x, "x")
    lddy = _like(dy, "dy", x, rows, cols)
    _vector(mean, "mean", rows, torch.float32)
    _vector(rstd, "rstd", rows, torch.float32)
    given = next((t for t in (w, dw, db) if t is not None), None)
    wdtype = torch.float32 if given is None else given.dtype
    wtype = 0 if given is None else _type(given, "w")
    if not with_input:
        dx = None
    elif dx is None:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    lddx = cols if dx is None else _like(dx, "dx", x, rows, cols)
    if not with_weight:
        dw = None
    elif dw is None:
        dw = torch.empty(cols, dtype=wdtype, device=x.device)
    if not with_bias:
        db = None
    elif db is None:
        db = torch.empty(cols, dtype=wdtype, device=x.device)
    for t, n in ((w, "w"), (dw, "dw"), (db, "db")):
        _vector(t, n, cols, wdtype)
    L = lib()
    if ws is None:
        ws = _workspace(int(L.layernorm_bwd_workspace_size(xtype, rows, cols)), x.device)
    _call(L.layernorm_bwd, "layernorm_bwd", xtype, wtype, rows, cols, _ptr(dy), lddy, _ptr(x),
          ldx, _ptr(mean), _ptr(rstd), _ptr(w), _ptr(dx), lddx, _ptr(dw), _ptr(db), _ptr(ws),
          _size(ws), _stream())
    return dx, dw, db


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
    rows, vocab, _ = _rows(logits, "logits")
    return _workspace(int(lib().logprob_fwd_workspace_size(_type(logits, "logits"), rows, vocab,
                                                           top)), logits.device)


def logprob_fwd(logits, targets=None, top=0, scale=1.0, ws=None):
    """LogProbs of the rows of logits [..., vocab] under softmax(scale * logits):
    the log probabilities of targets [...] (int64; negative: none given), the
    log of the softmax's sum, its entropy, the top likeliest tokens, and the
    statistics that logprob_bwd takes."""
    import torch
    rows, vocab, ld = _rows(logits, "logits")
    xtype = _type(logits, "logits")
    shape, device = logits.shape[:-1], logits.device
    _vector(targets, "targets", rows, torch.int64)
    # One buffer for the rows' float32 results.
    out = torch.empty((5 * rows,), dtype=torch.float32, device=device)
    lse, entropy = out[:rows].view(shape), out[rows:2 * rows].view(shape)
    stats = out[2 * rows:4 * rows].view(tuple(shape) + (2,))
    logp = None if targets is None else out[4 * rows:].view(shape)
    top_logp = top_index = None
    if top:
        top_logp = torch.empty(tuple(shape) + (top,), dtype=torch.float32, device=device)
        top_index = torch.empty(tuple(shape) + (top,), dtype=torch.int64, device=device)
    L = lib()
    if ws is None:
        ws = _workspace(int(L.logprob_fwd_workspace_size(xtype, rows, vocab, top)), device)
    _call(L.logprob_fwd, "logprob_fwd", xtype, rows, vocab, _ptr(logits), ld, _ptr(targets),
          scale, top, _ptr(logp), _ptr(lse), _ptr(entropy), _ptr(stats), _ptr(top_logp), _ptr(top_index),
          _ptr(ws), _size(ws), _stream())
    return LogProbs(logp, lse, entropy, stats, top_logp, top_index)


def logprob_bwd(logits, stats, targets=None, dlogp=None, entropy=None, dentropy=None, scale=1.0,
                dlogits=None):
    """The gradient in the logits of (dlogp * logp + dentropy * entropy).sum(): from
    the forward's stats [..., 2] (and entropy, for dentropy), targets and dlogp [...],
    dentropy [...]; one of the two may be None.  dlogits may be logits."""
    import torch
    rows, vocab, ld = _rows(logits, "logits")
    xtype = _type(logits, "logits")
    _vector(targets, "targets", rows, torch.int64)
    _vector(stats, "stats", 2 * rows, torch.float32)
    for t, n in ((dlogp, "dlogp"), (entropy, "entropy"), (dentropy, "dentropy")):
        _vector(t, n, rows, torch.float32)
    if dlogits is None:
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    ldd = _like(dlogits, "dlogits", logits, rows, vocab)
    _call(lib().logprob_bwd, "logprob_bwd", xtype, rows, vocab, _ptr(logits), ld, _ptr(targets),
          scale, _ptr(stats), _ptr(dlogp), _ptr(entropy), _ptr(dentropy), _ptr(dlogits), ldd,
          _stream())
    return dlogits


# ------------------------------------------------------------------ clipping
def _list(grads):
    """(pointers, counts, types) of a list of gradients, as ctypes arrays."""
    n = len(grads)
    for g in grads:
        if not g.is_contiguous():
            raise ValueError("gradients must be contiguous")
    return ((ctypes.c_void_p * n)(*[g.data_ptr() for g in grads]),
            (ctypes.c_longlong * n)(*[g.numel() for g in grads]),
            (ctypes.c_int * n)(*[_type(g, "a gradient") for g in grads]))


def _grad_ws(count, types, device):
    return _workspace(int(lib().grad_workspace_size(len(count), count, types)), device)


def _device(grads):
    import torch
    return grads[0].device if grads else torch.device("cuda")


def grad_workspace(grads):
    """A workspace for grad_norm and grad_clip on gradients of these sizes, or None."""
    _, count, types = _list(grads)
    return _grad_ws(count, types, _device(grads))


def grad_norm(grads, norm=None, ws=None):
    """norm [1] float32: the root of the sum of the squares of all gradients."""
    import torch
    grads = list(grads)
    ptrs, count, types = _list(grads)
    if norm is None:
        norm = torch.empty(1, dtype=torch.float32, device=_device(grads))
    _vector(norm, "norm", 1, torch.float32)
    if ws is None:
        ws = _grad_ws(count, types, _device(grads))
    _call(lib().grad_norm, "grad_norm", len(grads), ptrs, count, types, _ptr(norm), _ptr(ws),
          _size(ws), _stream())
    return norm


def grad_clip(grads, max_norm, out=None, norm=None, ws=None):
    """Scales the gradients to a global norm of at most max_norm, in place or to
    the tensors of out; returns their norm before that, [1] float32."""
    import torch
    grads = list(grads)
    ptrs, count, types = _list(grads)
    if out is None:
        outs = ptrs
    else:
        out = list(out)
        if len(out) != len(grads):
            raise ValueError("out must hold a tensor for each gradient")
        for g, o in zip(grads, out):
            if o.dtype != g.dtype or o.numel() != g.numel() or not o.is_contiguous() or (
                    o.device.type != "cuda"):
                raise ValueError("a tensor of out must be contiguous, of its gradient's type "
                                 "and size")
        outs = (ctypes.c_void_p * len(out))(*[o.data_ptr() for o in out])
    if norm is None:
        norm = torch.empty(1, dtype=torch.float32, device=_device(grads))
    _vector(norm, "norm", 1, torch.float32)
    if ws is None:
        ws = _grad_ws(count, types, _device(grads))
    _call(lib().grad_clip, "grad_clip", len(grads), ptrs, count, types, max_norm, outs,
          _ptr(norm), _ptr(ws), _size(ws), _stream())
    return norm
