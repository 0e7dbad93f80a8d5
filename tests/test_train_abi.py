"""include/mitrain.h on the CPU: the library exports what it declares, and every
call refuses bad arguments before touching a device.  The pointers are fake
device addresses that are never dereferenced."""
import ctypes
import os
import re

import pytest

import paper_1903_06934_amd as m
from paper_1903_06934_amd import build as libbuild

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "mitrain.h")
OK, SHAPE, NULL, WS, ALIAS, ALIGN, DEVICE, TYPE, VALUE = 0, -1, -2, -3, -4, -5, -6, -12, -13
F32, BF16, F16 = 0, 1, 2
A, B, C, D, E, G, H, W, S = (0x10000000 * i for i in range(1, 10))
BIG = 1 << 40
inf, nan = float("inf"), float("nan")


@pytest.fixture(scope="module")
def L():
    if not (os.path.exists(libbuild.LIBRARY) and os.path.exists(libbuild.BINDING)):
        libbuild.build()
    return m.lib()


def launched():
    """What a call that passes every check returns here."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present: a call with fake pointers would run")
    return DEVICE


def test_exports_every_declared_function(L):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b([a-z_][a-z0-9_]*)\s*\(", text)) - {"defined"}
    assert names == {"layernorm_fwd", "layernorm_bwd", "layernorm_fwd_workspace_size",
                     "layernorm_bwd_workspace_size", "logprob_fwd", "logprob_bwd",
                     "logprob_fwd_workspace_size", "grad_norm", "grad_clip",
                     "grad_workspace_size"}
    for n in names:
        assert hasattr(L, n), n
    for s in (TYPE, VALUE):
        assert L.conv_error_string(s) != b"unknown status"


def norm_fwd(L, xtype=F32, wtype=F32, rows=8, cols=64, x=A, ldx=64, w=B, b=C, eps=1e-5, y=D,
             ldy=64, mean=E, rstd=G, ws=S, n=BIG):
    return L.layernorm_fwd(xtype, wtype, rows, cols, x, ldx, w, b, eps, y, ldy, mean, rstd, ws, n,
                           None)


@pytest.mark.parametrize("want,args", [
    (TYPE, dict(xtype=3)), (TYPE, dict(xtype=-1)), (TYPE, dict(wtype=BF16)),
    (TYPE, dict(xtype=BF16, wtype=F16)),
    (SHAPE, dict(rows=-1)), (SHAPE, dict(cols=0)), (SHAPE, dict(cols=1 << 29, ldx=1 << 29,
                                                                ldy=1 << 29)),
    (SHAPE, dict(rows=1 << 31)), (SHAPE, dict(rows=1 << 20, cols=1 << 18, ldx=1 << 18,
                                              ldy=1 << 18)),
    (SHAPE, dict(ldx=63)), (SHAPE, dict(ldy=63)), (SHAPE, dict(ldx=1 << 47)),
    (VALUE, dict(eps=-1e-9)), (VALUE, dict(eps=nan)), (VALUE, dict(eps=inf)),
    (NULL, dict(x=None)), (NULL, dict(y=None)),
    (ALIGN, dict(x=A + 2)), (ALIGN, dict(xtype=BF16, x=A + 1)), (ALIGN, dict(w=B + 2)),
    (ALIGN, dict(mean=E + 2)),
    (ALIAS, dict(y=A)), (ALIAS, dict(y=A + 64 * 4)), (ALIAS, dict(mean=B)),
    (ALIAS, dict(mean=G)), (ALIAS, dict(y=C)),
    (ALIAS, dict(ldx=130, ldy=130, y=A + 4 * 63)),      # columns 0..63 and 63..126
    (ALIAS, dict(ldx=130, ldy=130, y=A + 4 * 67)),      # 67..130: the next row's first
    (ALIAS, dict(ldx=130, ldy=128, y=A + 4 * 64)),      # strides differ
    (WS, dict(rows=2, cols=1 << 20, ldx=1 << 20, ldy=1 << 20, n=16)),
    (WS, dict(rows=2, cols=1 << 20, ldx=1 << 20, ldy=1 << 20, ws=None)),
    (ALIGN, dict(rows=2, cols=1 << 20, ldx=1 << 20, ldy=1 << 20, ws=S + 8)),
    (ALIAS, dict(rows=2, cols=1 << 20, ldx=1 << 20, ldy=1 << 20, ws=A + (1 << 20))),
], ids=str)
def test_layernorm_fwd_refuses(L, want, args):
    assert norm_fwd(L, **args) == want


@pytest.mark.parametrize("args", [
    dict(), dict(w=None, b=None, mean=None, rstd=None), dict(rows=0, x=None, y=None),
    dict(xtype=BF16, x=A + 2, y=D + 6), dict(xtype=F16, wtype=F16),
    dict(ldx=128, ldy=128, y=A + 4 * 64),               # two halves of one matrix
    dict(rows=1, ldx=64, ldy=70)], ids=str)
def test_layernorm_fwd_takes(L, args):
    assert norm_fwd(L, **args) == launched()


def norm_bwd(L, xtype=F32, wtype=F32, rows=8, cols=64, dy=A, lddy=64, x=B, ldx=64, mean=C, rstd=D,
             w=E, dx=G, lddx=64, dw=H, db=W, ws=S, n=BIG):
    return L.layernorm_bwd(xtype, wtype, rows, cols, dy, lddy, x, ldx, mean, rstd, w, dx, lddx,
                           dw, db, ws, n, None)


@pytest.mark.parametrize("want,args", [
    (TYPE, dict(xtype=7)), (TYPE, dict(wtype=F16)), (SHAPE, dict(cols=0)), (SHAPE, dict(lddy=1)),
    (SHAPE, dict(ldx=63)), (SHAPE, dict(lddx=0)), (NULL, dict(dy=None)), (NULL, dict(x=None)),
    (NULL, dict(mean=None)), (NULL, dict(rstd=None)), (NULL, dict(dx=None, dw=None, db=None)),
    (ALIGN, dict(dw=H + 1)), (ALIGN, dict(dy=A + 2)), (ALIAS, dict(dx=A)), (ALIAS, dict(dx=B)),
    (ALIAS, dict(dw=W)), (ALIAS, dict(dw=E)), (ALIAS, dict(db=C)), (WS, dict(n=8)),
    (WS, dict(ws=None)), (ALIAS, dict(ws=H))], ids=str)
def test_layernorm_bwd_refuses(L, want, args):
    assert norm_bwd(L, **args) == want


@pytest.mark.parametrize("args", [
    dict(), dict(w=None), dict(dx=None, lddx=0), dict(dw=None), dict(db=None),
    dict(rows=0, dy=None, x=None, mean=None, rstd=None, dx=None),
    dict(xtype=BF16, wtype=BF16, dx=G + 2)], ids=str)
def test_layernorm_bwd_takes(L, args):
    assert norm_bwd(L, **args) == launched()


def logprob_fwd(L, xtype=F32, rows=8, vocab=100, z=A, ld=100, targets=B, scale=1.0, top=5, logp=C,
                lse=D, ent=E, stats=W, tl=G, ti=H, ws=S, n=BIG):
    return L.logprob_fwd(xtype, rows, vocab, z, ld, targets, scale, top, logp, lse, ent, stats,
                         tl, ti, ws, n, None)


@pytest.mark.parametrize("want,args", [
    (TYPE, dict(xtype=3)), (SHAPE, dict(vocab=0)), (SHAPE, dict(ld=99)), (SHAPE, dict(rows=-2)),
    (SHAPE, dict(top=-1)), (SHAPE, dict(top=65)), (SHAPE, dict(vocab=4, top=5)),
    (VALUE, dict(scale=0.0)), (VALUE, dict(scale=-1.0)), (VALUE, dict(scale=nan)),
    (VALUE, dict(scale=inf)), (VALUE, dict(scale=1e-7)),
    (NULL, dict(z=None)), (NULL, dict(targets=None)), (NULL, dict(tl=None)),
    (NULL, dict(ti=None)), (ALIGN, dict(targets=B + 4)), (ALIGN, dict(ti=H + 4)),
    (ALIGN, dict(z=A + 2)), (ALIAS, dict(lse=A + 400)), (ALIAS, dict(lse=C)),
    (ALIAS, dict(stats=E + 4)),
    (ALIAS, dict(tl=B)), (WS, dict(rows=1, vocab=1 << 20, ld=1 << 20, n=64))], ids=str)
def test_logprob_fwd_refuses(L, want, args):
    assert logprob_fwd(L, **args) == want


@pytest.mark.parametrize("args", [
    dict(), dict(targets=None, logp=None), dict(top=0, tl=None, ti=None),
    dict(lse=None, ent=None, stats=None),
    dict(rows=0, z=None, targets=None, tl=None, ti=None), dict(xtype=BF16, z=A + 2),
    dict(vocab=64, top=64)], ids=str)
def test_logprob_fwd_takes(L, args):
    assert logprob_fwd(L, **args) == launched()


def logprob_bwd(L, xtype=F32, rows=8, vocab=100, z=A, ld=100, targets=B, scale=1.0, stats=C, dlogp=D,
                ent=E, dent=G, dz=H, ldd=100):
    return L.logprob_bwd(xtype, rows, vocab, z, ld, targets, scale, stats, dlogp, ent, dent, dz,
                         ldd, None)


@pytest.mark.parametrize("want,args", [
    (TYPE, dict(xtype=-1)), (SHAPE, dict(vocab=0)), (SHAPE, dict(ld=10)), (SHAPE, dict(ldd=10)),
    (VALUE, dict(scale=0.0)), (NULL, dict(z=None)), (NULL, dict(dz=None)), (NULL, dict(stats=None)),
    (NULL, dict(z=None, dz=None)), (NULL, dict(targets=None)), (NULL, dict(ent=None)),
    (NULL, dict(dlogp=None, dent=None)), (ALIGN, dict(dz=H + 2)), (ALIGN, dict(stats=C + 2)),
    (ALIAS, dict(dz=A + 4)), (ALIAS, dict(dz=A, ldd=101)), (ALIAS, dict(dz=C)),
    (ALIAS, dict(z=C, dz=C))], ids=str)
def test_logprob_bwd_refuses(L, want, args):
    assert logprob_bwd(L, **args) == want


@pytest.mark.parametrize("args", [
    dict(), dict(dz=A), dict(dlogp=None, targets=None), dict(dent=None, ent=None),
    dict(rows=0, z=None, dz=None, stats=None, dlogp=None, dent=None),
    dict(dz=A + 400, ld=200, ldd=200)], ids=str)
def test_logprob_bwd_takes(L, args):
    assert logprob_bwd(L, **args) == launched()


def _list(ptrs, counts, types):
    n = len(ptrs)
    return ((ctypes.c_void_p * n)(*ptrs), (ctypes.c_longlong * n)(*counts),
            (ctypes.c_int * n)(*types))


def clip(L, grads=(A, B), counts=(100, 7), types=(F32, BF16), out=None, max_norm=1.0, norm=E, ws=S,
         n=BIG, norm_only=False):
    g, c, t = _list(grads, counts, types)
    if norm_only:
        return L.grad_norm(len(grads), g, c, t, norm, ws, n, None)
    o = g if out is None else (ctypes.c_void_p * len(out))(*out)
    return L.grad_clip(len(grads), g, c, t, max_norm, o, norm, ws, n, None)


@pytest.mark.parametrize("want,args", [
    (TYPE, dict(types=(F32, 5))), (SHAPE, dict(counts=(-1, 7))),
    (SHAPE, dict(counts=(1 << 48, 7))), (NULL, dict(grads=(A, None))),
    (NULL, dict(out=(A, None))), (ALIGN, dict(grads=(A + 2, B))), (ALIGN, dict(out=(A, C + 1))),
    (ALIGN, dict(norm=E + 2)), (VALUE, dict(max_norm=-1.0)), (VALUE, dict(max_norm=nan)),
    (WS, dict(n=8)), (WS, dict(ws=None)), (ALIGN, dict(ws=S + 4)),
    (ALIAS, dict(grads=(A, A + 12))), (ALIAS, dict(out=(C, C + 390))), (ALIAS, dict(out=(B, A))),
    (ALIAS, dict(out=(C, A + 10))), (ALIAS, dict(norm=A + 4)), (ALIAS, dict(ws=B)),
    (ALIAS, dict(norm=S)), (ALIAS, dict(out=(A + 4, B)))], ids=str)
def test_grad_clip_refuses(L, want, args):
    assert clip(L, **args) == want


@pytest.mark.parametrize("args", [
    dict(), dict(norm=None), dict(out=(C, D)), dict(max_norm=inf), dict(max_norm=0.0),
    dict(counts=(100, 0), grads=(A, None), out=(A, None)), dict(grads=(A, A), out=(C, D)),
    dict(grads=(), counts=(), types=()), dict(grads=(B, A), types=(F16, F32))], ids=str)
def test_grad_clip_takes(L, args):
    assert clip(L, **args) == launched()


@pytest.mark.parametrize("want,args", [
    (NULL, dict(norm=None)), (NULL, dict(grads=(None, B))), (TYPE, dict(types=(9, F32))),
    (ALIAS, dict(norm=A)), (ALIAS, dict(ws=A)), (WS, dict(n=0))], ids=str)
def test_grad_norm_refuses(L, want, args):
    assert clip(L, norm_only=True, **args) == want


def test_null_lists(L):
    assert L.grad_clip(1, None, None, None, 1.0, None, E, S, BIG, None) == NULL
    assert L.grad_clip(-1, None, None, None, 1.0, None, E, S, BIG, None) == SHAPE
    assert L.grad_workspace_size(3, None, None) == 0


def test_workspace_sizes(L):
    assert L.layernorm_fwd_workspace_size(F32, 4, 64) == 0
    assert L.layernorm_fwd_workspace_size(F32, 4, 1 << 20) > 0
    assert L.layernorm_bwd_workspace_size(F32, 4, 64) >= 2 * 64 * 4
    assert L.logprob_fwd_workspace_size(BF16, 4096, 32000, 5) == 0
    assert L.logprob_fwd_workspace_size(BF16, 1, 128000, 5) > 0
    for bad in ((3, 4, 64), (F32, -1, 64), (F32, 4, 0), (F32, 1 << 31, 4)):
        assert L.layernorm_fwd_workspace_size(*bad) == 0
        assert L.layernorm_bwd_workspace_size(*bad) == 0
        assert L.logprob_fwd_workspace_size(*bad, 0) == 0


def test_binding_refuses(L):
    """The binding's own checks, on CPU tensors and layouts that no row stride covers."""
    import torch
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        m.layernorm_fwd(x)
    with pytest.raises(ValueError):
        m.logprob_fwd(x)
    with pytest.raises(ValueError):
        m.grad_norm([x])
    from paper_1903_06934_amd import mitrain
    rows = mitrain._binding().rows
    assert rows(torch.zeros(4, 6, 8)) == (24, 8, 8)
    assert rows(torch.zeros(4, 6, 8)[:, :, :5]) == (24, 5, 8)
    assert rows(torch.zeros(4, 6, 8)[:, 0]) == (4, 8, 48)
    assert rows(torch.zeros(4, 1, 8)[:, :, 2:]) == (4, 6, 8)
    assert rows(torch.zeros(8)) == (1, 8, 8)
    assert rows(torch.zeros(0, 8)) == (0, 8, 8)
    for bad in (torch.zeros(4, 6, 8)[:, :3], torch.zeros(8, 4).t(), torch.zeros(1, 8).expand(3, 8),
                torch.zeros(())):
        with pytest.raises(ValueError):
            rows(bad)
