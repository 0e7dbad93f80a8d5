"""include/mitrain.h on the CPU: what calls that need no workspace ask for."""
import os

import pytest

import paper_1903_06934_amd as m
from paper_1903_06934_amd import build as libbuild

OK, WS, DEVICE = 0, -3, -6
F32, BF16, F16 = 0, 1, 2
A, B, C, D, E, G, H, W, S = (0x100000000 * i for i in range(1, 10))


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


@pytest.mark.parametrize("xtype", [F32, BF16, F16])
@pytest.mark.parametrize("cols", [1, 64, 5000, 100352, 1 << 28])
def test_no_rows_need_no_workspace(L, xtype, cols):
    assert L.layernorm_fwd_workspace_size(xtype, 0, cols) == 0
    assert L.layernorm_bwd_workspace_size(xtype, 0, cols) == 0
    assert L.logprob_fwd_workspace_size(xtype, 0, cols, 1) == 0
    assert L.layernorm_bwd(xtype, xtype, 0, cols, None, cols, None, cols, None, None, None, None,
                           cols, H, W, None, 0, None) == launched()


@pytest.mark.parametrize("xtype", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 32, 64])
def test_long_rows_in_one_chunk_need_their_own_sums_only(L, xtype, rows):
    """dw and db are written by the launch that sums them: at most 64 pieces of a row
    have two sums each."""
    cols = 100352
    need = L.layernorm_bwd_workspace_size(xtype, rows, cols)
    assert 0 < need <= rows * 64 * 2 * 4 + 16
    call = lambda ws, n: L.layernorm_bwd(xtype, xtype, rows, cols, A, cols, B, cols, C, D, E, G,
                                         cols, H, W, ws, n, None)
    assert call(S, need - 1) == WS and call(None, 0) == WS
    assert call(S, need) == launched()


def test_build_leaves_the_libraries_where_the_binding_fails(monkeypatch, tmp_path):
    """The binding needs torch's headers and a host compiler; the convolutions and
    the reference points need neither, and are built before it."""
    from paper_1903_06934_amd import isa_check

    def compiled(sources, out, verbose):
        with open(out + ".tmp", "w") as f:
            f.write(" ".join(sources))
        return out + ".tmp"

    def no_headers(verbose):
        raise RuntimeError("no headers")

    for name in ("LIBRARY", "PEAK_LIBRARY", "BINDING"):
        monkeypatch.setattr(libbuild, name, str(tmp_path / name))
    monkeypatch.setattr(libbuild, "_compile", compiled)
    monkeypatch.setattr(libbuild, "_binding", no_headers)
    monkeypatch.setattr(isa_check, "check", lambda *a: None)
    with pytest.raises(RuntimeError, match="no headers"):
        libbuild.build()
    assert (tmp_path / "LIBRARY").read_text().split() == libbuild.SOURCES
    assert (tmp_path / "PEAK_LIBRARY").read_text().split() == libbuild.PEAK_SOURCES
    assert not (tmp_path / "BINDING").exists()
