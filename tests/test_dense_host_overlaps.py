"""What the dense calls write beside their tensors (workspaces, the norm and
its scale) shares memory with no tensor, and a scaled update's streams share
none with each other: refused before a launch, so made-up addresses do."""
import ctypes

import pytest

from paper_1603_07846_amd import singa
from test_dense_host import A, UNSUPPORTED, bwd, ce, fwd, norm

X, W, Y, Z, DX, DW, V = (A + i * (1 << 24) for i in range(1, 8))
END = 1000 * 63 * 4  # bytes of x there, a multiple of 16: the last 16 of them overlap, what follows does not


@pytest.mark.parametrize("ws", [X, W, Y, Z, X + END - 16, Y - 1024, Y + 1000 * 64 * 4 - 16, DX])
def test_linear_fwd_keeps_its_workspace_apart(ws):
    assert fwd(rows=1000, din=63, x=X, w=W, y=Y, z=Z, res=DX, bias=None, ws=ws) == UNSUPPORTED


@pytest.mark.parametrize("ws", [X, W, Y, Z, DX, DW, V, Y + 16, DX - 1024])
def test_linear_bwd_keeps_its_workspace_apart(ws):
    assert bwd(rows=1000, x=X, w=W, dy=Y, z=Z, dx=DX, dw=DW, db=V, res=None, ws=ws) == UNSUPPORTED


@pytest.mark.parametrize("ws", [X, W, Y, Z, DX, DW, V, X - 1024, V + 992 * 4])
def test_the_loss_keeps_its_workspace_apart(ws):
    assert ce(x=X, w=W, bias=Y, labels=Z, loss=V + (1 << 20), dx=DX, dw=DW, db=V, ws=ws) == UNSUPPORTED


@pytest.mark.parametrize("change", [
    dict(stat=X), dict(stat=X + 36), dict(stat=X - 4), dict(stat=Y + 16), dict(ws=X), dict(ws=Y), dict(ws=X - 1024),
    dict(stat=W, ws=W), dict(stat=W + 8, ws=W)])
@pytest.mark.parametrize("outs", [None, "in place", "others"])
def test_the_norm_keeps_its_figures_apart(change, outs):
    to = {None: None, "in place": (X, Y), "others": (DX, DW)}[outs]
    args = dict(grads=(X, Y), sizes=(10, 10), stat=V, ws=Z, outs=to)
    assert norm(**{**args, **change}) == UNSUPPORTED


@pytest.mark.parametrize("change", [dict(stat=DX), dict(stat=DW + 16), dict(ws=DX), dict(ws=DW - 1024)])
def test_clipping_keeps_its_figures_apart_from_outputs(change):
    assert norm(**{**dict(grads=(X, Y), sizes=(10, 10), stat=V, ws=Z, outs=(DX, DW)), **change}) == UNSUPPORTED


@pytest.mark.parametrize("w,g,v,wb,scale", [
    (X, W, Y, None, X + 8), (X, W, Y, None, Y + 28), (X, W, Y, Z, Z), (X, X + 16, Y, None, Z), (X, W, X, None, Z),
    (X, W, W, None, Z), (X, W, Y, X + 16, Z), (X, W, Y, W, Z)])
def test_scaled_updates_keep_their_streams_apart(w, g, v, wb, scale):
    n = ctypes.c_size_t(8)
    assert singa.lib().singa_sgd_momentum_update_scaled(n, w, g, v, wb, 0.1, 0.9, 0.0, scale, None) == UNSUPPORTED
    assert singa.lib().singa_adagrad_update_scaled(n, w, g, v, wb, 0.1, 1e-6, 0.0, scale, None) == UNSUPPORTED
