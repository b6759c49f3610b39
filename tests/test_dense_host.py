"""Refusals and sizes of the dense calls (include/singa_mi_dense.h), on the
CPU: every check answers before a launch, so made-up addresses do."""
import ctypes
import os
import re

import pytest
import torch

from paper_1603_07846_amd import singa
from paper_1603_07846_amd import workloads as wl
from paper_1603_07846_amd.net import Net

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "singa_mi_dense.h")
A = 1 << 20  # an aligned address that nothing is ever read from
NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGN = -1, -2, -3, -4, -5


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(singa_[a-z0-9_]+)\s*\(", text))) == sorted(singa.DENSE_EXPORTS)
    for n in singa.DENSE_EXPORTS:
        assert hasattr(singa.lib(), n), n


def fwd(dt=0, rows=100, din=64, dout=64, x=A, w=A, bias=A, act=0, res=None, z=None, y=A, ws=A, nbytes=1 << 30):
    return singa.lib().singa_linear_fwd(dt, rows, din, dout, x, w, bias, act, res, z, y, ws, nbytes, None)


@pytest.mark.parametrize("change,want", [
    (dict(dt=2), UNSUPPORTED), (dict(act=4), UNSUPPORTED), (dict(act=-1), UNSUPPORTED), (dict(rows=-1), SHAPE),
    (dict(din=0), SHAPE), (dict(dout=0), SHAPE), (dict(din=(1 << 20) + 1), UNSUPPORTED), (dict(x=None), NULL),
    (dict(w=None), NULL), (dict(y=None), NULL), (dict(x=A + 4), ALIGN), (dict(y=A + 8), ALIGN), (dict(z=A + 2), ALIGN),
    (dict(res=A + 4), ALIGN), (dict(bias=A + 2), ALIGN), (dict(rows=1000, din=63, nbytes=100), WORKSPACE),
    (dict(rows=1000, din=63, ws=None), WORKSPACE), (dict(rows=1000, din=63, ws=A + 4), ALIGN), (dict(rows=1 << 29), UNSUPPORTED),
    (dict(rows=0, x=None, y=None), 0)])
def test_linear_fwd_refuses(change, want):
    assert fwd(**change) == want


def bwd(dt=1, rows=100, din=64, dout=64, x=A, w=A, z=A, act=2, dy=A, res=None, dx=A, dw=A, gt=0, db=A, acc=0, ws=A,
        nbytes=1 << 30):
    return singa.lib().singa_linear_bwd(dt, rows, din, dout, x, w, z, act, dy, res, dx, dw, gt, db, acc, ws, nbytes, None)


@pytest.mark.parametrize("change,want", [
    (dict(dt=3), UNSUPPORTED), (dict(act=9), UNSUPPORTED), (dict(gt=2), UNSUPPORTED), (dict(dt=0, gt=1), UNSUPPORTED),
    (dict(gt=1, acc=1), UNSUPPORTED), (dict(rows=-1), SHAPE), (dict(dout=0), SHAPE),
    (dict(dx=None, dw=None, db=None), NULL), (dict(dy=None), NULL), (dict(x=None), NULL), (dict(w=None), NULL),
    (dict(z=None), NULL), (dict(dx=A + 4), ALIGN), (dict(dw=A + 4), ALIGN), (dict(db=A + 2), ALIGN),
    (dict(dy=A + 2), ALIGN), (dict(res=A + 2), ALIGN), (dict(ws=None), WORKSPACE), (dict(nbytes=1000), WORKSPACE),
    (dict(rows=0, acc=1), 0)])
def test_linear_bwd_refuses(change, want):
    assert bwd(**change) == want


def ce(dt=1, rows=100, din=64, classes=1000, x=A, w=A, bias=A, labels=A, loss=A, dx=A, dw=A, gt=0, db=A, acc=0, ws=A,
       nbytes=1 << 30):
    return singa.lib().singa_linear_softmax_ce(dt, rows, din, classes, x, w, bias, labels, 1.0, loss, dx, dw, gt, db, acc,
                                               ws, nbytes, None)


@pytest.mark.parametrize("change,want", [
    (dict(dt=2), UNSUPPORTED), (dict(dt=0, gt=1), UNSUPPORTED), (dict(gt=1, acc=1), UNSUPPORTED), (dict(rows=-5), SHAPE),
    (dict(classes=0), SHAPE), (dict(classes=1 << 21), UNSUPPORTED), (dict(loss=None), NULL), (dict(w=None), NULL),
    (dict(x=None), NULL), (dict(labels=None), NULL), (dict(labels=A + 1), ALIGN), (dict(loss=A + 2), ALIGN),
    (dict(x=A + 8), ALIGN), (dict(w=A + 2), ALIGN), (dict(ws=None), WORKSPACE), (dict(nbytes=4096), WORKSPACE),
    (dict(ws=A + 8), ALIGN)])
def test_linear_softmax_ce_refuses(change, want):
    assert ce(**change) == want


def norm(count=2, dtypes=(0, 1), grads=(A, A), sizes=(10, 10), max_norm=1.0, stat=A, ws=A, nbytes=1 << 20, outs=None):
    n = len(grads)
    d, p, s = (ctypes.c_int * n)(*dtypes), (ctypes.c_void_p * n)(*grads), (ctypes.c_size_t * n)(*sizes)
    if outs is None:
        return singa.lib().singa_grad_norm(count, d, p, s, max_norm, stat, ws, nbytes, None)
    return singa.lib().singa_grad_clip(count, d, p, (ctypes.c_void_p * n)(*outs), s, max_norm, stat, ws, nbytes, None)


@pytest.mark.parametrize("change,want", [
    (dict(count=-1), SHAPE), (dict(max_norm=-1.0), UNSUPPORTED), (dict(max_norm=float("nan")), UNSUPPORTED),
    (dict(stat=None), NULL), (dict(grads=(A, None)), NULL), (dict(dtypes=(0, 2)), UNSUPPORTED),
    (dict(grads=(A + 2, A)), ALIGN), (dict(grads=(A, A + 1)), ALIGN), (dict(stat=A + 2), ALIGN),
    (dict(ws=None), WORKSPACE), (dict(nbytes=64), WORKSPACE), (dict(outs=(A, None)), NULL),
    (dict(outs=(A + 2, A)), ALIGN), (dict(sizes=(1 << 41, 1)), SHAPE)])
def test_grad_norm_refuses(change, want):
    assert norm(**change) == want


def test_scaled_updates_refuse():
    f, n = ctypes.c_float, ctypes.c_size_t
    sgd, ada = singa.lib().singa_sgd_momentum_update_scaled, singa.lib().singa_adagrad_update_scaled
    assert sgd(n(0), None, None, None, None, 0.1, 0.9, 0.0, None, None) == 0
    assert sgd(n(8), A, A, A, None, 0.1, 0.9, 0.0, None, None) == NULL
    assert sgd(n(8), A, A + 4, A, None, 0.1, 0.9, 0.0, A, None) == ALIGN
    assert ada(n(8), A, A, A, None, 0.1, 1e-6, 0.0, None, None) == NULL
    assert ada(n(8), A, A, A, None, 0.1, 0.0, 0.0, A, None) == UNSUPPORTED


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_workspaces(dt):
    es = torch.empty((), dtype=dt).element_size()
    # few rows read the weights as they are
    for rows in (0, 1, 16):
        assert singa.linear_fwd_workspace_bytes(dt, rows, 1001, 777) == 0
    # odd rows cost a copy of both matrices
    assert singa.linear_fwd_workspace_bytes(dt, 4096, 1001, 4096) >= 2 * 4096 * 1001 * es
    assert singa.linear_fwd_workspace_bytes(dt, 4096, 4096, 4096) == 0
    assert singa.linear_bwd_workspace_bytes(dt, 0, 64, 64) == 0
    # two further terms of the gradient where a smooth activation meets an fp32 dw
    one = singa.linear_bwd_workspace_bytes(torch.bfloat16, 4096, 4096, 4096, "gelu", torch.bfloat16)
    assert singa.linear_bwd_workspace_bytes(torch.bfloat16, 4096, 4096, 4096, "gelu") - one == 2 * 4096 * (4096 + 64) * 2
    assert singa.linear_bwd_workspace_bytes(torch.bfloat16, 4096, 4096, 4096, "relu") == one
    # the loss: never the logits of a large problem, with or without gradients
    rows, classes = 16384, 131072
    assert singa.linear_softmax_ce_workspace_bytes(dt, rows, 64, classes, False) < rows * classes // 4
    assert singa.linear_softmax_ce_workspace_bytes(dt, rows, 64, classes, True) < rows * classes // 2 + (512 << 20)
    for fn, args in ((singa.linear_fwd_workspace_bytes, (dt, -1, 4, 4)), (singa.linear_bwd_workspace_bytes, (dt, 4, 0, 4)),
                     (singa.linear_softmax_ce_workspace_bytes, (dt, 4, 4, 0))):
        with pytest.raises(singa.SingaError) as e:
            fn(*args)
        assert e.value.status == SHAPE
    with pytest.raises(singa.SingaError):
        singa.linear_bwd_workspace_bytes(torch.float32, 4, 4, 4, "none", torch.bfloat16)


def test_python_checks():
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    with pytest.raises(ValueError, match="x"):  # a host tensor
        singa.linear_fwd(x, w)
    with pytest.raises(ValueError, match="wanted"):
        singa.linear_fwd(x, torch.zeros(6, 7))
    with pytest.raises(TypeError):
        singa.linear_fwd(x.half(), w.half())
    with pytest.raises(ValueError, match="contiguous"):
        singa.linear_fwd(torch.zeros(8, 4).t(), w)
    with pytest.raises(ValueError, match="act"):
        singa._act("tanh")
    with pytest.raises(TypeError, match="dw_dtype"):
        singa._dw_dt(x, torch.bfloat16)
    with pytest.raises(ValueError, match="grads"):
        singa.grad_norm([])
    with pytest.raises(ValueError, match="grads"):
        singa.grad_norm([x])


X, W, Y, Z, B2 = (A + i * (1 << 24) for i in range(1, 6))  # far enough apart for every call below


@pytest.mark.parametrize("change", [
    dict(y=X), dict(y=W), dict(z=Y), dict(z=X + 16), dict(y=X + 100 * 64 * 4 - 16), dict(bias=Y + 4), dict(res=Y + 16),
    dict(z=B2, res=B2)])
def test_linear_fwd_refuses_shared_memory(change):
    assert fwd(**{**dict(x=X, w=W, y=Y, z=None, bias=None), **change}) == UNSUPPORTED


@pytest.mark.parametrize("change", [
    dict(dx=X), dict(dx=W), dict(dx=Y), dict(dx=Z), dict(dw=X), dict(dw=A + 16), dict(db=A + 4), dict(res=A + 16),
    dict(dw=None, db=None, dx=Y)])
def test_linear_bwd_refuses_shared_memory(change):
    args = dict(x=X, w=W, dy=Y, z=Z, dx=A, dw=B2, db=A + (1 << 23), ws=A + (1 << 28))
    assert bwd(**{**args, **change}) == UNSUPPORTED


@pytest.mark.parametrize("change", [
    dict(dx=X), dict(dw=W), dict(db=Z), dict(labels=A), dict(loss=X), dict(dx=Y), dict(dw=X + 100 * 64 * 2 - 16)])
def test_linear_softmax_ce_refuses_shared_memory(change):
    args = dict(x=X, w=W, bias=Z, labels=Z + 8192, loss=A, dx=A + 8192, dw=Y, db=B2, ws=A + (1 << 28))
    assert ce(**{**args, **change}) == UNSUPPORTED


@pytest.mark.parametrize("grads,outs,sizes", [
    ((A, A), (A, A), (10, 10)),                          # a gradient listed twice
    ((A, A + 16), (A, A + 16), (10, 10)),                # a view of another one
    ((A, A + 4096), (A + 4096, A), (10, 10)),            # outputs in the other's place
    ((A, A + 4096), (A + 8192, A + 8208), (10, 10)),     # outputs that overlap
    ((A, A + 4096), (A + 4, A + 4096), (10, 10)),        # an output a step beside its gradient
    ((A, A + 64), (A, A + 64), (1000, 1))])
def test_clipping_refuses_shared_memory(grads, outs, sizes):
    assert norm(dtypes=(0, 0), grads=grads, outs=outs, sizes=sizes) == UNSUPPORTED


def test_sizes_beyond_the_limits_are_refused():
    # rows x in, rows x out, in x out: 2^37 elements at most
    for r, i, o in ((1 << 28, 1 << 10, 8), (1 << 28, 8, 1 << 10), (8, 1 << 20, 1 << 18)):
        assert fwd(rows=r, din=i, dout=o) == UNSUPPORTED
        assert bwd(rows=r, din=i, dout=o) == UNSUPPORTED
        assert ce(rows=r, din=i, classes=o) == UNSUPPORTED


def test_fused_loss_wants_a_layer_to_fuse():
    layers = (wl.FC("fc", 6, out_shape=(6, 1, 1)), wl.Relu("relu"), wl.SoftmaxCE())
    with pytest.raises(ValueError, match="fused_loss"):
        Net(wl.Workload(51, "a ReLU before the loss", "f32", 2, (4, 6, 6), "normal", layers, classes=6), device="cpu",
            fused_loss=True)
