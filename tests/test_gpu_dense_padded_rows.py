"""Gradients whose rows in the workspace are a multiple of 4 KB long and take 64
elements more (out a multiple of 2048 in bf16, of 1024 in fp32): the widths
that layers usually have.  Bounds as in test_gpu_dense.py."""
import pytest
import torch

from paper_1603_07846_amd import singa
from test_gpu_dense import DT, check_bwd, check_ce, rnd

pytestmark = pytest.mark.gpu

WIDTH = {"f32": 1024, "bf16": 2048}


def beside_nan(g, *shape, dtype):
    """A tensor of that shape with NaN right behind its last element, in memory of its own."""
    n = 1
    for d in shape:
        n *= d
    flat = singa.empty((n + 4096,), dtype, "cuda")
    flat[n:] = float("nan")
    flat[:n] = torch.randn(n, generator=g).to(dtype).cuda()
    return flat[:n].view(shape)


@pytest.mark.parametrize("rows", [1, 3, 64, 131])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("dt,gt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
def test_only_the_rows_themselves_are_read(dt, gt, act, rows):
    """What lies in the columns between the end of a row of dz and the start of the next one is zero, as are the rows
    that only pad: a read past a row of dy or z would leave its product there."""
    T, out, din = DT[dt], WIDTH[dt], 16
    g = torch.Generator().manual_seed(41)
    x, w = rnd(g, rows, din, dtype=T), rnd(g, out, din, dtype=T)
    z, dy = beside_nan(g, rows, out, dtype=T), beside_nan(g, rows, out, dtype=T)
    z[:, :64] = 1.0  # what a row's end would read of the next one passes
    dy[:, :64] = 2.0
    ws = singa.empty((singa.linear_bwd_workspace_bytes(T, rows, din, out, act, DT[gt]),), torch.uint8, "cuda")
    ws.fill_(0xff)
    assert ws.data_ptr() % 256 == 0  # dz is the workspace's first part then
    grads = singa.linear_bwd(x, w, dy, act=act, z=z, dw_dtype=DT[gt], workspace=ws)
    assert all(bool(t.isfinite().all()) for t in grads)
    terms = 3 if dt == "bf16" and gt == "f32" and act != "relu" else 1
    held = -(-rows // 64) * 64 if terms == 3 else rows
    es = torch.finfo(T).bits // 8
    dz = ws[:terms * held * (out + 64) * es].view(T).view(terms, held, out + 64)
    assert not bool(dz[:, :, out:].any()) and not bool(dz[:, rows:].any())
    assert bool(dz[0, :rows, :64].all())


@pytest.mark.parametrize("rows", [5, 131])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dt,gt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
def test_gradients_of_usual_widths(dt, gt, act, rows):
    check_bwd(dt, rows, 72, WIDTH[dt], act, gt, res=rows == 5)
    check_bwd(dt, rows, 33, 2 * WIDTH[dt], act, gt)


@pytest.mark.parametrize("dt,gt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows,din,factor", [(7, 40, 1), (131, 33, 2), (600, 16, 4), (65, 24, 16)])
def test_losses_of_usual_numbers_of_classes(dt, gt, rows, din, factor):
    check_ce(dt, rows, din, factor * WIDTH[dt], gt, padded=0.2)


@pytest.mark.parametrize("dt,gt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
def test_pieces_of_whole_pages(dt, gt):
    """Logits that are not kept: one piece of 16 x 4 KB rows (600 rows), and pieces of a multiple of 4 KB and a rest."""
    check_ce(dt, 600, 16, 32768, gt, padded=0.2)
    rows = 2048 if dt == "f32" else 4096  # pieces of 32768 classes
    check_ce(dt, rows, 8, 32768 + 300, gt, padded=0.2)
