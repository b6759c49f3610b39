"""Softmax cross-entropy of rows whose logits share a large offset: the loss of
a confident row, and all probabilities, do not depend on it.

x picks one column of w, w is a multiple of 2^-4 below 8 and the bias a whole
number, so every logit is exact in fp32.  Bounds: a term of a row's sum is off
by (|z - max| log2(e) + 2) F of itself, at most 26 F here (|z - max| < 16), the
sums and the logarithm by at most 34 F more of the sum: 60 F, and F of the loss
itself.  A probability is off by F (|z - lse| log2(e) + 60) relative.
"""
import pytest
import torch

from paper_1603_07846_amd import singa
from test_gpu_dense import DT, F, G, dev, u_of, within

pytestmark = pytest.mark.gpu

SIZES = [(1, 16, 1), (1, 64, 1000), (5, 64, 300), (90, 16, 1000), (13, 24, 7817), (333, 24, 5003), (100, 16, 10007),
         (1100, 8, 200), (700, 24, 26003)]


def make(dt, rows, din, classes, offset):
    T = DT[dt]
    g = torch.Generator().manual_seed(43 + rows + classes)
    x = torch.zeros(rows, din)
    pick = torch.arange(rows) % din
    x[torch.arange(rows), pick] = 1
    w = torch.randint(-128, 0, (classes, din), generator=g) / 16.0
    labels = torch.randint(0, classes, (rows,), generator=g, dtype=torch.int32)
    # every other column belongs to rows that are sure of one class
    sure = torch.randint(0, classes, (din,), generator=g)
    for k in range(0, din, 2):
        w[sure[k], k] = 7.5
    confident = pick % 2 == 0
    labels[confident] = sure[pick[confident]].int()
    bias = torch.full((classes,), float(offset))
    assert torch.equal(w.to(T).float(), w)
    return dev(x, T), dev(w, T), dev(labels), dev(bias)


def check(dt, rows, din, classes, offset, grad):
    x, w, labels, bias = make(dt, rows, din, classes, offset)
    loss, _, dw, db = singa.linear_softmax_ce(x, w, labels, bias, grad=grad)
    z = x.double() @ w.double().t()  # without the offset
    at = labels.long()[:, None]
    lse = torch.logsumexp(z, 1)
    want = lse - z.gather(1, at)[:, 0]
    within("rows", loss[1:], want, 60 * F + F * want)
    within("mean", loss[0], want.mean(), 60 * F + 3 * F * want.mean())
    if not grad:
        return
    p = torch.exp(z - lse[:, None])
    dz = p.scatter_add(1, at, torch.full_like(lse[:, None], -1.0)) / rows
    e = (p * F * ((z - lse[:, None]).abs() * 1.4427 + 60) + 2 * F) / rows + 2 * F * dz.abs()
    within("db", db, dz.sum(0), e.sum(0) + G(rows) * dz.abs().sum(0))
    u = u_of(torch.bfloat16) ** 3 if dt == "bf16" else 0.0
    ref, xa = dz.t() @ x.double(), x.double().abs()
    off = (e + (u + 2 * G(3 * rows)) * dz.abs()).t() @ xa
    within("dw", dw, ref, off + F * ref.abs() + 1e-37)


@pytest.mark.parametrize("offset", [0, 1000, -65536, 524288])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_an_offset_of_all_logits_changes_nothing(size, dt, offset):
    check(dt, *size, offset, True)


@pytest.mark.parametrize("offset", [1000, -65536])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES + [(3, 64, 40000), (300, 72, 1111)])
def test_nor_of_the_loss_alone(size, dt, offset):
    check(dt, *size, offset, False)
