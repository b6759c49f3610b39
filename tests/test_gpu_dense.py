"""The dense calls (include/singa_mi_dense.h) on the GPU against 64-bit
formulas.

Bounds, per element, from the arithmetic alone: u = eps / 2 of the tensors'
type is one rounding of a stored value, G(n) = (n + 4) 2^-24 the relative
error of an fp32 sum of n products against the sum of their magnitudes.
  y, z      G(in) S, S = |x| |w|^T + |b|, through an activation whose slope is
            at most 1.13, plus the activation's own error: bf16 results 2^-21
            of |z| (a polynomial of relative error 4.5e-7 and the hardware's
            exponential), fp32 2^-21 as well (a few ulp of erf / exp).
  dz        4 ulp and 2^-20 of |dy| (the slope), rounded to the type: u |dz|,
            or u^3 |dz| where it is kept in three terms (fp32 dw of a smooth
            activation), or nothing (ReLU, none).
  softmax   p is off by e^(2 d) - 1 relative, d = the largest error of a
            row's logits, plus 2^-24 (|z - lse| log2(e) + 60) of the
            exponential, the sum and the logarithm.
"""
import math

import pytest
import torch

from paper_1603_07846_amd import singa

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
F = 2.0 ** -24


def u_of(dt):
    return torch.finfo(dt).eps / 2


def G(n):
    return (n + 4) * F


def dev(t, dtype=None):
    """A guarded device copy."""
    dtype = dtype or t.dtype
    out = singa.empty(tuple(t.shape), dtype, "cuda")
    out.copy_(t.to(dtype))
    return out


def rnd(g, *shape, dtype=torch.float32, scale=1.0):
    return dev(torch.randn(shape, generator=g) * scale, dtype)


def within(name, got, ref, bound):
    got, ref = got.double(), ref.double()
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    off = (got - ref).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (name, int(bad.sum()), "first", torch.nonzero(bad)[0].tolist(),
                                 float(got[bad][0]), float(ref[bad][0]), float(off[bad][0]),
                                 float(torch.as_tensor(bound, device=off.device).expand_as(off)[bad][0]))


def act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope64(z, act):
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


SIZES = [(1, 1, 1), (1, 4096, 257), (2, 7, 5), (3, 64, 1000), (16, 100, 250), (17, 513, 8), (33, 40, 300), (64, 1023, 17),
         (65, 7, 129), (100, 1001, 77), (129, 64, 128), (300, 8, 1), (256, 4096, 130), (500, 260, 1030)]
# the larger tile, one whole and one ragged problem
LARGE = [(3584, 128, 3584), (3333, 200, 4001)]


def check_fwd(dt, rows, din, dout, act, bias, res, keep, seed=0):
    g = torch.Generator().manual_seed(seed + rows + din + dout)
    T = DT[dt]
    x, w = rnd(g, rows, din, dtype=T), rnd(g, dout, din, dtype=T, scale=1 / math.sqrt(din))
    b = rnd(g, dout) if bias else None
    r = rnd(g, rows, dout, dtype=T) if res else None
    out = singa.linear_fwd(x, w, b, act=act, residual=r, keep_z=keep)
    y, z = out if keep else (out, None)
    zr = x.double() @ w.double().t()
    s = x.double().abs() @ w.double().abs().t()
    if bias:
        zr, s = zr + b.double(), s + b.double().abs()
    dz = G(din) * s
    yr = act64(zr, act)
    if z is not None:
        within("z", z, zr, dz + u_of(T) * (zr.abs() + dz))
    if res:
        yr = yr + r.double()
    off = 1.13 * dz + 2.0 ** -21 * zr.abs() + 2 * F * (yr.abs() + (r.double().abs() if res else 0))
    within("y", y, yr, off + u_of(T) * (yr.abs() + off))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", SIZES)
def test_linear_fwd(size, dt):
    i = SIZES.index(size)
    act = ("none", "relu", "gelu", "silu")[i % 4]
    check_fwd(dt, *size, act, bias=i % 2 == 0, res=i % 3 != 1, keep=i % 3 != 0)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_linear_fwd_activations(act, dt):
    check_fwd(dt, 40, 64, 64, act, True, True, True)
    check_fwd(dt, 200, 64, 136, act, True, True, True)


@pytest.mark.parametrize("size", LARGE)
def test_linear_fwd_large(size):
    check_fwd("bf16", *size, "gelu", True, True, True)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [5, 130])
def test_linear_fwd_values_far_out(rows, dt):
    """Infinities and NaN stay where the formula puts them, and in their own rows."""
    T = DT[dt]
    x = torch.zeros(rows, 64)
    x[0, 0], x[1, 0], x[2, 0], x[3, 0] = float("inf"), float("nan"), -1e4, 1e4
    w = torch.zeros(32, 64)
    w[:, 0] = 1
    for act in ("none", "relu", "gelu", "silu"):
        y = singa.linear_fwd(dev(x, T), dev(w, T), act=act).float()
        far = float(torch.tensor(1e4).to(T))
        assert bool((y[4:] == 0).all()) and bool(y[1].isnan().all()) and bool((y[0] == float("inf")).all())
        assert bool((y[2] == (-far if act == "none" else 0.0)).all()) and bool((y[3] == far).all())


def check_bwd(dt, rows, din, dout, act, gt="f32", bias=True, res=False, accumulate=False, seed=1):
    g = torch.Generator().manual_seed(seed + rows + din + dout)
    T, GT = DT[dt], DT[gt]
    x, w = rnd(g, rows, din, dtype=T), rnd(g, dout, din, dtype=T)
    z = rnd(g, rows, dout, dtype=T, scale=1.5) if act != "none" else None
    dy = rnd(g, rows, dout, dtype=T)
    r = rnd(g, rows, din, dtype=T) if res else None
    kw = {}
    if accumulate:
        kw = {"dw": rnd(g, dout, din), "db": rnd(g, dout), "accumulate": True}
        dw0, db0 = kw["dw"].double(), kw["db"].double()
    dx, dw, db = singa.linear_bwd(x, w, dy, act=act, z=z, dx_residual=r, with_bias=bias, dw_dtype=GT, **kw)
    smooth = act in ("gelu", "silu")
    dz = dy.double() * (slope64(z.double(), act) if z is not None else 1)
    e0 = (4 * F * dz.abs() + 2.0 ** -20 * dy.double().abs()) if smooth else torch.zeros_like(dz)
    u = u_of(T) if T == torch.bfloat16 and smooth else 0.0
    xa, wa, da = x.double().abs(), w.double().abs(), dz.abs()
    ref = dz @ w.double()
    off = (e0 + u * da + G(dout) * da) @ wa
    if res:
        ref = ref + r.double()
        off = off + F * (ref.abs() + r.double().abs())
    within("dx", dx, ref, off + u_of(T) * (ref.abs() + off))
    uw = u ** 3 if gt == "f32" else u
    ref = dz.t() @ x.double()
    off = (e0 + uw * da + G(3 * rows) * da * (1 + u)).t() @ xa
    if accumulate:
        ref = ref + dw0
        off = off + F * (ref.abs() + dw0.abs())
    within("dw", dw, ref, off + (u_of(GT) if GT != torch.float32 else F) * (ref.abs() + off))
    if bias:
        ref, off = dz.sum(0), e0.sum(0) + G(rows) * da.sum(0)
        if accumulate:
            ref = ref + db0
            off = off + F * (ref.abs() + db0.abs())
        within("db", db, ref, off)
    else:
        assert db is None


@pytest.mark.parametrize("dt,gt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("size", SIZES)
def test_linear_bwd(size, dt, gt):
    i = SIZES.index(size)
    check_bwd(dt, *size, ("gelu", "none", "relu", "silu")[i % 4], gt, bias=i % 3 != 2, res=i % 2 == 0)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_linear_bwd_accumulates(act, dt):
    check_bwd(dt, 70, 72, 130, act, accumulate=True)
    check_bwd(dt, 1000, 136, 40, act, accumulate=True)  # sums cut along the rows


@pytest.mark.parametrize("act,gt", [("gelu", "f32"), ("silu", "bf16"), ("none", "f32")])
def test_linear_bwd_large(act, gt):
    check_bwd("bf16", 3333, 4001, 200, act, gt)
    check_bwd("bf16", 300, 3584, 3600, act, gt, res=True)


def test_linear_bwd_parts_and_empty():
    g = torch.Generator().manual_seed(5)
    x, w, dy = rnd(g, 70, 24), rnd(g, 40, 24), rnd(g, 70, 40)
    all_ = singa.linear_bwd(x, w, dy)
    one = (singa.linear_bwd(x, w, dy, need_dw=False, with_bias=False), singa.linear_bwd(x, w, dy, need_dx=False, with_bias=False),
           singa.linear_bwd(x, w, dy, need_dx=False, need_dw=False))
    for i in range(3):
        assert torch.equal(one[i][i], all_[i]) and all(one[i][j] is None for j in range(3) if j != i)
    y = singa.linear_fwd(x[:0], w)
    assert y.shape == (0, 40)
    dx, dw, db = singa.linear_bwd(x[:0], w, dy[:0])
    assert dx.shape == (0, 24) and not bool(dw.any()) and not bool(db.any())
    dx, dw2, db2 = singa.linear_bwd(x[:0], w, dy[:0], dw=all_[1], db=all_[2], accumulate=True)
    assert bool(dw2.any()) and bool(db2.any())


def test_relu_gradient_is_zero_where_it_passes_nothing():
    g = torch.Generator().manual_seed(6)
    for T in DT.values():
        x, w, z = rnd(g, 80, 24, dtype=T), rnd(g, 40, 24, dtype=T), rnd(g, 80, 40, dtype=T)
        dy = rnd(g, 80, 40, dtype=T)
        dy[z <= 0] = float("nan")
        z[3], dy[3] = -1.0, float("inf")
        out = singa.linear_bwd(x, w, dy, act="relu", z=z)
        assert all(bool(t.isfinite().all()) for t in out) and not bool(out[0][3].any())


# ------------------------------------------------------------------- loss
def loss64(x, w, b, labels):
    z = x.double() @ w.double().t()
    s = x.double().abs() @ w.double().abs().t()
    if b is not None:
        z, s = z + b.double(), s + b.double().abs()
    return z, s


def check_ce(dt, rows, din, classes, gt="f32", bias=True, padded=0.0, scale=1.0, accumulate=False, grad=True, seed=2,
             spread=2.0):
    g = torch.Generator().manual_seed(seed + rows + din + classes)
    T, GT = DT[dt], DT[gt]
    x, w = rnd(g, rows, din, dtype=T), rnd(g, classes, din, dtype=T, scale=spread / math.sqrt(din))
    b = rnd(g, classes) if bias else None
    lab = torch.randint(0, classes, (rows,), generator=g, dtype=torch.int32)
    out = torch.rand(rows, generator=g) < padded
    lab[out] = torch.tensor([-1, -100, classes, 2 ** 31 - 1, -2 ** 31], dtype=torch.int64)[
        torch.arange(int(out.sum())) % 5].to(torch.int32)
    labels = dev(lab)
    live = ((labels >= 0) & (labels < classes))
    if bool((~live).any()):
        x[~live] = float("nan")
    xc = torch.where(live[:, None], x, torch.zeros_like(x))
    kw = {}
    if accumulate:
        kw = {"dw": rnd(g, classes, din), "accumulate": True}
        dw0 = kw["dw"].double()
        if bias:
            kw["db"] = rnd(g, classes)
            db0 = kw["db"].double()
    loss, dx, dw, db = singa.linear_softmax_ce(x, w, labels, b, grad=grad, scale=scale, dw_dtype=GT, **kw)
    z, s = loss64(xc, w, b, labels)
    n = int(live.sum())
    at = labels.long().clamp(0, classes - 1)[:, None]
    lse = torch.logsumexp(z, 1)
    d = (G(din) * s).max(1).values  # the largest error of a row's logits
    rows64 = torch.where(live, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    off = torch.where(live, 2 * d + 60 * F * (1 + lse.abs() + z.gather(1, at)[:, 0].abs()), torch.zeros_like(d))
    within("rows", loss[1:], rows64, off)
    mean = rows64.sum() / max(n, 1)
    within("mean", loss[0], mean, off.sum() / max(n, 1) + 2 * F * mean.abs())
    if not grad:
        assert dx is None and dw is None and db is None
        return
    unit = scale / n if n else 0.0
    p = torch.exp(z - lse[:, None])
    rel = torch.expm1(2 * d)[:, None] + F * ((z - lse[:, None]).abs() * 1.4427 + 60)
    dz = p.scatter_add(1, at, torch.full_like(lse[:, None], -1.0)) * unit * live[:, None]
    e = (p * rel + 2 * F) * abs(unit) * live[:, None] + 2 * F * dz.abs()
    u = u_of(T) if T == torch.bfloat16 else 0.0
    tiny = 1e-37  # values below the types' range may go to zero
    ref, wa, xa = dz @ w.double(), w.double().abs(), xc.double().abs()
    off = (e + u * dz.abs() + G(classes) * dz.abs()) @ wa + tiny
    within("dx", dx, ref, off + u_of(T) * (ref.abs() + off))
    uw = u ** 3 if gt == "f32" else u
    ref = dz.t() @ xc.double()
    off = (e + uw * dz.abs() + G(3 * rows) * dz.abs() * (1 + u)).t() @ xa + tiny
    if accumulate:
        ref = ref + dw0
        off = off + F * (ref.abs() + dw0.abs())
    within("dw", dw, ref, off + (u_of(GT) if GT != torch.float32 else F) * (ref.abs() + off))
    if bias:
        ref, off = dz.sum(0), e.sum(0) + G(rows) * dz.abs().sum(0) + tiny
        if accumulate:
            ref = ref + db0
            off = off + F * (ref.abs() + db0.abs())
        within("db", db, ref, off)


CE = [(1, 1, 1), (1, 64, 1000), (2, 9, 3), (5, 100, 10007), (16, 512, 250), (31, 33, 1025), (64, 1023, 77), (65, 24, 2049),
      (100, 7, 1000), (256, 1024, 1000), (333, 509, 5003), (1030, 16, 300)]


@pytest.mark.parametrize("dt,gt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("size", CE)
def test_linear_softmax_ce(size, dt, gt):
    i = CE.index(size)
    check_ce(dt, *size, gt, bias=i % 2 == 0, padded=0.3 if i % 3 == 1 and size[0] > 1 else 0.0)


@pytest.mark.parametrize("dt,gt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("size", [(700, 24, 26003), (20, 72, 900001), (1100, 16, 140001)])
def test_linear_softmax_ce_logits_not_kept(size, dt, gt):
    """More than 64 MiB of logits: formed twice, the last size in more than one piece of the classes."""
    check_ce(dt, *size, gt, bias=True, padded=0.2)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(1, 4096, 1000), (7, 63, 40000), (64, 128, 100), (300, 72, 1111), (700, 24, 26003)])
def test_linear_softmax_ce_loss_only(size, dt):
    check_ce(dt, *size, bias=True, padded=0.2 if size[0] > 1 else 0.0, grad=False)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(130, 40, 501), (1100, 16, 140001)])
def test_linear_softmax_ce_accumulates(size, dt):
    check_ce(dt, *size, padded=0.1, scale=-3.0, accumulate=True)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(3, 16, 50), (100, 16, 50), (700, 16, 26003)])
def test_no_label_at_all(size, dt):
    rows, din, classes = size
    g = torch.Generator().manual_seed(9)
    x, w, b = rnd(g, rows, din, dtype=DT[dt]), rnd(g, classes, din, dtype=DT[dt]), rnd(g, classes)
    labels = dev(torch.full((rows,), -1, dtype=torch.int32))
    for t in singa.linear_softmax_ce(x, w, labels, b):
        assert not bool(t.any())
    x.fill_(float("nan"))
    for t in singa.linear_softmax_ce(x, w, labels, b):
        assert not bool((t != 0).any())
    empty = singa.linear_softmax_ce(x[:0], w, labels[:0], b)
    assert empty[0].shape == (1,) and not any(bool(t.any()) for t in empty if t.numel())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(4, 16, 100), (80, 16, 100), (700, 16, 26003)])
def test_classes_taken_out(size, dt):
    """bias = -inf: those classes have probability and gradient zero, the rest is the softmax over the others."""
    rows, din, classes = size
    g = torch.Generator().manual_seed(10)
    T = DT[dt]
    x, w, b = rnd(g, rows, din, dtype=T), rnd(g, classes, din, dtype=T, scale=0.5), rnd(g, classes)
    keep = torch.arange(classes, device="cuda") % 70 < 3
    b[~keep] = float("-inf")
    at = torch.nonzero(keep)[:, 0].int()
    few = torch.randint(0, len(at), (rows,), generator=g, dtype=torch.int32).cuda()
    labels = dev(at[few.long()].cpu())
    full = singa.linear_softmax_ce(x, w, labels, b)
    part = singa.linear_softmax_ce(x, dev(w[keep].cpu()), dev(few.cpu()), dev(b[keep].cpu()))
    assert not bool(full[2][~keep].any()) and not bool(full[3][~keep].any())
    # the same sums, in another order and, in bf16, with dz rounded at another scale of neither
    tol = {"f32": 2e-5, "bf16": 4 * 2.0 ** -8}[dt]
    for a, c in ((full[0], part[0]), (full[1], part[1]), (full[2][keep], part[2]), (full[3][keep], part[3])):
        assert float((a.double() - c.double()).norm()) <= tol * float(c.double().norm())


def test_a_row_of_nan_is_its_own():
    g = torch.Generator().manual_seed(11)
    for rows, classes in ((6, 40), (90, 300), (700, 26003)):
        x, w = rnd(g, rows, 16, dtype=torch.bfloat16), rnd(g, classes, 16, dtype=torch.bfloat16)
        labels = dev(torch.randint(0, classes, (rows,), generator=g, dtype=torch.int32))
        x[2, 3] = float("nan")
        loss, dx, _, _ = singa.linear_softmax_ce(x, w, labels, None)
        bad = torch.zeros(rows, dtype=torch.bool, device="cuda")
        bad[2] = True
        assert torch.equal(loss[1:].isnan(), bad) and bool(loss[0].isnan())
        assert torch.equal(dx.isnan().any(1), bad)


def test_gradient_against_differences():
    g = torch.Generator().manual_seed(12)
    x, w, b = rnd(g, 70, 12), rnd(g, 30, 12), rnd(g, 30)
    labels = dev(torch.randint(-1, 30, (70,), generator=g, dtype=torch.int32))
    _, dx, dw, db = singa.linear_softmax_ce(x, w, labels, b)
    h = 2.0 ** -7
    for t, grad in ((x, dx), (w, dw), (b, db)):
        step = dev(torch.randn(t.shape, generator=g))
        hi, lo = t + h * step, t - h * step

        def at(v):
            return singa.linear_softmax_ce(v if t is x else x, v if t is w else w, labels, v if t is b else b,
                                           grad=False)[0][0].double()
        diff = (at(hi) - at(lo)) / (2 * h)
        want = (grad.double() * step.double()).sum()
        # the loss (about 5) is held to 2^-22 or so, divided by h; and third derivatives times h^2 / 6
        assert abs(float(diff - want)) <= 8 * 2.0 ** -21 / h + h * h * 20


# ------------------------------------------------------------------- norm
def lists(g, sizes, dts):
    return [rnd(g, n, dtype=dt, scale=10.0 ** (-(i % 5))) for i, (n, dt) in enumerate(zip(sizes, dts))]


@pytest.mark.parametrize("sizes", [[1], [0, 3], [5, 16384, 16385, 1], [7] * 300, [100001, 1 << 20, 31], [(1 << 24) + 5] * 5])
@pytest.mark.parametrize("kind", ["f32", "bf16", "mixed"])
def test_grad_norm_and_clip(sizes, kind):
    g = torch.Generator().manual_seed(13)
    dts = [DT["f32"] if kind == "f32" or (kind == "mixed" and i % 2) else DT["bf16"] for i in range(len(sizes))]
    grads = lists(g, sizes, dts)
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in grads))
    for ratio in (0.0, 0.3, 2.0):
        stat = singa.grad_norm(grads, ratio * norm)
        # fp64 inside: one rounding each
        assert abs(float(stat[0]) - norm) <= 2 * F * norm
        scale = min(1.0, float(torch.tensor(ratio * norm, dtype=torch.float32)) / norm)
        assert abs(float(stat[1]) - scale) <= 2 * F * scale
        outs = [singa.empty(t.shape, t.dtype, "cuda") for t in grads]
        before = [t.clone() for t in grads]
        assert torch.equal(singa.clip_grads(grads, ratio * norm, out=outs), stat)
        for o, t, c in zip(outs, grads, before):
            assert torch.equal(t, c)
            assert torch.equal(o, (t.float() * stat[1]).to(t.dtype))
        if ratio == 0.3:
            singa.clip_grads(grads, ratio * norm)
            for o, t, c in zip(outs, grads, before):
                assert torch.equal(t, o)
                t.copy_(c)


def test_grad_norm_of_views_and_far_values():
    g = torch.Generator().manual_seed(14)
    for T in DT.values():
        flat = rnd(g, 100000, dtype=T)
        views = [flat[1:40000], flat[40003:70001], flat[70002:70003], flat[70005:]]
        norm = math.sqrt(sum(float(t.double().square().sum()) for t in views))
        assert abs(float(singa.grad_norm(views)[0]) - norm) <= 2 * F * norm
        outs = rnd(g, 100000, dtype=T)
        keep = outs.clone()
        stat = singa.clip_grads(views[:2], norm / 7, out=[outs[:39999], outs[40003:70001]])
        assert torch.equal(outs[:39999], (views[0].float() * stat[1]).to(T))
        assert torch.equal(outs[40003:70001], (views[1].float() * stat[1]).to(T))
        assert torch.equal(outs[39999:40003], keep[39999:40003]) and torch.equal(outs[70001:], keep[70001:])
    big = dev(torch.full((1000,), 1e38))
    stat = singa.grad_norm([big], 1.0)
    assert float(stat[0]) == float("inf")  # past fp32, though the sum is not
    # the scale, 3.16e-40, is subnormal: its rounding is half of 2^-149, 2.2e-6 of it (1e38 in fp32 adds 2^-24)
    want = 1 / (1e38 * math.sqrt(1000))
    assert abs(float(stat[1]) - want) <= 2.0 ** -150 + 2 * F * want
    tiny = dev(torch.full((1000,), 1e-38))
    assert abs(float(singa.grad_norm([tiny])[0]) / (1e-38 * math.sqrt(1000)) - 1) < 1e-6
    for bad in (float("inf"), float("nan")):
        t = rnd(g, 50)
        t[7] = bad
        c = t.clone()
        stat = singa.clip_grads([t], 1e-3)
        assert not math.isfinite(float(stat[0])) and float(stat[1]) == 1.0
        assert torch.equal(t.nan_to_num(), c.nan_to_num())


@pytest.mark.parametrize("n", [1, 5, 4096, 100003])
def test_scaled_updates(n):
    g = torch.Generator().manual_seed(15)
    w, grad, v = rnd(g, n), rnd(g, n), rnd(g, n).abs()
    s = dev(torch.tensor([0.25]))  # a power of two: scaling first gives the same bits
    for fn, kw in ((singa.sgd_momentum_update, dict(lr=0.1, momentum=0.9, weight_decay=0.01)),
                   (singa.adagrad_update, dict(lr=0.1, weight_decay=0.01))):
        a, b = [t.clone() for t in (w, v)], [t.clone() for t in (w, v)]
        wb = [singa.empty((n,), torch.bfloat16, "cuda") for _ in range(2)]
        fn(a[0], grad, a[1], wb[0], grad_scale=s, **kw)
        fn(b[0], grad * 0.25, b[1], wb[1], **kw)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(wb[0], wb[1])


# --------------------------------------------------------- used as a whole
def step(x, w1, b1, w2, b2, labels, v, ws=None):
    """An inner product layer with a residual, the loss over a second one, the gradients, their clipping, the update."""
    h, z = singa.linear_fwd(x, w1, b1, act="gelu", residual=x, keep_z=True)
    loss, dh, dw2, db2 = singa.linear_softmax_ce(h, w2, labels, b2)
    dx, dw1, db1 = singa.linear_bwd(x, w1, dh, act="gelu", z=z, dx_residual=dh)
    grads = [dw1, db1, dw2, db2]
    stat = singa.grad_norm(grads, 0.5)
    return [loss, dx, stat] + grads


def parts(seed, rows=200, d=64, classes=500, T=torch.float32):
    g = torch.Generator().manual_seed(seed)
    x = rnd(g, rows, d, dtype=T)
    w1, b1, w2, b2 = rnd(g, d, d, dtype=T, scale=0.1), rnd(g, d), rnd(g, classes, d, dtype=T, scale=0.2), rnd(g, classes)
    labels = dev(torch.randint(-1, classes, (rows,), generator=g, dtype=torch.int32))
    return x, w1, b1, w2, b2, labels


def test_a_whole_step_against_autograd():
    x, w1, b1, w2, b2, labels = parts(20)
    got = step(x, w1, b1, w2, b2, labels, None)
    leaves = [t.double().cpu().requires_grad_() for t in (x, w1, b1, w2, b2)]
    X, W1, B1, W2, B2 = leaves
    h = torch.nn.functional.gelu(X @ W1.t() + B1) + X
    loss = torch.nn.functional.cross_entropy(h @ W2.t() + B2, labels.cpu().long(), ignore_index=-1)
    loss.backward()
    ref = [X.grad, W1.grad, B1.grad, W2.grad, B2.grad]
    assert abs(float(got[0][0]) - float(loss.detach())) <= 1e-6 * float(loss.detach())
    for name, a, r in zip(("dx", "dw1", "db1", "dw2", "db2"), (got[1], *got[3:]), ref):
        err = float((a.double().cpu() - r).norm() / r.norm())
        assert err <= 64 * 4 * F, (name, err)  # sums of up to 500 terms, three in a row
    norm = math.sqrt(sum(float(r.square().sum()) for r in ref[1:]))
    assert abs(float(got[2][0]) / norm - 1) <= 64 * F


@pytest.mark.parametrize("T", [torch.float32, torch.bfloat16])
def test_repeats_streams_and_graphs_give_the_same_bits(T):
    args = parts(21, T=T)
    want = step(*args, None)
    for a, b in zip(want, step(*args, None)):
        assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step(*args, None)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(want, other):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
    singa.set_allocator(None)  # the graph's own pool holds what the step makes
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*args, None)
    x2 = parts(22, T=T)[0]
    for i in range(4):
        if i == 2:
            args[0].copy_(x2)
            want = step(*args, None)
            torch.cuda.synchronize()
        for o in out:
            o.zero_()
        graph.replay()
        eager = step(*args, None)  # the program's own work between the replays
        torch.cuda.synchronize()
        for a, b, c in zip(want, out, eager):
            assert torch.equal(a, b) and torch.equal(a, c), i


def test_two_calls_at_once_with_workspaces_of_their_own():
    a, b = parts(23, rows=900, classes=3001), parts(24, rows=700, classes=2999)
    want = [singa.linear_softmax_ce(p[0], p[3], p[5], p[4]) for p in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, p in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            got.append(singa.linear_softmax_ce(p[0], p[3], p[5], p[4]))
    torch.cuda.synchronize()
    for w, q in zip(want, got):
        assert all(torch.equal(i, j) for i, j in zip(w, q))


def test_refusals_on_the_gpu():
    g = torch.Generator().manual_seed(25)
    x, w = rnd(g, 100, 64), rnd(g, 32, 64)
    labels = dev(torch.zeros(100, dtype=torch.int32))
    with pytest.raises(ValueError, match="contiguous"):
        singa.linear_fwd(x[:, :32], dev(w[:, :32].cpu()))
    with pytest.raises(singa.SingaError):  # not at a 16-byte boundary
        singa.linear_fwd(x.view(-1)[1:65].view(1, 64), w)
    with pytest.raises(TypeError):
        singa.linear_fwd(x, w.bfloat16())
    with pytest.raises(ValueError, match="shape"):
        singa.linear_fwd(x, w, dev(torch.zeros(31)))
    with pytest.raises(ValueError, match="z"):
        singa.linear_bwd(x, w, rnd(g, 100, 32), act="gelu")
    with pytest.raises(TypeError, match="labels"):
        singa.linear_softmax_ce(x, w, labels.long())
    with pytest.raises(ValueError, match="accumulate"):
        singa.linear_softmax_ce(x, w, labels, accumulate=True)
    with pytest.raises(singa.SingaError) as e:
        singa.linear_softmax_ce(x, w, labels, workspace=singa.empty((64,), torch.uint8, "cuda"))
    assert e.value.status == -4


@pytest.mark.parametrize("rows", [3, 150])
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_activations_far_below_zero(dt, act, rows):
    """Values that an activation nearly cancels keep their relative precision.  z is exact (one product of 1 and z).
    gelu: the argument of erfc is rounded twice (relative 2 F, so 4 u^2 F in exp(-u^2), u^2 = z^2 / 2), its square and
    the base-2 argument once each (2 u^2 F more); 2^-19 covers the exponential, the polynomial's 4.5e-7 or erfc's own
    ulps.  silu: 2 |z| F of the exponential's argument and 2^-20 of the rest."""
    T = DT[dt]
    z = torch.linspace(-11, 9, rows * 64).view(rows, 64).to(T)
    x, w = dev(z, T), dev(torch.eye(64), T)
    y = singa.linear_fwd(x, w, act=act)
    zr = x.double()
    yr = zr * torch.special.erfc(-zr / math.sqrt(2)) / 2 if act == "gelu" else act64(zr, act)
    off = (6 * zr.square() / 2 * F + 2.0 ** -19 if act == "gelu" else 2 * zr.abs() * F + 2.0 ** -20) * yr.abs()
    within("y", y, yr, off + u_of(T) * (yr.abs() + off))


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows,din,dout", [(5, 72, 40), (130, 72, 136), (130, 63, 77), (300, 1001, 264)])
def test_a_row_of_nan_or_infinity_reaches_its_own_outputs_only(rows, din, dout, dt):
    """The ends of rows, of K and of tiles: what lies beyond them is never multiplied with."""
    T = DT[dt]
    g = torch.Generator().manual_seed(31)
    x, w = rnd(g, rows, din, dtype=T), rnd(g, dout, din, dtype=T)
    dy = rnd(g, rows, dout, dtype=T)
    r, c = rows // 2, dout // 2
    for far in (float("nan"), float("inf")):
        xx, ww, dd = x.clone(), w.clone(), dy.clone()
        xx[r] = far
        bad = ~singa.linear_fwd(xx, w).isfinite()
        assert bool(bad[r].all()) and int(bad.sum()) == dout
        ww[c] = far
        bad = ~singa.linear_fwd(x, ww).isfinite()
        assert bool(bad[:, c].all()) and int(bad.sum()) == rows
        dd[r] = far
        dx, dw, db = singa.linear_bwd(x, w, dd)
        bad = ~dx.isfinite()
        assert bool(bad[r].all()) and int(bad.sum()) == din and not bool(dw.isfinite().any()) and not bool(db.isfinite().any())
        dd = dy.clone()
        dd[:, c] = far
        dx, dw, db = singa.linear_bwd(x, w, dd)
        bad = ~dw.isfinite()
        assert bool(bad[c].all()) and int(bad.sum()) == din and not bool(dx.isfinite().any()) and int((~db.isfinite()).sum()) == 1


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 8, 24, 64])
def test_few_rows_of_far_apart_weights(rows, dt):
    """Rows of 16 and 32 KB, where the workgroups begin at different places of K."""
    check_fwd(dt, rows, 8192, 4099, "none", True, False, False)


def test_shared_memory_is_refused():
    g = torch.Generator().manual_seed(32)
    x, w = rnd(g, 80, 64), rnd(g, 64, 64)
    with pytest.raises(singa.SingaError):
        singa.linear_fwd(x, w, out=x)
    with pytest.raises(singa.SingaError):
        singa.linear_bwd(x, w, x, dx=x)
    with pytest.raises(singa.SingaError):
        singa.clip_grads([w, w], 1.0)
    with pytest.raises(singa.SingaError):
        singa.clip_grads([w, w[:3]], 1.0)
    assert float(singa.grad_norm([w, w])[0]) == pytest.approx(math.sqrt(2) * float(w.double().norm()), rel=4 * F)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(3, 40, 100), (90, 63, 300), (100, 16, 10007), (1100, 24, 500), (700, 24, 26003)])
def test_parts_of_the_loss(size, dt):
    """Each gradient by itself: the same but for the order of sums and, in bf16, one rounding of dz and of the result."""
    rows, din, classes = size
    T = DT[dt]
    g = torch.Generator().manual_seed(33)
    x, w, b = rnd(g, rows, din, dtype=T), rnd(g, classes, din, dtype=T), rnd(g, classes)
    labels = dev(torch.randint(-1, classes, (rows,), generator=g, dtype=torch.int32))
    loss, dx, dw, db = singa.linear_softmax_ce(x, w, labels, b)
    only = [singa.linear_softmax_ce(x, w, labels, b, need_dw=False), singa.linear_softmax_ce(x, w, labels, b, need_dx=False),
            singa.linear_softmax_ce(x, w, labels, b, need_dx=False, need_dw=False), singa.linear_softmax_ce(x, w, labels)]
    bound = 2 * G(max(rows, classes)) + (4 * u_of(T) if T == torch.bfloat16 else 0)
    for got, want in zip((only[0][1], only[0][3], only[1][2], only[1][3], only[2][3]), (dx, db, dw, db, db)):
        assert float((got.double() - want.double()).norm() / want.double().norm()) <= bound
    assert only[0][2] is None and only[1][1] is None and only[2][1] is None and only[3][3] is None
    for o in only[:3]:
        assert torch.equal(o[0], loss)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_shapes_of_more_and_fewer_dimensions(dt):
    T = DT[dt]
    g = torch.Generator().manual_seed(34)
    x, w, b = rnd(g, 6, 16, dtype=T), rnd(g, 9, 16, dtype=T), rnd(g, 9)
    labels = dev(torch.randint(0, 9, (6,), generator=g, dtype=torch.int32))
    dy = rnd(g, 6, 9, dtype=T)
    want = singa.linear_fwd(x, w, b), *singa.linear_bwd(x, w, dy), *singa.linear_softmax_ce(x, w, labels, b)
    x3 = x.view(2, 3, 16)
    got = (singa.linear_fwd(x3, w, b), *singa.linear_bwd(x3, w, dy.view(2, 3, 9)),
           *singa.linear_softmax_ce(x3, w, labels.view(2, 3), b))
    for a, c in zip(want, got):
        assert torch.equal(a.reshape(-1), c.reshape(-1))
    assert got[0].shape == (2, 3, 9) and got[1].shape == x3.shape and got[5].shape == x3.shape
    one = singa.linear_fwd(x[0], w, b), singa.linear_softmax_ce(x[0], w, labels[0], b)
    assert one[0].shape == (9,) and one[1][0].shape == (2,) and one[1][1].shape == (16,)
    assert torch.equal(one[0], singa.linear_fwd(x[:1], w, b)[0])
    none = singa.linear_softmax_ce(x[:0], w, labels[:0], b)
    assert none[0].tolist() == [0.0] and not bool(none[2].any()) and not bool(none[3].any()) and none[1].shape == (0, 16)
    assert singa.linear_fwd(x[:0], w, b).shape == (0, 9)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(100, 1001, 777), (400, 63, 256), (512, 512, 500), (201, 130, 33), (65, 2000, 48)])
def test_several_blocks_of_few_rows(size, dt):
    check_fwd(dt, *size, "silu", True, True, True)
    check_ce(dt, size[0], size[1], size[2], grad=False, padded=0.2)
    check_ce(dt, size[0], size[1], size[2], padded=0.2)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(911, 40, 106), (70, 16, 1000), (17, 24, 5000), (3000, 16, 2056)])
def test_bias_gradients_of_few_and_many_rows(size, dt):
    check_bwd(dt, *size, "gelu")
    check_bwd(dt, *size, "none", accumulate=True)


@pytest.mark.parametrize("din", [2304, 2305])
def test_tensors_beyond_32_bit_offsets(din):
    """x and dx of 4.8 GB (2^31 elements lie within them), whole rows and rows that are copied."""
    rows, dout = (1 << 20) + 3, 40
    g = torch.Generator(device="cuda").manual_seed(35)
    x = torch.empty(rows, din, dtype=torch.bfloat16, device="cuda")
    for c in x.split(1 << 17):
        c.copy_(torch.randn(c.shape, generator=g, device="cuda"))
    w = rnd(torch.Generator().manual_seed(36), dout, din, dtype=torch.bfloat16)
    y = singa.linear_fwd(x, w)
    dx, dw, db = singa.linear_bwd(x, w, y)
    u = u_of(torch.bfloat16)
    half = (1 << 31) // din
    for a in (0, half - 2, (1 << 30) // din - 2, rows - 5):
        xs, ys = x[a:a + 5].double(), y[a:a + 5].double()
        off = G(din) * (xs.abs() @ w.double().abs().t())
        ref = xs @ w.double().t()
        within("y", y[a:a + 5], ref, off + u * (ref.abs() + off))
        off = G(dout) * (ys.abs() @ w.double().abs())
        ref = ys @ w.double()
        within("dx", dx[a:a + 5], ref, off + u * (ref.abs() + off))
    ref, mag = torch.zeros(dout, din, dtype=torch.double, device="cuda"), torch.zeros(dout, din, dtype=torch.double, device="cuda")
    for xs, ys in zip(x.split(1 << 16), y.split(1 << 16)):
        ref += ys.double().t() @ xs.double()
        mag += ys.double().abs().t() @ xs.double().abs()
    within("dw", dw, ref, G(rows) * mag)
    within("db", db, y.double().sum(0), G(rows) * y.double().abs().sum(0))
    labels = torch.randint(0, dout, (rows,), generator=g, device="cuda", dtype=torch.int32)
    loss, dx, _, _ = singa.linear_softmax_ce(x, w, labels, need_dw=False)
    z = x[-5:].double() @ w.double().t()
    lse, at = torch.logsumexp(z, 1), labels[-5:].long()[:, None]
    d = G(din) * (x[-5:].double().abs() @ w.double().abs().t()).max(1).values
    within("rows", loss[-5:], lse - z.gather(1, at)[:, 0], 2 * d + 60 * F * (1 + 3 * lse.abs()))
    assert bool(loss.isfinite().all()) and bool(dx[-5:].isfinite().all()) and bool((dx[-5:] != 0).any())
