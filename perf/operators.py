"""The fully connected half of a training step and of serving, as cases that
can be timed: an inner product with bias, activation and residual and its
gradients, the softmax cross-entropy of an inner product that does not keep
the logits, and the global gradient norm with clipping.

``listed()`` names the cases, ``draw(rng)`` gives further ones of the same
ranges, ``prepare(case, seed)`` builds on the GPU what a user's program holds
before the call, and ``run(state)`` is one pass: in elementary torch
operations, or, where ``own`` is true, through the entry points of
``paper_1603_07846_amd.singa``.  ``work`` is what a pass cannot do without,
``exact`` the same results in 64 bits.

Kinds of case:
  fwd    y = act(x w^T + b) + residual, with z = x w^T + b kept when it trains
  bwd    its gradients: dx, dw, db from dy and the kept z
  loss   softmax cross-entropy of x w^T + b, the loss alone
  train  the same with the gradients of x, w and b
  clip   gradients scaled down to a global norm
  step   the norm, then the momentum SGD step on every tensor with the scale
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTS = ("none", "relu", "gelu", "silu")
LR, MOMENTUM, DECAY = 0.01, 0.9, 5e-4


def _linear(kind, name, dtype, rows, din, dout, act, bias=True, residual=False, keep=False, gradient="f32"):
    return {"name": name, "kind": kind, "dtype": dtype, "rows": rows, "in": din, "out": dout, "act": act, "bias": bias,
            "residual": residual, "keep": keep, "gradient": gradient}


def _loss(kind, name, dtype, rows, din, classes, padded, bias=True, gradient="f32"):
    return {"name": name, "kind": kind, "dtype": dtype, "rows": rows, "in": din, "classes": classes, "padded": padded,
            "bias": bias, "gradient": gradient}


def _grads(kind, name, dtype, tensors, total, ratio):
    return {"name": name, "kind": kind, "dtype": dtype, "tensors": tensors, "total": total, "ratio": ratio}


def listed():
    return [
        # One row through a 4096-wide layer with everything in its epilogue: a
        # served request, where latency and the weights' bytes count.
        _linear("fwd", "fwd_bf16_1x4096x4096", "bf16", 1, 4096, 4096, "gelu", residual=True),
        # An odd batch through an odd layer in fp32: no size is a multiple of
        # a vector.
        _linear("fwd", "fwd_f32_100x1001x777", "f32", 100, 1001, 777, "silu"),
        # The wide layer of a block on a full batch of positions, training:
        # the pre-activation is kept.
        _linear("fwd", "fwd_bf16_8192x4096x8192", "bf16", 8192, 4096, 8192, "gelu", keep=True),
        # The gradients of the largest fully connected layer of the
        # AlexNet-shaped net at its batch.
        _linear("bwd", "bwd_bf16_256x9216x4096", "bf16", 256, 9216, 4096, "relu"),
        # A block's gradients on some thousand positions, with a smooth
        # activation and the gradient of the residual branch, kept in bf16.
        _linear("bwd", "bwd_bf16_4000x4096x4096", "bf16", 4000, 4096, 4096, "gelu", residual=True, gradient="bf16"),
        # The score of one row over a mid-sized vocabulary: evaluation.
        _loss("loss", "loss_bf16_1x4096x32000", "bf16", 1, 4096, 32000, False),
        # The classifier of the AlexNet-shaped net at its batch: a training
        # step's last layer and loss.
        _loss("train", "train_bf16_256x4096x1000", "bf16", 256, 4096, 1000, False),
        # A padded batch of an odd size over an odd vocabulary in fp32.
        _loss("train", "train_f32_333x509x5003", "f32", 333, 509, 5003, True),
        # A padded batch over a large vocabulary, where the logits would be
        # the largest tensor of the step.
        _loss("train", "train_bf16_4096x2048x100000", "bf16", 4096, 2048, 100000, True, gradient="bf16"),
        # A handful of small odd tensors: launches count.
        _grads("clip", "clip_f32_7x20000", "f32", 7, 20000, 0.5),
        # The gradients of a deep model in bf16, some hundred tensors.
        _grads("clip", "clip_bf16_200x120000000", "bf16", 200, 120000000, 0.25),
        # The clipped update of the AlexNet-shaped net's parameters.
        _grads("step", "step_f32_16x62378344", "f32", 16, 62378344, 0.5),
    ]


def _log(rng, lo, hi):
    """A whole number in [lo, hi], spread evenly over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Half of the sizes are rounded to a multiple of 64, as layers have them."""
    n = _log(rng, lo, hi)
    return max(64, n // 64 * 64) if rng.random() < 0.5 else n


def draw(rng):
    kind = rng.choice(("fwd", "bwd", "loss", "train", "clip", "step"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    most = 2.5e11 if dtype == "f32" else 5e11
    if kind in ("clip", "step"):
        tensors = _log(rng, 1, 300)
        c = _grads(kind, "", "f32" if kind == "step" else dtype, tensors, max(4 * tensors, _log(rng, 100, 150e6)),
                   rng.choice((0.1, 0.5, 0.9, 2.0)))
    elif kind in ("fwd", "bwd"):
        rows, din, dout = _log(rng, 1, 8192), _size(rng, 16, 9216), _size(rng, 16, 9216)
        while 4.0 * rows * din * dout > most:
            rows = max(1, rows // 2)
        c = _linear(kind, "", dtype, rows, din, dout, rng.choice(ACTS), rng.random() < 0.75, rng.random() < 0.5,
                    kind == "fwd" and rng.random() < 0.5, "bf16" if dtype == "bf16" and rng.random() < 0.5 else "f32")
    else:
        rows, din, classes = _log(rng, 1, 4096), _size(rng, 16, 4096), _size(rng, 10, 100000)
        while 6.0 * rows * din * classes > 4 * most:
            rows = max(1, rows // 2)
        c = _loss(kind, "", dtype, rows, din, classes, rng.random() < 0.5, rng.random() < 0.5,
                  "bf16" if dtype == "bf16" and rng.random() < 0.5 else "f32")
    del c["name"]
    return c


def _sizes(case):
    """The tensors' sizes: uneven, odd ones among them, adding up to the total."""
    k, total = case["tensors"], case["total"]
    left, sizes = total, []
    for i in range(k):
        rest = k - 1 - i
        n = left if rest == 0 else max(1, min(left - rest, (left * (1 + i % 7)) // (4 * (rest + 1)) | 1))
        sizes.append(n)
        left -= n
    return sizes


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0, dtype=dt):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)

    s = dict(case)
    if case["kind"] in ("clip", "step"):
        # gradients of one size class per tensor, as layers have them
        sizes = _sizes(case)
        scales = [10.0 ** -(1 + i % 4) for i in range(len(sizes))]
        s["max_norm"] = case["ratio"] * math.sqrt(sum(n * c * c for n, c in zip(sizes, scales)))
        # one flat buffer with a view per tensor, each at a multiple of 64
        # elements: where the clipped gradients go, or, for the update, what
        # holds all parameters, their momentum and their gradients
        at, end = [], 0
        for n in sizes:
            at.append(end)
            end += (n + 63) // 64 * 64
        flat = torch.zeros(end, dtype=dt, device="cuda")
        views = [flat[a:a + n] for a, n in zip(at, sizes)]
        if case["kind"] == "clip":
            s["g"] = [normal(n, scale=c) for n, c in zip(sizes, scales)]
            s["o"], s["o_flat"] = views, flat
            return s
        for v, n, c in zip(views, sizes, scales):
            v.copy_(normal(n, scale=c))
        s["g"], s["g_flat"] = views, flat
        s["w_flat"], s["v_flat"] = normal(end, scale=0.01), normal(end, scale=1e-4)
        return s
    rows, din = case["rows"], case["in"]
    dout = case["out"] if "out" in case else case["classes"]
    s["x"] = normal(rows, din)
    # an output layer's logits spread over a few units, a hidden layer's over one
    s["w"] = normal(dout, din, scale=(2.0 if "classes" in case else 1.0) / math.sqrt(din))
    s["b"] = normal(dout, scale=0.5, dtype=torch.float32) if case["bias"] else None
    if "classes" in case:
        labels = torch.randint(0, dout, (rows,), generator=g, device="cuda", dtype=torch.int32)
        if case["padded"]:  # the batch's last rows, and some others, have no label
            out = torch.rand((rows,), generator=g, device="cuda") < 0.1
            out[rows - rows // 8:] = True
            out[0] = False
            labels[out] = -1
        s["labels"] = labels
    elif case["kind"] == "fwd":
        s["r"] = normal(rows, dout) if case["residual"] else None
    else:
        s["z"] = normal(rows, dout) if case["act"] != "none" else None
        s["dy"] = normal(rows, dout)
        s["r"] = normal(rows, din) if case["residual"] else None
    return s


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    e = 1 / (1 + torch.exp(-z))
    return e * (1 + z * (1 - e))


def _plain_fwd(s):
    dt = s["x"].dtype
    z = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        z = z + s["b"]
    y = _act(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return [y.to(dt), z.to(dt)] if s["keep"] else [y.to(dt)]


def _plain_bwd(s):
    dt, gt = s["x"].dtype, DTYPES[s["gradient"]]
    dz = s["dy"].float()
    if s["act"] != "none":
        dz = dz * _act_slope(s["z"].float(), s["act"])
    dx = dz @ s["w"].float()
    if s["r"] is not None:
        dx = dx + s["r"].float()
    dw = dz.t() @ s["x"].float()
    return [dx.to(dt), dw.to(gt)] + ([dz.sum(0)] if s["bias"] else [])


def _plain_loss(s):
    train = s["kind"] == "train"
    x, w, labels = s["x"].float(), s["w"].float(), s["labels"].long()
    z = x @ w.t()
    if s["b"] is not None:
        z = z + s["b"]
    m = z.max(1, keepdim=True).values
    lse = m + (z - m).exp().sum(1, keepdim=True).log()
    counted = (labels >= 0) & (labels < z.shape[1])
    at = labels.clamp(0, z.shape[1] - 1)[:, None]
    rows = torch.where(counted, (lse - z.gather(1, at))[:, 0], torch.zeros_like(lse[:, 0]))
    count = counted.sum()
    loss = torch.cat([(rows.sum() / count)[None], rows])
    if not train:
        return [loss]
    dz = (z - lse).exp_()
    dz.scatter_add_(1, at, torch.full_like(lse, -1.0))
    dz *= (counted.float() / count)[:, None]
    dx = dz @ w
    dw = dz.t() @ torch.where(counted[:, None], x, torch.zeros_like(x))
    return [loss, dx.to(s["x"].dtype), dw.to(DTYPES[s["gradient"]])] + ([dz.sum(0)] if s["bias"] else [])


def _plain_scale(s):
    norm = torch.stack([t.float().square().sum() for t in s["g"]]).sum().sqrt()
    return norm, torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm))


def _plain_clip(s):
    norm, scale = _plain_scale(s)
    for o, t in zip(s["o"], s["g"]):
        o.copy_(t.float() * scale)
    return [norm[None], s["o_flat"]]


def _plain_step(s):
    norm, scale = _plain_scale(s)
    w, v, g = s["w_flat"], s["v_flat"], s["g_flat"]
    v.mul_(MOMENTUM).add_(g * scale + DECAY * w, alpha=LR)
    w.sub_(v)
    return [norm[None], w, v]


def run(s):
    kind = s["kind"]
    if not own:
        return {"fwd": _plain_fwd, "bwd": _plain_bwd, "loss": _plain_loss, "train": _plain_loss, "clip": _plain_clip,
                "step": _plain_step}[kind](s)
    from paper_1603_07846_amd import singa
    if kind == "fwd":
        if s["keep"]:
            return list(singa.linear_fwd(s["x"], s["w"], s["b"], act=s["act"], residual=s["r"], keep_z=True))
        return [singa.linear_fwd(s["x"], s["w"], s["b"], act=s["act"], residual=s["r"])]
    if kind == "bwd":
        return [t for t in singa.linear_bwd(s["x"], s["w"], s["dy"], act=s["act"], z=s["z"], dx_residual=s["r"],
                                            with_bias=s["bias"], dw_dtype=DTYPES[s["gradient"]]) if t is not None]
    if kind == "loss":
        return [singa.linear_softmax_ce(s["x"], s["w"], s["labels"], s["b"], grad=False)[0]]
    if kind == "train":
        return [t for t in singa.linear_softmax_ce(s["x"], s["w"], s["labels"], s["b"],
                                                   dw_dtype=DTYPES[s["gradient"]]) if t is not None]
    if kind == "clip":
        stat = singa.clip_grads(s["g"], s["max_norm"], out=s["o"])
        return [stat[:1], s["o_flat"]]
    stat = singa.grad_norm(s["g"], s["max_norm"])
    singa.sgd_momentum_update(s["w_flat"], s["g_flat"], s["v_flat"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY,
                              grad_scale=stat[1:])
    return [stat[:1], s["w_flat"], s["v_flat"]]


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "clip":
        # the norm has to be known before the first value is scaled
        return {"bytes": 3.0 * es * case["total"], "flops": 3.0 * case["total"]}
    if case["kind"] == "step":
        return {"bytes": 24.0 * case["total"], "flops": 8.0 * case["total"]}
    rows, din = case["rows"], case["in"]
    dout = case["out"] if "out" in case else case["classes"]
    gs = 4 if case["gradient"] == "f32" else 2
    inputs = es * (rows * din + dout * din) + (4 * dout if case["bias"] else 0)
    flops = 2.0 * rows * din * dout
    if case["kind"] == "fwd":
        return {"bytes": inputs + es * rows * dout * (1 + case["residual"] + case["keep"]), "flops": flops}
    if case["kind"] == "bwd":
        b = inputs + es * rows * dout * (1 + (case["act"] != "none")) + es * rows * din * (1 + case["residual"])
        return {"bytes": b + gs * dout * din, "flops": 2 * flops}
    if case["kind"] == "loss":
        return {"bytes": inputs + 8 * rows, "flops": flops}
    return {"bytes": inputs + 8 * rows + es * rows * din + gs * dout * din + (4 * dout if case["bias"] else 0),
            "flops": 3 * flops}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("clip", "step"):
        total = torch.zeros((), dtype=torch.float64, device="cuda")
        for t in s["g"]:
            t = t.double()
            total += torch.dot(t, t)
        norm = float(total.sqrt())
        scale = min(1.0, s["max_norm"] / norm)
        first = torch.tensor([norm], dtype=torch.float64)
        if kind == "clip":
            out = torch.zeros(s["o_flat"].shape, dtype=torch.float64, device="cuda")
            for o, t in zip(s["o"], s["g"]):
                out[o.storage_offset():o.storage_offset() + len(t)] = t.double() * scale
            return [first, out]
        w = s["w_flat"].double()
        v = MOMENTUM * s["v_flat"].double() + LR * (scale * s["g_flat"].double() + DECAY * w)
        return [first, w - v, v]
    x, w = s["x"].double(), s["w"].double()
    if kind == "bwd":
        dz = s["dy"].double()
        if case["act"] != "none":
            z = s["z"].double()
            if case["act"] == "relu":
                dz = dz * (z > 0)
            elif case["act"] == "gelu":
                dz = dz * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
            else:
                dz = dz * (torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z))
        dx = torch.mm(dz, w)
        if case["residual"]:
            dx += s["r"].double()
        return [dx, torch.mm(dz.t(), x)] + ([dz.sum(0)] if case["bias"] else [])
    z = torch.mm(x, w.t())
    if case["bias"]:
        z += s["b"].double()
    if kind == "fwd":
        y = {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * torch.special.ndtr(z),
             "silu": lambda: z * torch.sigmoid(z)}[case["act"]]()
        if case["residual"]:
            y = y + s["r"].double()
        return [y, z] if case["keep"] else [y]
    keep = torch.nonzero(s["labels"] >= 0)[:, 0]
    zk, xk, lk = z[keep], x[keep], s["labels"][keep].long()
    lse = torch.logsumexp(zk, 1)
    rows = torch.zeros(case["rows"], dtype=torch.float64, device="cuda")
    rows[keep] = lse - zk[torch.arange(len(keep), device="cuda"), lk]
    loss = torch.cat([rows[keep].mean()[None], rows])
    if kind == "loss":
        return [loss]
    p = torch.exp(zk - lse[:, None])
    p[torch.arange(len(keep), device="cuda"), lk] -= 1
    p /= len(keep)
    dx = torch.zeros_like(x)
    dx[keep] = torch.mm(p, w)
    return [loss, dx, torch.mm(p.t(), xk)] + ([p.sum(0)] if case["bias"] else [])
