"""The step driver with the loss fused into the last layer and with clipped
updates, against the driver without them and against its own gradients."""
import math

import numpy as np
import pytest
import torch

from _helpers import rel_l2
from paper_1603_07846_amd import net as gnet
from paper_1603_07846_amd import workloads as wl

pytestmark = pytest.mark.gpu

F32 = wl.CFG2
# a last layer with a ReLU in front, several columns of tiles wide, in bf16
BF16 = wl.Workload(
    50, "three layers", "bf16", 24, (16, 5, 5), "normal",
    (wl.Conv("conv1", 32, 3, 1, 1, out_shape=(32, 5, 5)), wl.Relu("relu1"), wl.FC("fc1", 64, out_shape=(64, 1, 1)),
     wl.Relu("relu2"), wl.FC("fc2", 300, out_shape=(300, 1, 1)), wl.SoftmaxCE()),
    classes=300, lr=0.05, momentum=0.9, weight_decay=1e-3, update=True)


def build(w, batch, seed=3, **kw):
    inp = wl.make_inputs(w, batch=batch, seed_offset=seed)
    net = gnet.Net(w, batch=batch, device="cuda", **kw)
    net.load_params(inp.params)
    return net, net.to_device_input(inp.x), torch.from_numpy(inp.labels).cuda()


@pytest.mark.parametrize("w,batch", [(F32, 70), (BF16, 24), (BF16, 150)])
def test_fused_loss_matches_the_stored_logits(w, batch):
    """Same loss and gradients but for roundings: in fp32 the sums' order, in
    bf16 logits that are not rounded (2^-9 each) and dz rounded once where the
    other path rounds logits and dz."""
    a, x, labels = build(w, batch, keep_grads=True)
    b, _, _ = build(w, batch, keep_grads=True, fused_loss=True)  # (else a fused update's layer stores no gradient)
    for n in (a, b):
        n.forward(x, labels)
        n.backward()
    torch.cuda.synchronize()
    tol = 1e-5 if w.dtype == "f32" else 3 * 2.0 ** -8
    assert rel_l2(b.layers[-1].loss.cpu(), a.layers[-1].loss.cpu()) <= tol
    assert rel_l2(b.g_flat.cpu(), a.g_flat.cpu()) <= tol
    assert b.param_layers()[-1].head and not b.param_layers()[-1].fused_update


def test_fused_loss_takes_padding_rows():
    net, x, labels = build(BF16, 24, fused_loss=True, fuse_update=False)  # a fused update would change fc1's weights
    net.forward(x, labels)
    net.backward()
    rows = net.layers[-1].loss.clone()
    labels[20:] = -1
    net.forward(x, labels)
    net.backward()
    loss = net.layers[-1].loss
    assert torch.equal(loss[1:21], rows[1:21]) and not bool(loss[21:].any())
    assert abs(float(loss[0]) - float(rows[1:21].double().mean())) <= 2.0 ** -23 * float(loss[0])
    assert not bool(net.param_layers()[-1].dx[20:].any())


@pytest.mark.parametrize("w,batch,updater", [(F32, 30, "sgd"), (F32, 30, "adagrad"), (BF16, 24, "sgd")])
def test_clipped_update_is_the_update_of_scaled_gradients(w, batch, updater):
    a, x, labels = build(w, batch, updater=updater, clip_norm=1e-2)
    b, _, _ = build(w, batch, updater=updater, fuse_update=False, side_update=False)
    for _ in range(2):
        a.train_one_batch(x, labels)
        b.forward(x, labels)
        b.backward()
        norm = math.sqrt(float(b.g_flat.double().square().sum()))
        assert norm > 1e-2
        assert abs(float(a.grad_stat[0]) / norm - 1) <= 2.0 ** -22
        assert abs(float(a.grad_stat[1]) * norm / 1e-2 - 1) <= 2.0 ** -21
        b.g_flat.mul_(a.grad_stat[1])
        b.update()
        assert torch.equal(a.w_flat, b.w_flat) and torch.equal(a.v_flat, b.v_flat)
    loose, _, _ = build(w, batch, updater=updater, clip_norm=1e9)
    plain, _, _ = build(w, batch, updater=updater, fuse_update=False, side_update=False)
    for n in (loose, plain):
        n.train_one_batch(x, labels)
    assert float(loose.grad_stat[1]) == 1.0 and torch.equal(loose.w_flat, plain.w_flat)


def test_captured_step_with_both():
    net, x, labels = build(BF16, 24, fused_loss=True, clip_norm=1e-2)
    ref, _, _ = build(BF16, 24, fused_loss=True, clip_norm=1e-2, concurrent_wgrad=False)
    torch.cuda.synchronize()
    graph = net.capture(x, labels)
    for i in range(4):
        if i == 2:
            x.copy_(torch.flip(x, (0,)))
        graph.replay()
        ref.train_one_batch(x, labels)
        torch.cuda.synchronize()
        assert torch.equal(net.w_flat, ref.w_flat) and torch.equal(net.layers[-1].loss, ref.layers[-1].loss), i
        assert torch.equal(net.grad_stat, ref.grad_stat)
    assert float(net.grad_stat[1]) < 1 and np.isfinite(float(net.grad_stat[0]))
