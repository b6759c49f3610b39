"""An evaluation between a step's backward pass and its update, with the loss
fused into the last layer: it reads the net and changes no gradient."""
import pytest
import torch

from paper_1603_07846_amd import singa
from test_gpu_dense_net import BF16, F32, build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w,batch", [(F32, 30), (BF16, 24), (BF16, 150)])
@pytest.mark.parametrize("kw", [{}, {"clip_norm": 1e-2}, {"concurrent_wgrad": False}])
def test_evaluation_leaves_the_gradients(w, batch, kw):
    a, x, labels = build(w, batch, fused_loss=True, **{"fuse_update": False, **kw})
    b, _, _ = build(w, batch, fused_loss=True, **{"fuse_update": False, **kw})
    other = torch.flip(x, (0,)).contiguous()
    few = labels.clone()
    few[batch // 2:] = -1
    for n in (a, b):
        n.forward(x, labels)
        n.backward()
    grads, dx = a.g_flat.clone(), a.param_layers()[-1].dx.clone()
    a.forward(other, few)
    torch.cuda.synchronize()
    loss = a.layers[-1].loss
    assert not bool(loss[1 + batch // 2:].any()) and bool((loss[1:1 + batch // 2] > 0).all())
    assert torch.equal(a.g_flat, grads) and torch.equal(a.param_layers()[-1].dx, dx)
    for n in (a, b):
        n.update()
    assert torch.equal(a.w_flat, b.w_flat) and torch.equal(a.v_flat, b.v_flat)


def loss64(net, x):
    """The last layer's loss on its input as the net holds it, in 64 bits."""
    fc = net.param_layers()[-1]
    return fc.x.reshape(len(x), -1).double() @ fc.w_compute.reshape(fc.K, -1).double().t() + fc.b.double()


@pytest.mark.parametrize("w,batch", [(F32, 30), (BF16, 24)])
def test_the_loss_stands_after_each_of_the_passes(w, batch):
    """After forward, after forward and backward, and after a whole step (which leaves it to the backward pass): the
    logits hold at most 4096 products here, G = 4100 2^-24 of magnitudes of which the largest row has some tens."""
    net, x, labels = build(w, batch, fused_loss=True, fuse_update=False)
    net.forward(x, labels)
    z = loss64(net, x)
    rows = torch.logsumexp(z, 1) - z.gather(1, labels.long()[:, None])[:, 0]
    want = torch.cat([rows.mean()[None], rows])
    got = [net.layers[-1].loss.clone()]
    net.backward()
    got.append(net.layers[-1].loss.clone())
    net.layers[-1].loss.fill_(float("nan"))
    net.train_one_batch(x, labels)
    got.append(net.layers[-1].loss.clone())
    for g in got:
        assert float((g.double() - want).abs().max()) <= 4100 * 2.0 ** -24 * float(1 + z.abs().max())
    assert torch.equal(got[1], got[2])


def test_only_the_backward_pass_forms_gradients():
    net, x, labels = build(BF16, 24, fused_loss=True, fuse_update=False)
    net.g_flat.fill_(7.0)
    net.forward(x, labels)
    assert bool((net.g_flat == 7.0).all())
    singa.trace_enable(True)
    net.train_one_batch(x, labels)
    torch.cuda.synchronize()
    names = [r[0] for r in singa.trace_records()]
    singa.trace_enable(False)
    # a whole step forms the logits once
    assert sum(n in ("skinny_kernel", "product_kernel<logits>", "product_kernel<lse>") for n in names) == 1


def test_evaluations_between_replays():
    net, x, labels = build(BF16, 24, fused_loss=True, clip_norm=1e-2)
    ref, _, _ = build(BF16, 24, fused_loss=True, clip_norm=1e-2)
    torch.cuda.synchronize()
    graph = net.capture(x, labels)
    other = torch.flip(x, (0,)).contiguous()
    for i in range(4):
        graph.replay()
        loss = net.layers[-1].loss.clone()
        ref.train_one_batch(x, labels)
        assert torch.equal(net.w_flat, ref.w_flat) and torch.equal(loss, ref.layers[-1].loss), i
        grads = net.g_flat.clone()
        net.forward(other, labels)
        torch.cuda.synchronize()
        assert torch.equal(net.g_flat, grads) and not torch.equal(net.layers[-1].loss, loss)
