"""The step driver with the loss fused into its last layer, built on the CPU:
what it allocates."""
import torch

from paper_1603_07846_amd import singa
from paper_1603_07846_amd import workloads as wl
from paper_1603_07846_amd.net import Net

BATCH, CLASSES = 96, 5000
LAYERS = (wl.FC("fc1", 32, out_shape=(32, 1, 1)), wl.Relu("relu"), wl.FC("fc2", CLASSES, out_shape=(CLASSES, 1, 1)),
          wl.SoftmaxCE())
W = wl.Workload(52, "many classes", "bf16", BATCH, (4, 6, 6), "normal", LAYERS, classes=CLASSES, update=True)


def allocated(**kw):
    made = []

    def alloc(shape, dtype, device):
        made.append((tuple(shape), dtype))
        return torch.empty(shape, dtype=dtype, device=device)

    singa.set_allocator(alloc)
    try:
        net = Net(W, device="cpu", **kw)
    finally:
        singa.set_allocator(None)
    return net, made


def test_the_fused_layer_holds_no_logits():
    plain, made = allocated()
    assert ((BATCH, 1, 1, CLASSES), torch.bfloat16) in made
    fused, made = allocated(fused_loss=True)
    assert not [s for s, _ in made if s[-1] == CLASSES]
    head = fused.param_layers()[-1]
    assert head.head and head.y is None and not head.fused_update and not head.reduce_update
    assert head.out_shape == plain.param_layers()[-1].out_shape
    # nor workspaces for convolutions that it does not run
    only = Net(wl.Workload(53, "without it", "bf16", BATCH, (4, 6, 6), "normal", LAYERS[:2], update=True), device="cpu")
    assert fused.ws_bytes == only.ws_bytes and fused.ws_wgrad_bytes == only.ws_wgrad_bytes
    assert plain.ws_bytes > only.ws_bytes
