"""What the update calls refuse before they reach the library: tensors that are
not n fp32 values (the bf16 gradients that linear_bwd makes with dw_dtype among
them) would be read and written past their ends."""
import pytest
import torch

from paper_1603_07846_amd import singa


class OnGpu:
    """What the binding asks of a tensor on the current GPU, with a made-up address that nothing is read from."""

    def __init__(self, n, dtype=torch.float32, device=0, contiguous=True):
        self.shape, self.dtype, self.dense, self.at = torch.Size((n,)), dtype, contiguous, device
        self.device = torch.device("cuda", device)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return self.dense

    def get_device(self):
        return self.at

    def data_ptr(self):
        return 8  # no multiple of 16: the library refuses it in its turn (SINGA_ERR_ALIGN)


BF = torch.bfloat16
GOOD = dict(w=lambda: OnGpu(100), g=lambda: OnGpu(100), v=lambda: OnGpu(100), wb=lambda: None)


@pytest.mark.parametrize("fn", [singa.sgd_momentum_update, singa.adagrad_update])
@pytest.mark.parametrize("scaled", [False, True])
@pytest.mark.parametrize("change,error", [
    ({}, singa.SingaError), (dict(g=lambda: OnGpu(100, BF)), TypeError), (dict(w=lambda: OnGpu(100, BF)), TypeError),
    (dict(v=lambda: OnGpu(100, torch.float64)), TypeError), (dict(wb=lambda: OnGpu(100)), TypeError),
    (dict(g=lambda: OnGpu(99)), ValueError), (dict(v=lambda: OnGpu(99)), ValueError),
    (dict(wb=lambda: OnGpu(99, BF)), ValueError), (dict(g=lambda: OnGpu(100, contiguous=False)), ValueError),
    (dict(w=lambda: OnGpu(100, contiguous=False)), ValueError), (dict(g=lambda: OnGpu(100, device=1)), ValueError),
    (dict(g=lambda: torch.zeros(100)), ValueError)])
def test_updates_refuse(fn, scaled, change, error, monkeypatch):
    monkeypatch.setattr(singa, "_current", lambda: 0)
    monkeypatch.setattr(singa, "_stream", lambda: None)
    t = {k: f() for k, f in {**GOOD, **change}.items()}
    with pytest.raises(error) as e:
        fn(t["w"], t["g"], t["v"], t["wb"], grad_scale=OnGpu(1) if scaled else None)
    if not change:
        assert e.value.status == -5  # every check of the binding passed
