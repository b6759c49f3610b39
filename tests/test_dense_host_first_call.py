"""The norm and clipping as a process's first call of the library."""
import pytest
import torch

from paper_1603_07846_amd import singa


class OnGpu:
    """What the binding asks of a tensor on the current GPU, with a made-up address."""
    is_cuda, dtype, device, shape = True, torch.float32, "cuda:0", torch.Size((2,))

    def __init__(self, n, at):
        self.n, self.at = n, at

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0

    def numel(self):
        return self.n

    def dim(self):
        return 1

    def data_ptr(self):
        return self.at


class Bytes(OnGpu):
    dtype = torch.uint8


@pytest.mark.parametrize("call", [singa.grad_norm, lambda g, **kw: singa.clip_grads(g, 1.0, **kw)])
def test_norm_first(call, monkeypatch):
    monkeypatch.setattr(singa, "_LIB", None)  # not loaded yet
    monkeypatch.setattr(singa, "_current", lambda: 0)
    monkeypatch.setattr(singa, "_current_stream", lambda cur: None)
    with pytest.raises(singa.SingaError) as e:  # 8 bytes of workspace: the library's own refusal
        call([OnGpu(10, 1 << 20)], stat=OnGpu(2, 1 << 21), workspace=Bytes(8, 1 << 22))
    assert e.value.status == -4
