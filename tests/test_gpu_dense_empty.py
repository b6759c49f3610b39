"""Gradients of an empty batch, each by itself."""
import pytest
import torch

from paper_1603_07846_amd import singa
from test_gpu_dense import DT, dev, rnd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_each_gradient_of_an_empty_batch(dt):
    T = DT[dt]
    g = torch.Generator().manual_seed(42)
    x, w, dy = (rnd(g, *s, dtype=T) for s in ((3, 24), (40, 24), (3, 40)))
    none = dict(need_dx=False, need_dw=False, with_bias=False)
    for act in ("none", "gelu"):
        z = None if act == "none" else dy[:0]
        dx, dw, db = singa.linear_bwd(x[:0], w, dy[:0], act=act, z=z, **{**none, "need_dx": True})
        assert dx.shape == (0, 24) and dw is None and db is None
        dw = singa.linear_bwd(x[:0], w, dy[:0], act=act, z=z, **{**none, "need_dw": True})[1]
        db = singa.linear_bwd(x[:0], w, dy[:0], act=act, z=z, **{**none, "with_bias": True})[2]
        assert not bool(dw.any()) and not bool(db.any())
    labels = dev(torch.zeros(0, dtype=torch.int32))
    loss, dx, dw, db = singa.linear_softmax_ce(x[:0], w, labels, need_dw=False)
    assert loss.tolist() == [0.0] and dx.shape == (0, 24) and dw is None and db is None
