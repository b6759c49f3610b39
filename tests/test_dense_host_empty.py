"""Calls on an empty batch, each output by itself: its tensors have no memory
to point at."""
import pytest

from test_dense_host import bwd, ce, fwd


@pytest.mark.parametrize("dt", [0, 1])
def test_an_empty_batch_is_a_call_without_work(dt):
    none = dict(rows=0, x=None, ws=None, nbytes=0)
    assert fwd(dt, y=None, **none) == 0
    # dx of no rows is NULL, and nothing else is asked for
    assert bwd(dt, dy=None, z=None, dx=None, dw=None, db=None, **none) == 0
    assert bwd(dt, dy=None, z=None, dx=None, acc=1, **none) == 0
    assert ce(dt, w=None, **none) == -1
