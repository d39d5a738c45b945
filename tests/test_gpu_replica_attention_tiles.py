"""Attention within a window in launches of more tiles than fit the GPU at once."""
import pytest
import torch

from test_gpu_replica_attention import HALVES, Case

pytestmark = pytest.mark.gpu


def _results(c):
    return c.out + c.lse + c.dq + c.dk + c.dv


def _both(c):
    c.forward()
    c.backward()


@pytest.mark.parametrize("kind", HALVES)
def test_warps_that_run_ahead_of_others(kind):
    """Tiles with first keys, whose first 32 rows' warps take longest (they add the sums of chunks), and behind each some more tiles of the
    same CTA: the other warps may be a step ahead, and wait there."""
    import paper_2403_04206_b200 as grawa
    c = Case(kind, 2300, 4, 2, 64, left=100, sinks=3, M=18, seed=30)
    c.check_forward()
    c.check_backward()
    want = [t.clone() for t in _results(c)]
    for _ in range(30):
        for t in _results(c):
            t.zero_()
        _both(c)
        assert all(torch.equal(a, b) for a, b in zip(_results(c), want))
    assert grawa.grawa_window_attention_status() == 0
