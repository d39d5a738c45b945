"""Attention within a window where some operand is not finite: what the rows and sums keep that do not depend on it."""
import pytest
import torch

from attention_util import attention_backward64
from replica_util import check
from test_gpu_replica_attention import ALL, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("large", ["q", "k"])
@pytest.mark.parametrize("where", ["dout", "v"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_small_half_precision_gradients_beside_an_infinity(where, bad, large):
    """Half precision's dS carries a power of two that the longest finite rows of dout and v set: something else in one sequence leaves the
    small gradients (1e-6, weights of 1 / 600) of another as they are.  (Keys, or queries, of 50 make sums of them that half precision holds.)"""
    c = Case(torch.float16, 1200, 2, 1, 64, right=ALL, lengths=[[600, 600], [550, 640]], size=0.05, seed=22)
    for t in c.dout:
        t.mul_(1e-5)
    for t, by in [(t, 1e3) for t in getattr(c, large)] + [(t, 1e-3) for t in (c.k if large == "q" else c.q)]:
        t.mul_(by)
    if where == "v":
        for t in c.v:
            t[100, 0, 7] = bad
    c.forward()
    if where == "dout":
        for t in c.dout:
            t[100, 1, 7] = bad
    blind = [torch.arange(1200, device="cuda") < b[0][1] for b in c.bounds]
    c.backward()
    for m in range(c.M):
        want = attention_backward64(c.dout[m], c.q[m], c.k[m], c.v[m], c.out[m], c.lse[m], c.seen[m], c.scale)
        for name, got, (exact, e) in zip(("dq", "dk", "dv"), (c.dq, c.dk, c.dv), want):
            rows = c.inside[m] & ~blind[m]
            check(got[m][rows], exact[rows], c.kind, e[rows], name)
