"""Norms of query and key heads with rotation over so many rows that each warp takes several."""
import pytest
import torch

from attention_util import head_rotary64, head_rotary_backward64
from replica_util import TYPES, check
from test_gpu_replica_head_rotary import EPS, heads_of, sizes, vectors

pytestmark = pytest.mark.gpu

# Two workers: a warp takes several rows from 2368 on in the forward pass, from 1184 on in the backward pass.  Whole words, as
# neighbours and halves; what is rotated no whole number of words; odd sizes; long heads of single elements.
SHAPES = [(6001, 12, 12, 64, 64, 0, 0), (5003, 5, 1, 128, 128, 8, 8), (6002, 3, 2, 80, 40, 0, 0), (5001, 2, 3, 75, 40, 1, 1), (4999, 1, 1, 202, 100, 0, 0)]


@pytest.mark.parametrize("pairing, given", [("halves", False), ("neighbours", True)])
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_warps_with_several_rows(shape, kind, pairing, given):
    import paper_2403_04206_b200 as grawa
    rows, heads, kv_heads, dim, _, pad, lead = shape
    gen, M, q, k, qw, kw, f, where, places = sizes(shape, kind, pairing, given, seed=8)
    out, k_out = (heads_of(gen, M, rows, n, dim, kind, pad, lead)[0] for n in (heads, kv_heads))
    grawa.grawa_head_rotary_forward(q, k, qw, kw, out, k_out, f, **where)
    for x, w, y in ((q, qw, out), (k, kw, k_out)):
        for m in range(M):
            want, error = head_rotary64(x[m], w[m], places[m], f, pairing, EPS)
            check(y[m], want, kind, error, "y")
    dy, dk_out, dq, dk = (heads_of(gen, M, rows, n, dim, kind, pad, lead)[0] for n in (heads, kv_heads, heads, kv_heads))
    dqw, dkw = vectors(gen, M, dim, kind), vectors(gen, M, dim, kind)
    was = [[t.clone() for t in dw] for dw in (dqw, dkw)]
    grawa.grawa_head_rotary_backward(dy, dk_out, q, k, qw, kw, dq, dk, dqw, dkw, f, accumulate=True, **where)
    for g, x, w, dx, dw, before in ((dy, q, qw, dq, dqw, was[0]), (dk_out, k, kw, dk, dkw, was[1])):
        for m in range(M):
            (want, error), (want_w, error_w) = head_rotary_backward64(g[m], x[m], w[m], places[m], f, pairing, EPS)
            check(dx[m], want, kind, error, "dx")
            check(dw[m], want_w + before[m].double(), kind, error_w + 2.0 ** -24 * before[m].double().abs(), "dw")
