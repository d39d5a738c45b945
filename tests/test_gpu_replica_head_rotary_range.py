"""Norms of query and key heads with rotation at the ends of what eps and the elements may be."""
import numpy as np
import pytest
import torch

from attention_util import head_rotary64, head_rotary_backward64
from replica_util import TYPES, check
from test_gpu_replica_head_rotary import heads_of, sizes, vectors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("heads, kv_heads, dim", [(5, 3, 64), (1, 0, 128), (7, 2, 32), (3, 1, 75)])
def test_gradients_without_eps_where_heads_do_not_fill_a_warp(kind, heads, kv_heads, dim):
    """eps = 0: what stands in the lanes of a warp that hold no head adds nothing to the weights' gradients."""
    import paper_2403_04206_b200 as grawa
    gen, M, q, k, qw, kw, f, where, places = sizes((40, heads, kv_heads, dim, dim // 2 // 2 * 2, 0, 0), kind, "neighbours", True, seed=7)
    where["eps"] = 0.0
    args = []
    for x, w, n in ((q, qw, heads), (k, kw, kv_heads)):
        args.append((heads_of(gen, M, 40, n, dim, kind)[0], [torch.empty_like(t) for t in x], vectors(gen, M, dim, kind)) if n else (None,) * 3)
    (dq_out, dq, dqw), (dk_out, dk, dkw) = args
    grawa.grawa_head_rotary_backward(dq_out, dk_out, q, k, qw, kw, dq, dk, dqw, dkw, f, **where)
    for dy, x, w, dx, dw in ((dq_out, q, qw, dq, dqw), (dk_out, k, kw, dk, dkw))[:2 if kv_heads else 1]:
        for m in range(M):
            (want, error), (want_w, error_w) = head_rotary_backward64(dy[m], x[m], w[m], places[m], f, "neighbours", 0.0)
            check(dx[m], want, kind, error, "dx")
            check(dw[m], want_w, kind, error_w, "dw")


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dim, rotary", [(64, 64), (128, 36), (75, 40), (8, 0)])
@pytest.mark.parametrize("size, eps", [(1e25, 1e-6), (3e37, 1e-6), (1e-25, 0.0), (1e-38, 0.0), (1e-25, 1e-45), (1e-30, 1e-20), (1e-25, 1e-30), (1e30, 0.0)])
def test_heads_whose_squares_leave_the_range_of_32_bits(kind, dim, rotary, size, eps):
    """Norms of elements of 1e25 or 1e-25, beside heads of ordinary size in the same row, both ways."""
    import paper_2403_04206_b200 as grawa
    gen, M, q, k, qw, kw, f, where, places = sizes((40, 5, 2, dim, rotary, 0, 0), kind, "neighbours", True, seed=6)
    eps = float(np.float32(eps))
    where["eps"] = eps
    for t in q + k:
        t[::3] = (t[::3].double() * size).to(kind)
        t[1, 0] = (t[1, 0].double() * size).to(kind)
    out, k_out = [torch.empty_like(t) for t in q], [torch.empty_like(t) for t in k]
    grawa.grawa_head_rotary_forward(q, k, qw, kw, out, k_out, f, **where)
    # upstream gradients as small as the rows are large, so that dx = dy / norm stays inside the range
    dy, dk_out = ([(torch.randn(t.shape, generator=gen, device="cuda") * min(1.0, max(size, eps ** 0.5) * 1e6)).to(kind) for t in x] for x in (q, k))
    dq, dk = [torch.empty_like(t) for t in q], [torch.empty_like(t) for t in k]
    dqw, dkw = [torch.empty_like(t) for t in qw], [torch.empty_like(t) for t in kw]
    grawa.grawa_head_rotary_backward(dy, dk_out, q, k, qw, kw, dq, dk, dqw, dkw, f, **where)
    small = 2.0 ** -126 if kind == torch.bfloat16 else 2.0 ** -120         # what is lost below the smallest normal number
    for x, w, y, g, dx, dw in ((q, qw, out, dy, dq, dqw), (k, kw, k_out, dk_out, dk, dkw)):
        for m in range(M):
            want, error = head_rotary64(x[m], w[m], places[m], f, "neighbours", eps)
            check(y[m], want, kind, error + small, "y")
            (want, error), (want_w, error_w) = head_rotary_backward64(g[m], x[m], w[m], places[m], f, "neighbours", eps)
            check(dx[m], want, kind, error + small, "dx")
            check(dw[m], want_w, kind, error_w + small, "dw")
