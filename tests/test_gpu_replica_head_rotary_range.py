"""Norms of query and key heads with rotation at the ends of what eps and the elements may be."""
import pytest
import torch

from attention_util import head_rotary_backward64
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
