"""The 64-bit statements of the attention operators that the GPU tests compare with: gradients against differences."""
import pytest
import torch

from attention_util import attention64, attention_backward64, head_rotary64, head_rotary_backward64, visible


def difference(f, x, d, step=1e-5):
    return (f(x + step * d) - f(x - step * d)) / (2 * step)


@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
@pytest.mark.parametrize("dim, rotary", [(8, 8), (7, 4), (5, 0)])
def test_head_rotary_gradients_against_differences(pairing, dim, rotary):
    gen = torch.Generator().manual_seed(1)
    x, w, dy, d = (torch.randn(s, dtype=torch.float64, generator=gen) for s in ((3, 2, dim), (dim,), (3, 2, dim), (3, 2, dim)))
    at, f = torch.tensor([0, 5, 1000]), torch.rand(rotary // 2, dtype=torch.float64, generator=gen) if rotary else None
    (dx, _), (dw, _) = head_rotary_backward64(dy, x, w, at, f, pairing, 1e-6)
    by_x = difference(lambda t: (head_rotary64(t, w, at, f, pairing, 1e-6)[0] * dy).sum(), x, d)
    by_w = difference(lambda t: (head_rotary64(x, t, at, f, pairing, 1e-6)[0] * dy).sum(), w, d[0, 0])
    # central differences of step 1e-5: 1e-10 of curvature, and 2^-53 / 1e-5 of rounding
    assert abs((dx * d).sum() - by_x) < 1e-7 and abs((dw * d[0, 0]).sum() - by_w) < 1e-7


@pytest.mark.parametrize("left, right, sinks", [(20, 0, 0), (3, 0, 2), (2, 3, 0), (0, 1, 4), (20, 20, 0)])
def test_attention_gradients_against_differences(left, right, sinks):
    gen = torch.Generator().manual_seed(2)
    rows, heads, kv_heads, dim = 13, 4, 2, 8
    q, dout, a = (torch.randn(rows, heads, dim, dtype=torch.float64, generator=gen) for _ in range(3))
    k, v, b = (torch.randn(rows, kv_heads, dim, dtype=torch.float64, generator=gen) for _ in range(3))
    seen = visible(rows, [(0, 4), (4, 5), (5, 12)], left, right, sinks)       # the last row belongs to none
    for t in (q, k, v, dout):
        assert t.dtype == torch.float64
    import replica_util
    replica_util.HALF_ULP[torch.float64] = replica_util.TINY[torch.float64] = 0.0
    (out, _), (lse, _) = attention64(q, k, v, seen, 0.3)
    grads = attention_backward64(dout, q, k, v, out, lse, seen, 0.3)
    for which, d in enumerate((a, b, b)):
        def f(t):
            args = [q, k, v]
            args[which] = t
            return (attention64(*args, seen, 0.3)[0][0] * dout).sum()
        assert abs((grads[which][0] * d).sum() - difference(f, (q, k, v)[which], d)) < 1e-7
    assert (out[12] == 0).all() and (grads[0][0][12] == 0).all()
