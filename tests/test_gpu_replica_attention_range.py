"""Attention within a window at the ends of the exponentials' range."""
import math

import pytest
import torch

from replica_util import HALF_ULP

pytestmark = pytest.mark.gpu


def one_row(kind, scores, values, dim=64, query=1.0):
    """The results of `query` times the first unit vector, in each row, whose scores against the keys are `scores` times that."""
    import paper_2403_04206_b200 as grawa
    n = len(scores)
    q, k, v = (torch.zeros(n, 1, dim, dtype=kind, device="cuda") for _ in range(3))
    q[..., 0] = query
    k[:, 0, 0] = torch.as_tensor(scores, dtype=torch.float64).cuda().to(kind)
    v[:, 0, 0] = torch.as_tensor(values, dtype=torch.float64).cuda().to(kind)
    out, lse = torch.full_like(q, 5.0), torch.full((1, n), 5.0, device="cuda")
    grawa.grawa_window_attention_forward([q], [k], [v], [out], lse=[lse], right=None, scale=1.0)
    return out[:, 0, 0], lse[0]


def test_weights_below_the_smallest_normal_number_are_zero_wherever_they_stand():
    """Weights of 2^-126.2 (-87.5 log2 e) are zero for every key, by both ways to an exponential; those of 2^-125.5 (-87) are there."""
    n = 200
    for place in range(n):
        scores, values = [-200.0] * n, [0.0] * n
        top = (place + 100) % n
        scores[top], scores[place], values[place] = 0.0, -87.5, 2.0 ** 127
        out, lse = one_row(torch.bfloat16, scores, values)
        assert (out == 0).all() and (lse == 0).all(), place
        scores[place] = -87.0
        out, _ = one_row(torch.bfloat16, scores, values)
        # the bfloat16 weight and the bfloat16 result are each rounded once, the argument 125.5 carries 2 roundings of 2^-24
        assert (out.double() / (2.0 ** 127 * math.exp(-87.0)) - 1).abs().max() < 2.0 ** -7, place


def test_scores_whose_rounding_is_past_the_exponentials_range():
    """Scores of 2^34, at every place of a step: a product with log2 e is off by up to 2^10 there, but the largest score's row still is
    that of its value, and lse that score."""
    n = 128
    for place, turn in [(place, (37 * place + 5 * turn) % 128) for place in range(n) for turn in range(5)]:
        scores, values = [float(-j) for j in range(n)], [float(j) for j in range(n)]
        scores[place] = 2.0 ** 34 * (1.0 + turn / 128.0)
        out, lse = one_row(torch.bfloat16, scores, values)
        assert (out == values[place]).all(), (place, turn)
        assert (lse.double() / scores[place] - 1).abs().max() < 2.0 ** -21, (place, turn, lse[0])


def test_small_weights_of_half_precision_keep_their_digits():
    """One key with all the weight and a value of 0, and many whose weights, 2^-24 to 2^-28, are below half precision's smallest normal
    number: their sum is the result.  The weights are carried with 2^6, which keeps most of them above 2^-24."""
    n = 6000
    for low in (-16.5, -17.5, -19.0):
        out, lse = one_row(torch.float16, [0.0] + [low] * (n - 1), [0.0] + [100.0] * (n - 1))
        total = 1.0 + (n - 1) * math.exp(low)
        # each weight carries 2^6 and is off by at most half of half precision's smallest subnormal, 2^-25; the result by its rounding
        want = (n - 1) * math.exp(low) * 100.0 / total
        assert (out.double() / want - 1).abs().max() < 2.0 ** -25 / (math.exp(low) * 2.0 ** 6) + 2.0 ** -11 + 2.0 ** -16, (low, out[-1], want)
        # 47 steps' additions to the sum, and 16 in the first step beside the large term, of 2^-24 each; the logarithm's terms are below 8 and
        # each rounded by at most 2^-21
        assert (lse.double() - math.log(total)).abs().max() < 70 * 2.0 ** -24 + 2 * 2.0 ** -21


def test_weights_of_the_backward_pass_below_the_smallest_normal_number():
    """As above, for the weights that make dv: those of 2^-126.2 are zero wherever the key stands, those of 2^-125.5 are there."""
    import paper_2403_04206_b200 as grawa
    n, dim = 200, 64
    for place in range(n):
        for low in (-87.5, -87.0):
            top = (place + 100) % n
            q, k, v, dout = (torch.zeros(n, 1, dim, dtype=torch.bfloat16, device="cuda") for _ in range(4))
            q[..., 0] = 1.0
            k[:, 0, 0] = -200.0
            k[top, 0, 0], k[place, 0, 0] = 0.0, low
            dout[n - 1, 0, 0] = 2.0 ** 127
            out, lse, dk, dv = torch.zeros_like(q), torch.zeros(1, n, device="cuda"), torch.empty_like(k), torch.empty_like(v)
            grawa.grawa_window_attention_backward([dout], [q], [k], [v], [out], [lse], None, [dk], [dv], right=None, scale=1.0)
            if low == -87.5:
                assert dv[place, 0, 0] == 0, place
            else:                                             # the bfloat16 weight and result are each rounded once
                assert abs(dv[place, 0, 0].item() / (2.0 ** 127 * math.exp(low)) - 1) < 2.0 ** -7, place


@pytest.mark.parametrize("power", [22, 24, 26, 28, 30])
@pytest.mark.parametrize("kind", [torch.bfloat16, torch.float16])
def test_scores_whose_rounding_is_past_half_precision(kind, power):
    """Scores of 2^22 to 2^30, where the rounding of the largest one's product with log2 e is 2^-2 to 2^6: weights are taken of what
    the largest one is, in half precision too, whose numbers end at 2^16 and 2^-24."""
    n = 128
    for turn in range(64):
        place = 2 * turn + 1
        scores, values = [-float(j) for j in range(n)], [float(j) for j in range(n)]
        scores[place] = 2.0 ** (power - 15) * (1.0 + turn / 64.0)
        out, lse = one_row(kind, scores, values, query=2.0 ** 15)
        # the weight is rounded once to the storage type before the product, the result once
        assert ((out.double() - values[place]).abs() <= 2 * HALF_ULP[kind] * values[place]).all(), (place, out[0])
        assert (lse.double() / (scores[place] * 2.0 ** 15) - 1).abs().max() < 2.0 ** -21, (place, lse[0])
        scores[place - 1] = scores[place]                     # two of the same weight
        out, lse = one_row(kind, scores, values, query=2.0 ** 15)
        assert ((out.double() - values[place] + 0.5).abs() <= 2 * HALF_ULP[kind] * values[place]).all(), (place, out[0])
