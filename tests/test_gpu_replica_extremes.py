"""The replica operators at the ends of their values' ranges, element by element against the definitions in 64 bits."""
import math

import pytest
import torch

from replica_util import activation64, bound, layernorm_backward64

pytestmark = pytest.mark.gpu
HALF = [torch.bfloat16, torch.float16]
# The smallest subnormals are 2^-133 and 2^-24; below the normal numbers a store rounds to a multiple of them.  (bound() has the
# half of it for float16 alone.)
HALF_SUBNORMAL = {torch.bfloat16: 2.0 ** -134, torch.float16: 0.0}


@pytest.fixture(scope="module")
def grawa():
    import paper_2403_04206_b200 as g
    return g


def gates(low, high, kind):
    """Every value of a 16-bit type between low < high <= 0, as a column: weights of a gate whose input is 1."""
    values = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(kind)
    values = values[(values.double() >= low) & (values.double() <= high)]
    return values[torch.argsort(values.double())].cuda()[:, None].contiguous()


def value64(act, a):
    """The activation with its relative accuracy in the tail (0.5 (1 + erf) cancels there)."""
    if act == "gelu":
        return 0.5 * a * torch.erfc(-a / math.sqrt(2.0))
    return activation64(act, a)[0]


# The exponential's argument is rounded once or twice (2^-24 of it each), and the fast exponential adds 2 + 1.16 |argument|
# units of 2^-23 in relative error; the rest (quotient, polynomial, products) is below 2^-20.
def relative(argument):
    return 2.0 ** -20 + 2.0 ** -23 * (2.0 + 2.2 * argument.abs())


@pytest.mark.parametrize("kind", HALF)
@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("act,low", [("gelu", -12.0), ("silu", -90.0)])
def test_forward_of_each_gate_value(grawa, kind, rows, act, low):
    """h = act(a) with a exact: a row of one element that is 1, and u = 1."""
    w = gates(low, 0.0, kind)
    x, up = torch.ones(rows, 1, dtype=kind, device="cuda"), torch.ones_like(w)
    h = torch.empty(rows, len(w), dtype=kind, device="cuda")
    grawa.grawa_gated_ffn_forward([x], [w], [up], [h], activation=act)
    a = w.double().T
    want = value64(act, a)
    lim = bound(want, kind, relative(a * a / 2 if act == "gelu" else a) * want.abs()) + HALF_SUBNORMAL[kind]
    over = ((h.double() - want).abs() - lim)
    at = over.flatten().argmax().item() % len(w)
    assert (over <= 0).all(), f"at {a[0, at].item()}: got {h[0, at].item()}, expected {want[0, at].item()}"


@pytest.mark.parametrize("kind", HALF)
@pytest.mark.parametrize("act,low", [("gelu", -12.0), ("silu", -90.0)])
def test_backward_of_each_gate_value(grawa, kind, act, low):
    """One row, x = dh = u = 1: the weights' gradients are da and du themselves, which are rounded once."""
    gate = gates(low, 0.0, kind).T.contiguous()
    hidden = gate.shape[1]
    one, ones, w = torch.ones(1, 1, dtype=kind, device="cuda"), torch.ones_like(gate), torch.ones(hidden, 1, dtype=kind, device="cuda")
    dwg, dwu = torch.empty_like(w), torch.empty_like(w)
    grawa.grawa_gated_ffn_backward([ones], [one], [w], [w], [gate], [ones], None, [dwg], [dwu], activation=act)
    a = gate.double()[0]
    rel = relative(a * a / 2 if act == "gelu" else a)
    value = value64(act, a)
    assert ((dwu[:, 0].double() - value).abs() <= bound(value, kind, rel * value.abs()) + HALF_SUBNORMAL[kind]).all()
    if act == "gelu":
        terms = [0.5 * torch.erfc(-a / math.sqrt(2.0)), a * torch.exp(-a * a / 2) / math.sqrt(2.0 * math.pi)]
    else:                                                     # s (1 + a (1 - s)): the two terms cancel near their zero
        s = torch.sigmoid(a)
        terms = [s, s * a * torch.sigmoid(-a)]
    slope, size = terms[0] + terms[1], terms[0].abs() + terms[1].abs()
    assert ((dwg[:, 0].double() - slope).abs() <= bound(slope, kind, 2 * rel * size) + HALF_SUBNORMAL[kind]).all()


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [60, 768, 2000, 20000])
@pytest.mark.parametrize("scale,dy_scale", [(2.0 ** -60, 2.0 ** 14), (2.0 ** 50, 2.0 ** -34)])
def test_layernorm_gradients_of_tiny_and_huge_rows(grawa, kind, cols, scale, dy_scale):
    """The gradients are of the size of dy / sigma, which the types hold, though its square or the mean's products with it
    are not: rows of standard deviation 2^-60 and 2^50, without eps."""
    gen = torch.Generator(device="cuda").manual_seed(cols)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    rows = 9
    h, gamma = normal(rows, cols), (1.0 + 0.3 * normal(cols)).to(kind)
    x = (h * scale).to(kind)
    dy = ((normal(rows, cols) + h) * dy_scale).to(kind)        # so that mean(g h) is of dy's size
    mean = x.double().mean(-1)
    rstd = (1.0 / (x.double() - mean[:, None]).square().mean(-1).sqrt()).float()
    mean = mean.float()
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
    grawa.grawa_layernorm_backward([dy], [x], [gamma], [mean], [rstd], [dx], [dgamma], [dbeta])
    for name, got, (want, e) in zip(("dx", "dgamma", "dbeta"), (dx, dgamma, dbeta), layernorm_backward64(dy, x, gamma, mean, rstd)):
        err = (got.double() - want).abs()
        assert torch.isfinite(got).all() and (err <= bound(want, kind, e)).all(), f"{name}: off by {(err / want.abs().max()).max().item()} of the largest"


def test_half_precision_limits_of_the_gated_gradients(grawa):
    """da and du are values of the storage type: past 65504 infinite in half, and what bfloat16 holds in bfloat16."""
    for kind, finite in ((torch.float16, False), (torch.bfloat16, True)):
        def full(rows, cols, value):
            return torch.full((rows, cols), value, dtype=kind, device="cuda")

        x, dh, gate, up, w = full(1, 8, 2.0 ** -10), full(1, 16, 512.0), full(1, 16, 1.0), full(1, 16, 256.0), full(16, 8, 1.0)
        dx, dwg, dwu = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
        grawa.grawa_gated_ffn_backward([dh], [x], [w], [w], [gate], [up], [dx], [dwg], [dwu], activation="relu")
        assert (dwu == 0.5).all()                             # du = 512
        assert (dwg == (128.0 if finite else math.inf)).all() and torch.isfinite(dx).all() == finite      # da = 2^17
