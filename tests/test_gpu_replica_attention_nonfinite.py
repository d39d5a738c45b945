"""Attention within a window where some operand is not finite: what the rows and sums keep that do not depend on it."""
import pytest
import torch

from attention_util import attention64, attention_backward64
from replica_util import check
from test_gpu_replica_attention import HALVES, ALL, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("dim, left, sinks", [(64, ALL, 0), (128, 250, 3)])
@pytest.mark.parametrize("lost", ["one", "all"])
def test_values_of_nan_leave_lse_and_the_values_gradients(kind, dim, left, sinks, lost):
    """Neither lse nor dv depends on v: one row of v that is NaN throughout, among many that a query sees, or all of them."""
    c = Case(kind, 900, 4, 2, dim, left=left, sinks=sinks, seed=21)
    for t in c.v:
        t[200 if lost == "one" else slice(None)] = float("nan")
    c.forward()
    c.backward()
    for m in range(c.M):
        _, (lse, e) = attention64(c.q[m], c.k[m], c.v[m], c.seen[m], c.scale)
        check(c.lse[m], lse, torch.float32, e, "lse")
        dv, e = attention_backward64(c.dout[m], c.q[m], c.k[m], c.v[m], c.out[m], c.lse[m], c.seen[m], c.scale)[2]
        check(c.dv[m], dv, kind, e, "dv")
        sees = c.seen[m][:, 200] if lost == "one" else torch.ones(900, dtype=torch.bool, device="cuda")
        assert c.out[m][sees].isnan().all() and torch.isfinite(c.out[m][~sees]).all()


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


def _time(call):
    call()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    call()
    end.record()
    end.synchronize()
    return start.elapsed_time(end)


@pytest.mark.parametrize("dim", [64, 128])
def test_what_rows_of_no_sequence_hold_costs_nothing(dim):
    """Rows in front of the first and behind the last sequence may hold anything, as buffers do that nothing was written to: the same
    bits in the same time."""
    c = Case(torch.bfloat16, 8200, 2, 1, dim, lengths=[[8000, 0], [4000, 4100]], front=70, M=2, seed=23)
    c.forward()
    c.backward()
    results = c.out + c.lse + c.dq + c.dk + c.dv
    want, plain = [t.clone() for t in results], (_time(c.forward), _time(c.backward))
    for m, t in enumerate(c.bounds):
        for x in (c.q, c.k, c.v, c.dout):
            x[m][:t[0][0]] = float("nan")
            x[m][t[-1][1]:] = float("inf")
    taken = (_time(c.forward), _time(c.backward))
    assert all(torch.equal(a, b) for a, b in zip(results, want))
    for t, p in zip(taken, plain):
        assert t < 2.0 * p + 0.1, (taken, plain)


def test_first_keys_of_many_queries_one_of_which_is_infinite():
    """The first keys of a long text with many query heads on one key head, whose values' gradients meet one infinity: a walk over 19
    million queries, which is done with care once, at about the speed of the first time."""
    import time
    import paper_2403_04206_b200 as grawa
    rows, heads, dim, first = 300000, 64, 8, 130
    gen = torch.Generator(device="cuda").manual_seed(24)
    q, k, v, dout = (torch.randn(rows, h, dim, generator=gen, device="cuda").bfloat16() for h in (heads, 1, 1, heads))
    out, lse = torch.empty_like(q), torch.empty(heads, rows, device="cuda")
    dk, dv = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
    window = dict(left=0, sinks=first)
    grawa.grawa_window_attention_forward([q], [k], [v], [out], lse=[lse], **window)
    assert grawa.grawa_window_attention_status() == 0
    dout[5, 0, 3] = float("inf")
    start = time.perf_counter()
    grawa.grawa_window_attention_backward([dout], [q], [k], [v], [out], [lse], None, [dk], [dv], **window)
    assert grawa.grawa_window_attention_status() == 0 and time.perf_counter() - start < 10.0
    lost = torch.zeros_like(dv, dtype=torch.bool)
    lost[:6, 0, 3] = True                                     # the keys that query 5 sees
    assert torch.equal(~torch.isfinite(dv), lost) and (dv.float() != 9.0).all()
    j = torch.arange(first, device="cuda")
    want, size = torch.zeros(first, dim, dtype=torch.float64, device="cuda"), torch.zeros(first, dim, dtype=torch.float64, device="cuda")
    for a in range(0, rows, 10000):
        i = torch.arange(a, min(a + 10000, rows), device="cuda")
        s = dim ** -0.5 * (q[i].double().transpose(0, 1) @ k[:first, 0].double().T) - lse[:, i].double()[..., None]
        p = torch.where(j <= i[:, None], torch.exp(s), 0.0)
        g = dout[i].double().transpose(0, 1).nan_to_num(posinf=0.0)
        want += (p.mT @ g).sum(0)
        size += (p.mT @ g.abs()).sum(0)
    keep = ~lost[:first, 0]
    # one rounding of the store, and a rounding of each weight and sum: fp32 sums of rows * heads terms, whose errors grow as the
    # root of their number (4400) where the terms' signs are mixed, as here; 4 times that
    err, lim = (dv[:first, 0].double() - want).abs()[keep], (2.0 ** -8 * want.abs() + (4 * 4400 * 2.0 ** -24 + 2.0 ** -18) * size)[keep]
    assert (err <= lim).all(), (err / lim).max()


def _with_infinities(x, rows):
    """A row each of +inf, -inf and NaN elements, and one with both infinities, in some columns of head 0; returns their rows."""
    for row, col, bad in zip(rows, (3, 5, 7, 6), (float("inf"), -float("inf"), float("nan"), -float("inf"))):
        x[row, 0, col] = bad
    x[rows[3], 0, 3] = float("inf")
    x[rows[0], 0, 6] = float("inf")
    return rows


def _expected(got, weights, x, name):
    """What sums of positive weights times the rows of x that are seen have where those are not finite: [to, from] weights, x [from, dim]."""
    seen = (weights > 0).double()
    plus, minus = seen @ ((x == float("inf")) | x.isnan()).double() > 0, seen @ ((x == -float("inf")) | x.isnan()).double() > 0
    assert torch.equal(got.isnan(), plus & minus), name
    assert torch.equal(got == float("inf"), plus & ~minus), name
    assert torch.equal(got == -float("inf"), minus & ~plus), name


@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("dim, left, sinks", [(64, 300, 2), (128, ALL, 0), (40, 70, 140)])
def test_signs_of_the_infinities_of_values_and_upstream_gradients(kind, dim, left, sinks):
    """Infinities of both signs and NaN in elements of v (out) and dout (dv), where exactly the sums that see them have them."""
    c = Case(kind, 1300, 2, 2, dim, left=left, sinks=sinks, lengths=[[700, 600], [1299, 1]], seed=25)
    for t in c.v:
        _with_infinities(t, (1, 400, 650, 900))
    c.forward()
    for m in range(c.M):
        _expected(c.out[m][:, 0][c.inside[m]], c.seen[m][c.inside[m]], c.v[m][:, 0], "out")
        assert torch.isfinite(c.out[m][:, 1]).all()
        (out, e), _ = attention64(c.q[m], c.k[m], c.v[m], c.seen[m], c.scale)
        fine = torch.isfinite(c.out[m])
        check(c.out[m][fine], out[fine], kind, e[fine], "out")
    c = Case(kind, 1300, 2, 2, dim, left=left, sinks=sinks, lengths=[[700, 600], [1299, 1]], seed=26)
    c.forward()
    for t in c.dout:
        _with_infinities(t, (1, 400, 650, 900))
    c.backward()
    for m in range(c.M):
        _expected(c.dv[m][:, 0], c.seen[m].mT, c.dout[m][:, 0], "dv")
        want = attention_backward64(c.dout[m], c.q[m], c.k[m], c.v[m], c.out[m], c.lse[m], c.seen[m], c.scale)
        for name, got, (exact, e) in zip(("dq", "dk", "dv"), (c.dq, c.dk, c.dv), want):
            fine = torch.isfinite(got[m])
            rows = c.seen[m][list((1, 400, 650, 900))].any(0) if name == "dk" else torch.zeros(1300, dtype=torch.bool, device="cuda")
            if name == "dq":
                rows[[1, 400, 650, 900]] = True
            assert fine[~rows].all() or name == "dv", name
            check(got[m][fine], exact[fine], kind, e[fine], name)


@pytest.mark.parametrize("kind", HALVES)
def test_every_bit_beside_infinities_in_a_launch_of_many_tiles(kind):
    """More tiles than CTAs at once, some of them walked again: what sees no infinity has the bits of a call without any."""
    def case():
        return Case(kind, 2500, 16, 4, 64, left=200, sinks=3, lengths=[[1200, 1300], [100, 2400]], seed=27)

    places = (90, 1500, 2450)
    clean, spoilt = case(), case()
    for c in (clean, spoilt):
        for t in c.v + c.dout:
            t[list(places)] *= 0.125                          # not the longest rows, by which half precision's power of two goes
        c.forward()
    for t in spoilt.v:
        for place in places:
            t[place, 1, 9] = float("inf")
    spoilt.forward()
    for m in range(clean.M):
        hit = clean.seen[m][:, list(places)].any(1)
        assert torch.equal(spoilt.out[m][~hit], clean.out[m][~hit]) and torch.equal(spoilt.lse[m], clean.lse[m])
        want = clean.out[m].clone()
        want[hit, 4:8, 9] = float("inf")
        assert torch.equal(spoilt.out[m], want)
    spoilt = case()
    for t in spoilt.v + spoilt.dout:
        t[list(places)] *= 0.125
    spoilt.forward()
    for t in spoilt.dout:
        for place in places:
            t[place, 1, 9] = -float("inf")
    clean.backward()
    spoilt.backward()
    for m in range(clean.M):
        hit = clean.seen[m][list(places)].any(0)
        rows = torch.ones(2500, dtype=torch.bool, device="cuda")
        rows[list(places)] = False
        assert torch.equal(spoilt.dk[m][~hit], clean.dk[m][~hit]) and torch.equal(spoilt.dk[m][:, 1:], clean.dk[m][:, 1:])
        assert torch.equal(spoilt.dq[m][rows], clean.dq[m][rows])
        want = clean.dv[m].clone()
        want[hit, 0, 9] = -float("inf")
        assert torch.equal(spoilt.dv[m], want)


def test_sums_of_values_near_the_largest_number():
    """Values of 3e38: their weighted mean is inside bfloat16's range where the sum of weights times values is not inside that of 32 bits."""
    c = Case(torch.bfloat16, 300, 2, 1, 64, right=ALL, seed=28)
    for t in c.v:
        t.copy_((t.sign() * 2.5e38).to(t.dtype))
        t[:, :, 8:] = 3.0e38
        t[:, :, 8:16].neg_()
    c.check_forward()
