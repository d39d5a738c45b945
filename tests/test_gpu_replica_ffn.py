"""The gated feed-forward product over all workers and its gradients: exact on small integers (every product and
sum is representable, so a stored value has one right answer), and against 64 bits on real values."""
import pytest
import torch

from replica_util import EPS32, check, gated_ffn64, gated_ffn_backward64

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
# one element, odd sizes, both sides of the tiles (64 along a sum, 128 rows, 128 and 256 columns), several tiles
SIZES = [(1, 1, 1), (1, 8, 8), (2, 7, 5), (3, 64, 128), (5, 63, 127), (8, 65, 129), (9, 72, 136), (64, 128, 64), (127, 120, 250), (128, 64, 256), (129, 200, 264),
         (130, 257, 255), (200, 768, 300), (257, 264, 520), (300, 1000, 1030), (640, 96, 1100)]


@pytest.fixture(scope="module")
def grawa():
    import paper_2403_04206_b200 as g
    return g


class Case:
    def __init__(self, M, rows, d_in, hidden, kind, seed, integers, lead=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.kind, self.M = kind, M

        def draw(*shape, scale=1.0):
            if integers:
                return torch.randint(-2, 3, shape, generator=gen, device="cuda").to(kind)
            return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(kind)

        size = d_in * hidden
        flat = draw(M, lead + 2 * size, scale=d_in ** -0.5)
        self.wg = [t[lead:lead + size].view(hidden, d_in) for t in flat]
        self.wu = [t[lead + size:].view(hidden, d_in) for t in flat]
        self.x, self.dh, self.a, self.u = ([draw(*shape) for _ in range(M)] for shape in ((rows, d_in), (rows, hidden), (rows, hidden), (rows, hidden)))
        if integers:                                           # da = dh u and du = dh a stay below 2^8: exact in both types
            self.a = [torch.where(t > 0, t, -t) for t in self.a]
        self.grads = torch.full((M, lead + 2 * size), 5.0, device="cuda").to(kind)
        self.dwg = [t[lead:lead + size].view(hidden, d_in) for t in self.grads]
        self.dwu = [t[lead + size:].view(hidden, d_in) for t in self.grads]
        self.lead = lead

    def forward(self, grawa, act, **kw):
        h, a, u = ([torch.full_like(t, 9.0) for t in self.dh] for _ in range(3))
        grawa.grawa_gated_ffn_forward(self.x, self.wg, self.wu, h, activation=act, gate_out=a, up_out=u, **kw)
        assert grawa.grawa_gated_ffn_status() == 0
        return h, a, u

    def backward(self, grawa, act, dx=True, dw=True, **kw):
        out = [torch.full_like(t, 9.0) for t in self.x]
        grawa.grawa_gated_ffn_backward(self.dh, self.x, self.wg, self.wu, self.a, self.u, out if dx else None, self.dwg if dw else None,
                                       self.dwu if dw else None, activation=act, **kw)
        assert grawa.grawa_gated_ffn_status() == 0
        return out, self.dwg, self.dwu


def same(got, want, kind, what):
    """`want` are exact values in float64; the stored one is their rounding."""
    want = want.to(kind)
    bad = (got != want) & ~(torch.isinf(got.float()) & torch.isinf(want.float()) & (got == want))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} differ, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}"


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lead", [0, 3])
@pytest.mark.parametrize("rows,d_in,hidden", SIZES)
def test_forward_on_integers(grawa, kind, lead, rows, d_in, hidden):
    c = Case(2, rows, d_in, hidden, kind, rows + d_in, True, lead)
    h, a, u = c.forward(grawa, "relu")
    for m in range(c.M):
        wa, wu = c.x[m].double() @ c.wg[m].double().T, c.x[m].double() @ c.wu[m].double().T
        same(a[m], wa, kind, f"gate of worker {m}")
        same(u[m], wu, kind, f"up of worker {m}")
        same(h[m], torch.clamp(wa, min=0) * wu, kind, f"h of worker {m}")


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lead", [0, 3])
@pytest.mark.parametrize("rows,d_in,hidden", SIZES)
def test_backward_on_integers(grawa, kind, lead, rows, d_in, hidden):
    c = Case(2, rows, d_in, hidden, kind, rows + d_in, True, lead)
    dx, dwg, dwu = c.backward(grawa, "relu")
    for m in range(c.M):
        dh, x, a, u = (t[m].double() for t in (c.dh, c.x, c.a, c.u))
        da, du = dh * u * (a > 0), dh * a
        same(dx[m], da @ c.wg[m].double() + du @ c.wu[m].double(), kind, f"dx of worker {m}")
        same(dwg[m], da.T @ x, kind, f"dw_gate of worker {m}")
        same(dwu[m], du.T @ x, kind, f"dw_up of worker {m}")
    assert (c.grads[:, :lead] == 5.0).all()                    # what stands in front of the layer stays


# sums long enough beside few tiles that they are split (forward; dx; the weights' gradients), operands larger together
# than L2 (two launches in the backward pass), few rows against weights in rows of every alignment
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("lead", [0, 3])
@pytest.mark.parametrize("rows,d_in,hidden", [(64, 4096, 256), (100, 4100, 130), (64, 200, 4096), (70, 201, 3001), (4096, 200, 130), (5000, 136, 72), (4096, 2048, 2816)])
def test_split_sums_on_integers(grawa, rows, d_in, hidden, lead, accumulate):
    kind = torch.bfloat16
    c = Case(1, rows, d_in, hidden, kind, rows + hidden, True, lead)
    if accumulate:
        h, a, u = c.forward(grawa, "relu")
        wa, wu = c.x[0].double() @ c.wg[0].double().T, c.x[0].double() @ c.wu[0].double().T
        same(a[0], wa, kind, "gate")
        same(u[0], wu, kind, "up")
        same(h[0], torch.clamp(wa, min=0) * wu, kind, "h")
    held = 5.0 if accumulate else 0.0
    for dx_too in (True, False):
        c.grads.fill_(5.0)
        dx, dwg, dwu = c.backward(grawa, "relu", dx=dx_too, accumulate=accumulate)
        dh, x, a, u = (t[0].double() for t in (c.dh, c.x, c.a, c.u))
        da, du = dh * u * (a > 0), dh * a
        if dx_too:
            same(dx[0], da @ c.wg[0].double() + du @ c.wu[0].double(), kind, "dx")
        same(dwg[0], held + da.T @ x, kind, "dw_gate")
        same(dwu[0], held + du.T @ x, kind, "dw_up")
        assert (c.grads[:, :lead] == 5.0).all()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 3, 5, 7, 8, 9, 15, 16, 17])
@pytest.mark.parametrize("d_in,hidden,lead", [(768, 80, 0), (768, 80, 1), (97, 33, 0), (260, 40, 2), (2056, 3, 5), (8, 2000, 0), (8, 70, 3), (16, 65, 7), (12288, 17, 0), (4096, 48, 6)])
def test_few_rows_on_integers(grawa, kind, rows, d_in, hidden, lead):
    c = Case(3, rows, d_in, hidden, kind, rows + d_in, True, lead)
    h, a, u = c.forward(grawa, "relu")
    for m in range(c.M):
        wa, wu = c.x[m].double() @ c.wg[m].double().T, c.x[m].double() @ c.wu[m].double().T
        same(a[m], wa, kind, "gate")
        same(u[m], wu, kind, "up")
        same(h[m], torch.clamp(wa, min=0) * wu, kind, "h")


@pytest.mark.parametrize("rows,d_in,hidden", [(3, 40, 50), (130, 100, 264), (257, 70, 131)])
@pytest.mark.parametrize("shift", [0, 1, 2])
def test_nothing_is_written_around_the_outputs(grawa, rows, d_in, hidden, shift):
    kind = torch.float16
    c = Case(1, rows, d_in, hidden, kind, 11, True)

    def guarded(n):
        return torch.full((n + 128,), 3.0, dtype=kind, device="cuda")

    full = [guarded(rows * hidden) for _ in range(3)] + [guarded(rows * d_in)] + [guarded(d_in * hidden) for _ in range(2)]
    shapes = [(rows, hidden)] * 3 + [(rows, d_in)] + [(hidden, d_in)] * 2
    h, a, u, dx, dwg, dwu = ([t[64 + shift:64 + shift + r * k].view(r, k)] for t, (r, k) in zip(full, shapes))
    grawa.grawa_gated_ffn_forward(c.x, c.wg, c.wu, h, activation="relu", gate_out=a, up_out=u)
    grawa.grawa_gated_ffn_backward(c.dh, c.x, c.wg, c.wu, c.a, c.u, dx, dwg, dwu, activation="relu")
    wa = c.x[0].double() @ c.wg[0].double().T
    same(a[0], wa, kind, "gate")
    same(dwu[0], (c.dh[0].double() * c.a[0].double()).T @ c.x[0].double(), kind, "dw_up")
    for t, (r, k) in zip(full, shapes):
        assert (t[:64 + shift] == 3.0).all() and (t[64 + shift + r * k:] == 3.0).all()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("rows,d_in,hidden", [(1, 768, 512), (6, 264, 200), (33, 100, 77), (197, 768, 640), (300, 1024, 515)])
def test_real_values(grawa, kind, act, rows, d_in, hidden):
    c = Case(2, rows, d_in, hidden, kind, rows, False)
    h, a, u = c.forward(grawa, act)
    dx, dwg, dwu = c.backward(grawa, act)
    for m in range(2):
        for got, (want, err), what in zip((h[m], a[m], u[m]), gated_ffn64(act, c.x[m], c.wg[m], c.wu[m]), ("h", "gate", "up")):
            check(got, want, kind, err, what)
        wanted = gated_ffn_backward64(act, c.dh[m], c.x[m], c.wg[m], c.wu[m], c.a[m], c.u[m], kind)
        for got, (want, err), what in zip((dx[m], dwg[m], dwu[m]), wanted, ("dx", "dw_gate", "dw_up")):
            check(got, want, kind, err, what)


def test_accumulation_partial_outputs_and_many_workers(grawa):
    kind, M = torch.bfloat16, 19                               # more workers than one launch takes
    c = Case(M, 70, 96, 160, kind, 3, True)
    held = c.grads.clone()
    dx, dwg, dwu = c.backward(grawa, "relu", accumulate=True)
    h, a, u = c.forward(grawa, "relu")
    alone = [torch.empty_like(t) for t in h]
    grawa.grawa_gated_ffn_forward(c.x, c.wg, c.wu, alone, activation="relu")
    for m in range(M):
        da, du = c.dh[m].double() * c.u[m].double() * (c.a[m] > 0), c.dh[m].double() * c.a[m].double()
        same(dwg[m], 5.0 + da.T @ c.x[m].double(), kind, "dw_gate")
        same(dwu[m], 5.0 + du.T @ c.x[m].double(), kind, "dw_up")
        same(dx[m], da @ c.wg[m].double() + du @ c.wu[m].double(), kind, "dx")
        wa, wu = c.x[m].double() @ c.wg[m].double().T, c.x[m].double() @ c.wu[m].double().T
        same(h[m], torch.clamp(wa, min=0) * wu, kind, "h")
        assert torch.equal(alone[m], h[m])
    c.grads.copy_(held)
    only, *_ = c.backward(grawa, "relu", dw=False)
    assert all(torch.equal(p, q) for p, q in zip(only, dx)) and torch.equal(c.grads, held)
    untouched, dwg, _ = c.backward(grawa, "relu", dx=False)
    assert all((t == 9.0).all() for t in untouched)
    same(dwg[0], (c.dh[0].double() * c.u[0].double() * (c.a[0] > 0)).T @ c.x[0].double(), kind, "dw_gate")


def test_large_values_of_the_gate(grawa):
    """The ends of the activations: no overflow of the exponential shows."""
    kind = torch.bfloat16
    c = Case(1, 64, 64, 64, kind, 4, False)
    c.a = [torch.linspace(-120, 120, 64 * 64, device="cuda").view(64, 64).to(kind)]
    for act in ("silu", "gelu"):
        dx, dwg, dwu = c.backward(grawa, act)
        wanted = gated_ffn_backward64(act, c.dh[0], c.x[0], c.wg[0], c.wu[0], c.a[0], c.u[0], kind)
        for got, (want, err) in zip((dx[0], dwg[0], dwu[0]), wanted):
            check(got, want, kind, err, act)
    x = [torch.cat([torch.full((1, 64), s, device="cuda") for s in (-16.0, 16.0)]).to(kind)]
    w = [torch.full((8, 64), 0.25, device="cuda", dtype=kind)]
    h, a = [torch.empty(2, 8, device="cuda", dtype=kind)], [torch.empty(2, 8, device="cuda", dtype=kind)]
    for act in ("silu", "gelu"):
        grawa.grawa_gated_ffn_forward(x, w, w, h, activation=act, gate_out=a, up_out=[torch.empty_like(a[0])])
        assert (a[0][0] == -256).all() and (h[0][0] == 0).all() and (h[0][1] == 65536).all()


def test_no_rows(grawa):
    c = Case(1, 0, 24, 40, torch.float16, 5, True)
    c.forward(grawa, "silu")
    c.backward(grawa, "silu", accumulate=True)
    assert (c.grads == 5.0).all()
    c.backward(grawa, "silu")
    assert (c.grads == 0.0).all()


def test_replayed_graphs_on_two_streams_give_the_same_bits(grawa):
    cases = [Case(2, 150 + 100 * k, 256, 384, torch.bfloat16, 6 + k, False, lead=k) for k in range(2)]
    state = []
    for c in cases:
        h, a, u = ([torch.empty_like(t) for t in c.dh] for _ in range(3))
        dx = [torch.empty_like(t) for t in c.x]

        def both(c=c, h=h, a=a, u=u, dx=dx):
            grawa.grawa_gated_ffn_forward(c.x, c.wg, c.wu, h, gate_out=a, up_out=u)
            grawa.grawa_gated_ffn_backward(c.dh, c.x, c.wg, c.wu, a, u, dx, c.dwg, c.dwu)

        both()
        outs = h + a + u + dx + c.dwg + c.dwu              # (not what stands in front of the weights: nothing writes it)
        want = [t.clone() for t in outs]
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            both()
        state.append((g, outs, want))
    streams = [torch.cuda.Stream() for _ in state]
    for _ in range(3):
        for g, outs, want in state:
            for t in outs:
                t.fill_(9.0)
        torch.cuda.synchronize()
        for s, (g, _, _) in zip(streams, state):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for _, outs, want in state:
            assert all(torch.equal(p, q) for p, q in zip(outs, want))
    assert grawa.grawa_gated_ffn_status() == 0


def test_gradients_against_differences(grawa):
    """Central differences of sum(h dh) in 64 bits around 16-bit inputs, in random directions: the slope along a direction
    is the inner product of the direction and the gradient."""
    kind, rows, d_in, hidden = torch.float16, 24, 40, 56
    c = Case(1, rows, d_in, hidden, kind, 8, False)
    h, a, u = c.forward(grawa, "gelu")
    c.a, c.u = a, u
    dx, dwg, dwu = c.backward(grawa, "gelu")
    gen = torch.Generator(device="cuda").manual_seed(1)
    base = [t[0].double() for t in (c.x, c.wg, c.wu)]

    def value(x, wg, wu):
        return (gated_ffn64("gelu", x, wg, wu)[0][0] * c.dh[0].double()).sum()

    for which, grad in enumerate((dx[0], dwg[0], dwu[0])):
        v = torch.randn(base[which].shape, generator=gen, device="cuda", dtype=torch.float64)
        step = 1e-5
        ends = [value(*[b + s * step * v if k == which else b for k, b in enumerate(base)]) for s in (1, -1)]
        slope = (ends[0] - ends[1]) / (2 * step)
        # a and u carry one rounding (2^-11), da and du another, the gradient a third: at most 2^-11 of each term
        # in absolute value; slopes and second derivatives of gelu are below 1.13
        got = (grad.double() * v).sum()
        terms = (c.dh[0].double().abs() * (u[0].double().abs() + a[0].double().abs()) * 1.13)
        reach = {0: (terms @ (c.wg[0].double().abs() + c.wu[0].double().abs())), 1: terms.T @ c.x[0].double().abs(), 2: terms.T @ c.x[0].double().abs()}[which]
        assert (got - slope).abs() < 4 * 2.0 ** -11 * (reach * v.abs()).sum() + 1e-6 * slope.abs()
        assert slope.abs() > 20 * 2.0 ** -11                   # the direction says something


def test_binding_refuses_wrong_tensors(grawa):
    c = Case(2, 16, 32, 48, torch.bfloat16, 9, True)
    h = [torch.empty_like(t) for t in c.dh]
    with pytest.raises(grawa.GrawaError):
        grawa.grawa_gated_ffn_forward(*[[t.float() for t in v] for v in (c.x, c.wg, c.wu, h)])
    with pytest.raises(ValueError):
        grawa.grawa_gated_ffn_forward(c.x, [t.T for t in c.wg], c.wu, h)
    with pytest.raises(ValueError):
        grawa.grawa_gated_ffn_forward(c.x, c.wg, c.wu, [t[:8] for t in h])
    with pytest.raises(KeyError):
        grawa.grawa_gated_ffn_forward(c.x, c.wg, c.wu, h, activation="tanh")
    with pytest.raises(grawa.GrawaError):
        grawa.grawa_gated_ffn_forward(c.x, c.wg, c.wu, [h[0], h[0]])
    with pytest.raises(ValueError):
        grawa.grawa_gated_ffn_forward([t.cpu() for t in c.x], c.wg, c.wu, h)


def test_results_past_two_to_the_31_elements(grawa):
    """Small integers: every sum stays below 2^24, so float32 holds it however it is added up."""
    rows, d_in, hidden, kind = 131077, 8, 16400, torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(12)

    def draw(*shape, low=-2):
        return torch.randint(low, 3, shape, generator=gen, device="cuda", dtype=torch.int8).to(kind)

    x, wg, wu = draw(rows, d_in), draw(hidden, d_in), draw(hidden, d_in)
    h, gate, up = (torch.full((rows, hidden), 9.0, device="cuda", dtype=kind) for _ in range(3))
    grawa.grawa_gated_ffn_forward([x], [wg], [wu], [h], activation="relu", gate_out=[gate], up_out=[up])
    chunks = [slice(i, min(i + 8192, rows)) for i in range(0, rows, 8192)]
    for c in chunks:
        a, u = x[c].float() @ wg.float().T, x[c].float() @ wu.float().T
        for name, got, want in (("h", h, a.clamp(min=0) * u), ("gate", gate, a), ("up", up, u)):
            same(got[c], want, kind, f"{name} of rows from {c.start}")
    del h
    dh, gate[:], up[:] = draw(rows, hidden), draw(rows, hidden, low=0), draw(rows, hidden)
    dx, dwg, dwu = (torch.full_like(t, 9.0) for t in (x, wg, wu))
    grawa.grawa_gated_ffn_backward([dh], [x], [wg], [wu], [gate], [up], [dx], [dwg], [dwu], activation="relu")
    assert grawa.grawa_gated_ffn_status() == 0
    sums = [torch.zeros(hidden, d_in, device="cuda") for _ in range(2)]
    for c in chunks:
        da, du = dh[c].float() * up[c].float() * (gate[c] > 0), dh[c].float() * gate[c].float()
        same(dx[c], da @ wg.float() + du @ wu.float(), kind, f"dx of rows from {c.start}")
        for s, d in zip(sums, (da, du)):
            s += d.T @ x[c].float()
    same(dwg, sums[0], kind, "dw_gate")
    same(dwu, sums[1], kind, "dw_up")


@pytest.mark.parametrize("rows,d_in,hidden,lead", [(70, 61, 133, 0), (70, 64, 133, 3), (300, 127, 250, 1)])
def test_scratch_full_of_nan_and_shared_inputs(grawa, rows, d_in, hidden, lead):
    """Operands laid out again in the scratch, whose rows are then longer than the operands': what lies behind them is
    not read.  Both workers read the same tensors."""
    c = Case(1, rows, d_in, hidden, torch.bfloat16, 13, True, lead)
    two = Case(2, rows, d_in, hidden, torch.bfloat16, 13, True, lead)
    for name in ("wg", "wu", "x", "dh", "a", "u"):
        setattr(two, name, getattr(c, name) * 2)

    def scratch(backward):
        need = grawa.grawa_gated_ffn_workspace_bytes(rows, d_in, hidden, 2, backward=backward, aligned=False)
        return torch.full((need,), 255, dtype=torch.uint8, device="cuda")

    h, a, u = two.forward(grawa, "relu", workspace=scratch(False))
    dx, dwg, dwu = two.backward(grawa, "relu", workspace=scratch(True))
    (wh, _), (wa, _), (wu, _) = gated_ffn64("relu", c.x[0], c.wg[0], c.wu[0])
    (wdx, _), (wdg, _), (wdu, _) = gated_ffn_backward64("relu", c.dh[0], c.x[0], c.wg[0], c.wu[0], c.a[0], c.u[0], torch.bfloat16)
    for m in range(2):
        for name, got, want in (("h", h, wh), ("gate", a, wa), ("up", u, wu), ("dx", dx, wdx), ("dw_gate", dwg, wdg), ("dw_up", dwu, wdu)):
            same(got[m], want, torch.bfloat16, f"{name} of worker {m}")
