"""Norms of query and key heads with rotation, forward and backward, against their statements in 64 bits."""
import pytest
import torch

from attention_util import head_rotary64, head_rotary_backward64
from replica_util import TYPES, check

pytestmark = pytest.mark.gpu
EPS = 1e-6


def heads_of(gen, M, rows, heads, dim, kind, pad=0, lead=0, scale=1.0):
    """M tensors [rows, heads, dim] whose rows are `pad` elements apart and begin `lead` elements into a buffer, and the buffers."""
    held = [(torch.randn(lead + rows * (heads * dim + pad), generator=gen, device="cuda") * scale).to(kind) for _ in range(M)]
    return [t[lead:].view(rows, heads * dim + pad)[:, :heads * dim].unflatten(1, (heads, dim)) for t in held], held


def vectors(gen, M, dim, kind, lead=3):
    return [(1.0 + 0.1 * torch.randn(lead + dim, generator=gen, device="cuda")).to(kind)[lead:] for _ in range(M)]


# rows, query heads, key heads, dim, rotary, pad, lead: one token, whole words, fp32 and 16-bit words cut, odd sizes, single elements
SHAPES = [(1, 12, 12, 64, 64, 0, 0), (5, 3, 1, 128, 128, 0, 0), (70, 4, 2, 64, 32, 8, 8), (9, 1, 1, 256, 256, 0, 0), (33, 5, 0, 40, 24, 0, 0),
          (17, 3, 2, 80, 40, 4, 4), (7, 2, 3, 7, 4, 1, 1), (3, 2, 1, 1, 0, 0, 0), (11, 2, 2, 255, 254, 0, 0), (300, 7, 7, 96, 0, 0, 0), (4, 40, 8, 8, 8, 0, 0),
          (6, 1, 1, 2, 2, 0, 1), (5, 3, 3, 24, 8, 0, 0), (12, 2, 1, 128, 36, 0, 0)]


def sizes(shape, kind, pairing, given, seed=0):
    rows, heads, kv_heads, dim, rotary, pad, lead = shape
    M, gen = 2, torch.Generator(device="cuda").manual_seed(seed)
    q, _ = heads_of(gen, M, rows, heads, dim, kind, pad, lead)
    k = heads_of(gen, M, rows, kv_heads, dim, kind, pad, lead)[0] if kv_heads else None
    qw, kw = vectors(gen, M, dim, kind), vectors(gen, M, dim, kind) if kv_heads else None
    f = 10.0 ** -torch.linspace(0, 4, rotary // 2, dtype=torch.float64, device="cuda") if rotary else None
    at = [torch.randint(0, 3_000_000, (rows,), generator=gen, device="cuda") for _ in range(M)] if given else None
    places = at if given else [torch.arange(rows, device="cuda") % 16] * M
    return gen, M, q, k, qw, kw, f, dict(positions=at, period=16, pairing=pairing, eps=EPS), places


@pytest.mark.parametrize("pairing, given", [("halves", False), ("neighbours", True)])
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, kind, pairing, given):
    import paper_2403_04206_b200 as grawa
    rows, heads, kv_heads, dim, _, pad, lead = shape
    gen, M, q, k, qw, kw, f, where, places = sizes(shape, kind, pairing, given)
    out = heads_of(gen, M, rows, heads, dim, kind, 2 * pad, lead)
    k_out = heads_of(gen, M, rows, kv_heads, dim, kind, pad, lead) if kv_heads else (None, [])
    before = [t.clone() for t in out[1] + k_out[1]]
    grawa.grawa_head_rotary_forward(q, k, qw, kw, out[0], k_out[0], f, **where)
    for x, w, y in ((q, qw, out[0]),) + (((k, kw, k_out[0]),) if kv_heads else ()):
        for m in range(M):
            want, error = head_rotary64(x[m], w[m], places[m], f, pairing, EPS)
            check(y[m], want, kind, error, "y")
            y[m].zero_()
    for held, was, views in zip(out[1] + k_out[1], before, out[0] + (k_out[0] or [])):     # nothing around the rows has changed
        rows_of = was[lead:].view(rows, -1)[:, :views.shape[1] * dim]
        rows_of.zero_()
        assert torch.equal(held, was)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("pairing, given", [("halves", True), ("neighbours", False)])
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(shape, kind, pairing, given, accumulate):
    import paper_2403_04206_b200 as grawa
    rows, heads, kv_heads, dim, _, pad, lead = shape
    gen, M, q, k, qw, kw, f, where, places = sizes(shape, kind, pairing, given, seed=1)
    args = []
    for x, w, n in ((q, qw, heads), (k, kw, kv_heads)):
        if n:
            dy = heads_of(gen, M, rows, n, dim, kind, 2 * pad, lead)[0]
            dx = heads_of(gen, M, rows, n, dim, kind, pad, lead)[0]
            dw = vectors(gen, M, dim, kind)
            args.append((dy, x, w, dx, dw, [t.clone() for t in dw]))
        else:
            args.append((None,) * 6)
    (dq_out, _, _, dq, dqw, _), (dk_out, _, _, dk, dkw, _) = args
    grawa.grawa_head_rotary_backward(dq_out, dk_out, q, k, qw, kw, dq, dk, dqw, dkw, f, accumulate=accumulate, **where)
    for dy, x, w, dx, dw, was in args[:2 if kv_heads else 1]:
        for m in range(M):
            (want, error), (want_w, error_w) = head_rotary_backward64(dy[m], x[m], w[m], places[m], f, pairing, EPS)
            check(dx[m], want, kind, error, "dx")
            check(dw[m], want_w + (was[m].double() if accumulate else 0.0), kind, error_w + 2.0 ** -24 * was[m].double().abs(), "dw")


def test_parts_of_the_gradient_alone_and_in_place():
    import paper_2403_04206_b200 as grawa
    shape = (70, 4, 2, 64, 64, 8, 8)
    gen, M, q, k, qw, kw, f, where, places = sizes(shape, torch.bfloat16, "halves", True, seed=2)
    def like(n):
        return heads_of(gen, M, 70, n, 64, torch.bfloat16, 8, 8)[0]
    dq_out, dk_out, dq, dk = like(4), like(2), like(4), like(2)
    dqw, dkw = vectors(gen, M, 64, torch.bfloat16), vectors(gen, M, 64, torch.bfloat16)
    grawa.grawa_head_rotary_backward(dq_out, dk_out, q, k, qw, kw, dq, dk, dqw, dkw, f, **where)
    want = [t.clone() for t in dq + dk + dqw + dkw]
    for t in dq + dk + dqw + dkw:
        t.fill_(7.0)
    grawa.grawa_head_rotary_backward(dq_out, dk_out, q, k, qw, kw, None, dk, dqw, None, f, **where)
    grawa.grawa_head_rotary_backward(dq_out, dk_out, q, k, qw, kw, dq, None, None, dkw, f, **where)
    assert all(torch.equal(a, b) for a, b in zip(dq + dk + dqw + dkw, want))
    grawa.grawa_head_rotary_backward(dq_out, dk_out, q, k, qw, kw, dq_out, dk_out, dqw, dkw, f, **where)
    assert all(torch.equal(a, b) for a, b in zip(dq_out + dk_out + dqw + dkw, want))
    q_out, k_out = like(4), like(2)
    grawa.grawa_head_rotary_forward(q, k, qw, kw, q_out, k_out, f, **where)
    grawa.grawa_head_rotary_forward(q, k, qw, kw, q, k, f, **where)
    assert all(torch.equal(a, b) for a, b in zip(q + k, q_out + k_out))


def test_no_weights_no_rows_and_special_rows():
    import paper_2403_04206_b200 as grawa
    gen, M, q, k, _, _, f, where, places = sizes((6, 2, 1, 64, 64, 0, 0), torch.float32, "halves", True, seed=3)
    q[0][2] = 0.0
    q[0][3, 1, 5] = float("nan")
    out, k_out = [torch.empty_like(t) for t in q], [torch.empty_like(t) for t in k]
    grawa.grawa_head_rotary_forward(q, k, None, None, out, k_out, f, **where)
    assert out[0][3, 1].isnan().all() and (out[0][2] == 0).all()          # a head of NaN is that head's alone
    q[0][3, 1, 5] = 0.0
    want, error = head_rotary64(q[0], None, places[0], f, "halves", EPS)
    out[0][3, 1] = want[3, 1].float()
    check(out[0], want, torch.float32, error)
    dw = [torch.full((64,), 3.0, device="cuda") for _ in range(M)]
    none = [t[:0] for t in q]
    grawa.grawa_head_rotary_backward(none, None, none, None, None, None, None, None, dw, None, f, accumulate=True)
    assert all((t == 3.0).all() for t in dw)
    grawa.grawa_head_rotary_backward(none, None, none, None, None, None, None, None, dw, None, f)
    assert all((t == 0.0).all() for t in dw)


def test_captured_and_on_another_stream():
    import paper_2403_04206_b200 as grawa
    gen, M, q, k, qw, kw, f, where, places = sizes((500, 4, 2, 128, 128, 0, 0), torch.bfloat16, "neighbours", True, seed=4)
    dq_out, dk_out = [torch.randn_like(t) for t in q], [torch.randn_like(t) for t in k]
    q_out, k_out, dq, dk = ([torch.empty_like(t) for t in x] for x in (q, k, q, k))
    dqw, dkw = [torch.empty_like(t) for t in qw], [torch.empty_like(t) for t in kw]
    results = q_out + k_out + dq + dk + dqw + dkw

    def both():
        grawa.grawa_head_rotary_forward(q, k, qw, kw, q_out, k_out, f, **where)
        grawa.grawa_head_rotary_backward(dq_out, dk_out, q, k, qw, kw, dq, dk, dqw, dkw, f, **where)

    both()
    want = [t.clone() for t in results]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for t in results:
        t.zero_()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(results, want))
    for t in results:
        t.zero_()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both()
    torch.cuda.current_stream().wait_stream(stream)
    assert all(torch.equal(a, b) for a, b in zip(results, want))


def test_far_positions_keep_their_digits():
    """Positions of billions: the angles are those of 64 bits (off by 2^-53 of themselves), as in 32 bits not even their sign would be."""
    import paper_2403_04206_b200 as grawa
    gen, M, q, k, qw, kw, f, where, _ = sizes((64, 2, 1, 64, 64, 0, 0), torch.float32, "halves", True, seed=5)
    where["positions"] = [torch.randint(0, 1 << 32, (64,), generator=gen, device="cuda") for _ in range(M)]
    out, k_out = [torch.empty_like(t) for t in q], [torch.empty_like(t) for t in k]
    grawa.grawa_head_rotary_forward(q, k, qw, kw, out, k_out, f, **where)
    for m in range(M):
        want, error = head_rotary64(q[m], qw[m], where["positions"][m], f, "halves", EPS)
        # two products and a reduction on either side, each 2^-53 of an angle of up to 2^32, against elements of up to 8
        check(out[m], want, torch.float32, error + 8 * 6 * 2.0 ** (32 - 53))
