"""Attention within a window in launches of more tiles than fit the GPU at once, on several streams, captured, without overlapping
launches; and what stands around its results."""
import pytest
import torch

from test_gpu_replica_attention import ALL, HALVES, Case

pytestmark = pytest.mark.gpu

# A CTA takes several tiles from 296 of them on in the forward pass, 148 in the others.
MANY = [
    dict(rows=2500, heads=12, kv_heads=6, dim=64, M=4),
    dict(rows=2500, heads=6, kv_heads=6, dim=128, M=4, left=300, sinks=4, lengths=[[2493, 0, 0, 0], [700, 0, 1800, 0], [1, 2300, 130, 60], [128, 128, 512, 1700]]),
    dict(rows=197 * 12, heads=6, kv_heads=6, dim=64, M=4, right=ALL, period=197),
    dict(rows=1300, heads=16, kv_heads=8, dim=80, M=3, left=64, right=30, period=500),
    dict(rows=4100, heads=2, kv_heads=2, dim=64, M=16, left=64, sinks=3),                  # 160 chunks of queries set apart
]


@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("case", MANY, ids=lambda c: " ".join(f"{k}={v}" for k, v in c.items() if k != "lengths")[:70])
def test_ctas_with_several_tiles_against_64_bits(case, kind):
    c = Case(kind, seed=31, **case)
    c.check_forward()
    c.check_backward()


def _results(c):
    return c.out + c.lse + c.dq + c.dk + c.dv


def _both(c):
    c.forward()
    c.backward()


@pytest.mark.parametrize("kind", HALVES)
def test_warps_that_run_ahead_of_others(kind):
    """Tiles with first keys, whose first 32 rows' warps take longest (they add the sums of chunks), and behind each some more tiles of the
    same CTA: the other warps may be a step ahead, and wait there."""
    import paper_2403_04206_b200 as grawa
    c = Case(kind, 2300, 4, 2, 64, left=100, sinks=3, M=18, seed=30)
    c.check_forward()
    c.check_backward()
    want = [t.clone() for t in _results(c)]
    for _ in range(30):
        for t in _results(c):
            t.zero_()
        _both(c)
        assert all(torch.equal(a, b) for a, b in zip(_results(c), want))
    assert grawa.grawa_window_attention_status() == 0


@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("M", [2, 18])
def test_without_overlapping_launches(kind, M):
    """The same bits where each launch waits for the end of the one in front: dq beside dk and dv, chunks in front of them."""
    import paper_2403_04206_b200 as grawa
    c = Case(kind, 2300, 4, 2, 64, left=100, sinks=3, M=M, seed=32)
    _both(c)
    want = [t.clone() for t in _results(c)]
    for t in _results(c):
        t.zero_()
    before = grawa.grawa_get_option("dependent_launch")
    assert before == 1
    try:
        grawa.grawa_set_option("dependent_launch", 0)
        _both(c)
        torch.cuda.synchronize()
    finally:
        grawa.grawa_set_option("dependent_launch", before)
    assert all(torch.equal(a, b) for a, b in zip(_results(c), want))


def test_half_precision_captured_and_replayed():
    """The backward pass in half precision starts with a set of its scratch: in a graph that stands in front of a launch that overlaps."""
    c = Case(torch.float16, 1500, 4, 2, 64, left=100, sinks=4, lengths=[[600, 600, 290], [10, 1200, 250]], seed=33)
    _both(c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _both(c)
    for scale in (1.0, 2.0 ** -8, 4.0):                       # other longest rows than those of the replay in front
        for t in c.dout:
            t.mul_(scale)
        graph.replay()
        graph.replay()
        replayed = [t.clone() for t in _results(c)]
        _both(c)
        assert all(torch.equal(a, b) for a, b in zip(_results(c), replayed))


def test_large_calls_on_two_streams_at_once():
    cases = [Case(torch.bfloat16, 6000, 8, 2, 64, left=1000, sinks=2, seed=34), Case(torch.float16, 5000, 8, 4, 128, seed=35)]
    want = []
    for c in cases:
        _both(c)
        want.append([t.clone() for t in _results(c)])
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(10):
        for c in cases:
            for t in _results(c):
                t.zero_()
        torch.cuda.synchronize()
        for _ in range(3):
            for c, stream in zip(cases, streams):
                with torch.cuda.stream(stream):
                    _both(c)
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert all(torch.equal(a, b) for a, b in zip(_results(c), w))


def _inside(gen, rows, heads, dim, kind, margin=256):
    """[rows, heads, dim] in the middle of a buffer with `margin` rows on either side, and the buffer, all of it 5."""
    held = torch.full((rows + 2 * margin, heads, dim), 5.0, dtype=kind, device="cuda")
    return held[margin:margin + rows], held


@pytest.mark.parametrize("sinks", [0, 3])
@pytest.mark.parametrize("kind", HALVES)
def test_offsets_that_make_no_sense_leave_what_is_around_the_buffers(kind, sinks):
    """Offsets that decrease or leave the rows: nothing in front of or behind any result or the scratch changes."""
    import paper_2403_04206_b200 as grawa
    rows, heads, kv_heads, dim, M = 1300, 4, 2, 64, 2
    gen = torch.Generator(device="cuda").manual_seed(36)
    q, k, v, dout = ([torch.randn(rows, n, dim, generator=gen, device="cuda").to(kind) for _ in range(M)] for n in (heads, kv_heads, kv_heads, heads))
    views = {name: [_inside(gen, rows, n, dim, kind) for _ in range(M)] for name, n in (("out", heads), ("dq", heads), ("dk", kv_heads), ("dv", kv_heads))}
    lse = [torch.full((3 * heads * rows,), 5.0, device="cuda") for _ in range(M)]
    stats = [t[heads * rows:2 * heads * rows].view(heads, rows) for t in lse]
    need = grawa.grawa_window_attention_backward_workspace_bytes(rows, heads, kv_heads, dim, sinks, M)
    space = torch.full((need + 2 * 65536,), 77, dtype=torch.uint8, device="cuda")
    out, dq, dk, dv = ([t for t, _ in views[name]] for name in ("out", "dq", "dk", "dv"))
    for bad in ([-50, 100, 400, 1 << 40], [200, 100, 50, 0], [0, 1250, 50, 1300], [1 << 62, 0, -(1 << 62), 1300], [0, 0, 0, 0], [1290, 5, 1299, 1], [-(1 << 62), 1300, 1300, 1 << 62],
                [0, 1024, 1000, 1290], [1300, 1300, 1300, 1300], [-5, -4, -3, -2], [700, 1 << 33, 3, 1200]):
        window = dict(offsets=[torch.tensor(bad, device="cuda") for _ in range(M)], left=90, right=2, sinks=sinks)
        grawa.grawa_window_attention_forward(q, k, v, out, lse=stats, **window)
        grawa.grawa_window_attention_backward(dout, q, k, v, out, stats, dq, dk, dv, workspace=space[65536:65536 + need], **window)
        assert grawa.grawa_window_attention_status() == 0
        for name in views:
            for _, held in views[name]:
                assert (held[:256] == 5.0).all() and (held[256 + rows:] == 5.0).all(), (name, bad)
        for t in lse:
            assert (t[:heads * rows] == 5.0).all() and (t[2 * heads * rows:] == 5.0).all(), bad
        assert (space[:65536] == 77).all() and (space[65536 + need:] == 77).all(), bad
