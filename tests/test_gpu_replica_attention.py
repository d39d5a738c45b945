"""Attention within a window, forward and backward, against its statement in 64 bits."""
import pytest
import torch

from attention_util import attention64, attention_backward64, visible
from replica_util import check

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]
ALL = 1 << 40                              # no limit


def heads_of(gen, M, rows, heads, dim, kind, pad=0, scale=1.0):
    """M tensors [rows, heads, dim] whose rows are `pad` elements apart."""
    return [(torch.randn(rows, heads * dim + pad, generator=gen, device="cuda") * scale).to(kind)[:, :heads * dim].unflatten(1, (heads, dim)) for _ in range(M)]


class Case:
    """Inputs of M workers.  lengths: of the packed sequences of every worker, or None for sequences of `period` rows; `front` rows
    stand in front of the first packed sequence."""

    def __init__(self, kind, rows, heads, kv_heads, dim, left=ALL, right=0, sinks=0, period=None, lengths=None, front=0, pad=0, M=2, seed=0, scale=None,
                 size=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.kind, self.rows, self.M, self.scale = kind, rows, M, dim ** -0.5 if scale is None else scale
        self.q, self.k = heads_of(gen, M, rows, heads, dim, kind, pad, size), heads_of(gen, M, rows, kv_heads, dim, kind, 0, size)
        self.v, self.dout = heads_of(gen, M, rows, kv_heads, dim, kind, 2 * pad), heads_of(gen, M, rows, heads, dim, kind, pad, 0.1)
        self.out, self.lse = heads_of(gen, M, rows, heads, dim, kind, pad), [torch.full((heads, rows), 7.0, device="cuda") for _ in range(M)]
        self.dq, self.dk = heads_of(gen, M, rows, heads, dim, kind, pad), heads_of(gen, M, rows, kv_heads, dim, kind, 0)
        self.dv = heads_of(gen, M, rows, kv_heads, dim, kind, 2 * pad)
        offsets = None
        if lengths is None:
            period = rows if period is None else period
            self.bounds = [[(a, min(a + period, rows)) for a in range(0, rows, period)]] * M
        else:
            at = [torch.tensor([front] + n).cumsum(0) for n in lengths]
            self.bounds = [list(zip(t[:-1].tolist(), t[1:].tolist())) for t in at]
            offsets = [t.cuda() for t in at]
        self.window = dict(offsets=offsets, period=period, left=left, right=right, sinks=sinks, scale=self.scale)
        self.seen = [visible(rows, b, min(left, rows), min(right, rows), sinks, "cuda") for b in self.bounds]
        self.inside = [s.any(-1) for s in self.seen]

    def forward(self):
        import paper_2403_04206_b200 as grawa
        grawa.grawa_window_attention_forward(self.q, self.k, self.v, self.out, lse=self.lse, **self.window)

    def backward(self, **kw):
        import paper_2403_04206_b200 as grawa
        grawa.grawa_window_attention_backward(self.dout, self.q, self.k, self.v, self.out, self.lse, self.dq, self.dk, self.dv, **self.window, **kw)

    def check_forward(self, blind=None):
        """blind: truth values of the rows that see something which is no number."""
        before = [t.clone() for t in self.out]
        self.forward()
        for m in range(self.M):
            (out, e), (lse, el) = attention64(self.q[m], self.k[m], self.v[m], self.seen[m], self.scale)
            rows = self.inside[m] if blind is None else self.inside[m] & ~blind[m]
            check(self.out[m][rows], out[rows], self.kind, e[rows], "out")
            check(self.lse[m][:, rows], lse[:, rows], torch.float32, el[:, rows], "lse")
            assert torch.equal(self.out[m][~self.inside[m]], before[m][~self.inside[m]]) and (self.lse[m][:, ~self.inside[m]] == 7.0).all()

    def check_backward(self, blind_q=None, blind_k=None):
        before = [[t.clone() for t in g] for g in (self.dq, self.dk, self.dv)]
        self.backward()
        for m in range(self.M):
            want = attention_backward64(self.dout[m], self.q[m], self.k[m], self.v[m], self.out[m], self.lse[m], self.seen[m], self.scale)
            for name, got, was, (exact, e), blind in zip(("dq", "dk", "dv"), (self.dq, self.dk, self.dv), before, want, (blind_q, blind_k, blind_k)):
                rows = self.inside[m] if blind is None else self.inside[m] & ~blind[m]
                check(got[m][rows], exact[rows], self.kind, e[rows], name)
                assert torch.equal(got[m][~self.inside[m]], was[m][~self.inside[m]]), name


# rows, heads, kv_heads, dim, window
CASES = [
    dict(rows=1, heads=1, kv_heads=1, dim=64),
    dict(rows=5, heads=12, kv_heads=12, dim=64),
    dict(rows=128, heads=2, kv_heads=1, dim=128),
    dict(rows=129, heads=3, kv_heads=3, dim=8, right=ALL),
    dict(rows=257, heads=6, kv_heads=2, dim=80, left=99, sinks=3),
    dict(rows=300, heads=4, kv_heads=2, dim=128, left=40, right=7, pad=8),
    dict(rows=394, heads=2, kv_heads=2, dim=64, right=ALL, period=197),
    dict(rows=300, heads=2, kv_heads=1, dim=96, left=0),                                        # every row sees itself
    dict(rows=300, heads=2, kv_heads=1, dim=112, left=0, sinks=130),                            # first keys over more than one tile
    dict(rows=700, heads=1, kv_heads=1, dim=64, left=63, sinks=1),
    dict(rows=700, heads=4, kv_heads=1, dim=128, left=200, sinks=4, lengths=[[0, 3, 0, 500, 1, 100, 0], [690, 0, 0, 1, 1, 0, 8]], pad=16),
    dict(rows=520, heads=2, kv_heads=2, dim=40, left=10, right=20, sinks=2, lengths=[[100, 29, 200], [1, 1, 1]], front=130),
    dict(rows=520, heads=2, kv_heads=1, dim=64, lengths=[[0], [520]]),                          # no sequence but an empty one
    dict(rows=1000, heads=2, kv_heads=2, dim=64, right=ALL, lengths=[[250] * 4, [999, 1, 0, 0]], sinks=5),
    dict(rows=650, heads=2, kv_heads=2, dim=128, period=1),                                     # sequences of one token
    dict(rows=650, heads=8, kv_heads=2, dim=128, period=640, left=300, scale=1.0),              # sharp rows
    dict(rows=2050, heads=1, kv_heads=1, dim=128, left=ALL),
    dict(rows=3500, heads=2, kv_heads=1, dim=64, left=100, sinks=4),                            # first keys whose queries lie in more than one chunk
    dict(rows=3500, heads=2, kv_heads=2, dim=128, left=300, right=5, sinks=128, lengths=[[200, 3000, 300], [5, 1000, 2490]]),
    dict(rows=3300, heads=1, kv_heads=1, dim=64, left=0, sinks=200, period=1600),
]


@pytest.mark.parametrize("kind", HALVES)
@pytest.mark.parametrize("case", CASES, ids=lambda c: " ".join(f"{k}={v}" for k, v in c.items() if k != "lengths")[:70])
def test_against_64_bits(case, kind):
    c = Case(kind, **case)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("kind", HALVES)
def test_large_scores_and_one_ahead_of_all(kind):
    """Rows whose largest score stands in the last of many tiles, far above the others: what was summed before shrinks to nothing."""
    c = Case(kind, 900, 2, 1, 64, scale=0.125, size=4.0, seed=3)
    for m in range(c.M):
        c.k[m][880] = c.q[m][890, :1]
        c.k[m][0] *= 4
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_a_row_does_not_see_does_not_reach_it(bad, dim):
    """NaN and infinities in keys, values and upstream gradients: exactly the rows that see them are affected."""
    c = Case(torch.bfloat16, 400, 2, 1, dim, left=50, sinks=2, lengths=[[150, 100, 140], [350, 20, 10]], seed=5)
    lost = 170
    for t in c.k + c.v:
        t[lost] = bad
    for t in c.q + c.k + c.v + c.dout:
        t[392:] = bad                                       # behind the last sequence
    blind = [s[:, lost] for s in c.seen]
    c.check_forward(blind)
    c = Case(torch.bfloat16, 400, 2, 1, dim, left=50, sinks=2, lengths=[[150, 100, 140], [350, 20, 10]], seed=5)
    for t in c.q + c.k + c.v + c.dout:
        t[392:] = bad
    c.check_forward()
    for t in c.dout:
        t[lost] = bad
    own = [torch.arange(400, device="cuda") == lost for _ in c.seen]
    c.check_backward(own, [s[lost] for s in c.seen])
    for m in range(c.M):
        assert not torch.isfinite(c.dv[m][c.seen[m][lost]].float()).any()
    c = Case(torch.bfloat16, 400, 2, 1, dim, left=50, sinks=2, lengths=[[150, 100, 140], [350, 20, 10]], seed=5)
    c.forward()
    for t in c.k:                                           # (the statistics are those of the forward call before)
        t[lost] = bad
    c.check_backward([s[:, lost] for s in c.seen], own)


def test_half_precision_gradients_of_long_rows_and_small_upstream_gradients():
    """P of 1 / 2000 and gradients of 1e-6: products far below the smallest normal half are kept by their powers of two."""
    c = Case(torch.float16, 2000, 1, 1, 64, right=ALL, size=0.05, seed=6)
    for t in c.dout:
        t.mul_(1e-3)
    c.forward()
    c.check_backward()


def test_parts_alone_and_the_callers_scratch():
    import paper_2403_04206_b200 as grawa
    c = Case(torch.float16, 300, 4, 2, 64, left=70, sinks=1, seed=7)
    c.forward()
    c.backward()
    want = [t.clone() for t in c.dq + c.dk + c.dv]
    for t in c.dq + c.dk + c.dv:
        t.fill_(3.0)
    need = grawa.grawa_window_attention_backward_workspace_bytes(300, 4, 2, 64, 1, 2)
    scratch = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")       # NaN, in every type
    args = (c.dout, c.q, c.k, c.v, c.out, c.lse)
    grawa.grawa_window_attention_backward(*args, None, c.dk, c.dv, workspace=scratch[:need], **c.window)
    assert all((t == 3.0).all() for t in c.dq)
    grawa.grawa_window_attention_backward(*args, c.dq, None, None, workspace=scratch[:need], **c.window)
    assert all(torch.equal(a, b) for a, b in zip(c.dq + c.dk + c.dv, want)) and (scratch[need:] == 255).all()


def test_offsets_that_make_no_sense_touch_nothing_outside():
    c = Case(torch.bfloat16, 300, 2, 1, 64, lengths=[[100, 100, 50], [10, 200, 50]], seed=8)
    guard = [torch.full((64, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for bad in ([-50, 100, 400, 1 << 40], [200, 100, 50, 0], [0, 250, 50, 300], [1 << 62, 0, -(1 << 62), 300], [0, 0, 0, 0]):
        for t in c.window["offsets"]:
            t.copy_(torch.tensor(bad))
        c.forward()
        c.backward()
        torch.cuda.synchronize()
    assert all((t == 5.0).all() for t in guard)


def test_captured_replayed_with_other_offsets_and_reproducible():
    c = Case(torch.bfloat16, 700, 4, 2, 128, left=100, sinks=4, lengths=[[300, 300, 90], [10, 600, 50]], seed=9)
    results = c.out + c.lse + c.dq + c.dk + c.dv

    def both():
        c.forward()
        c.backward()

    both()
    want = [t.clone() for t in results]
    both()
    assert all(torch.equal(a, b) for a, b in zip(results, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(results, want))
    for t in c.window["offsets"]:
        t.copy_(torch.tensor([0, 200, 450, 700]))
    graph.replay()
    replayed = [t.clone() for t in results]
    both()
    assert all(torch.equal(a, b) for a, b in zip(results, replayed)) and not torch.equal(replayed[0], want[0])


def test_many_workers():
    """More workers than one launch takes."""
    c = Case(torch.bfloat16, 140, 2, 1, 64, left=30, M=37, seed=10)
    c.check_forward()
    c.check_backward()


def test_no_rows():
    c = Case(torch.bfloat16, 8, 2, 1, 64)
    for name in ("q", "k", "v", "dout", "out", "dq", "dk", "dv"):
        setattr(c, name, [t[:0] for t in getattr(c, name)])
    c.lse = [t[:, :0].contiguous() for t in c.lse]
    c.window["period"] = None
    c.forward()
    c.backward()


@pytest.mark.parametrize("which", ["q", "k", "v", "dout", "all"])
def test_rows_of_nothing_but_nan_end_and_stay_nan(which):
    """A replica that has diverged: what depends on NaN is NaN, in all elements, and the calls return as ever."""
    import time
    import paper_2403_04206_b200 as grawa
    c = Case(torch.bfloat16, 6000, 2, 1, 128, seed=11)
    for name in ("q", "k", "v", "dout") if which == "all" else (which,):
        for t in getattr(c, name):
            t.fill_(float("nan"))
    start = time.perf_counter()
    c.forward()
    c.backward()
    assert grawa.grawa_window_attention_status() == 0 and time.perf_counter() - start < 5.0
    nan = dict(q=("out", "dq", "dk", "dv"), k=("out", "dq", "dk", "dv"), v=("out", "dq", "dk"), dout=("dq", "dk", "dv"), all=("out", "dq", "dk", "dv"))[which]
    for name in ("out", "dq", "dk", "dv"):
        for t in getattr(c, name):
            assert t.isnan().all() if name in nan else torch.isfinite(t.float()).all(), name


@pytest.mark.parametrize("dim", [64, 128])
def test_infinite_values_of_a_seen_key(dim):
    """An infinity in a value: an infinity or NaN in that element of exactly the rows that see it, and finite numbers beside it."""
    c = Case(torch.float16, 900, 2, 2, dim, left=200, seed=12)
    for t in c.v:
        t[300, 1, 5] = float("inf")
    c.forward()
    for m in range(c.M):
        bad = ~torch.isfinite(c.out[m].float())
        want = torch.zeros_like(bad)
        want[300:501, 1, 5] = True
        # a weight that rounds to zero gives NaN or zero times infinity: not finite either way
        assert torch.equal(bad, want)


def test_rows_past_2_31_elements():
    """q, k, v and their gradients side by side in rows so far apart that the last ones lie past 2^31 elements: the bits of packed ones."""
    import paper_2403_04206_b200 as grawa
    rows, stride = 17000, 131200
    assert rows * stride > 2 ** 31
    wide = torch.empty(rows, stride, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(13)
    at = {name: wide[:, 64 * i:64 * (i + 1)].unflatten(1, (1, 64)) for i, name in enumerate(("q", "k", "v", "dout", "out", "dq", "dk", "dv", "q2", "dq2"))}
    own = {name: torch.randn(rows, 1, 64, generator=gen, device="cuda").bfloat16() for name in at}
    for name in ("q", "k", "v", "dout"):
        at[name].copy_(own[name])
    lse = [torch.empty(1, rows, device="cuda") for _ in range(2)]
    for t, s in zip((own, at), lse):
        one = {k: [v] for k, v in t.items()}
        grawa.grawa_window_attention_forward(one["q"], one["k"], one["v"], one["out"], lse=[s], left=99, sinks=3)
        grawa.grawa_window_attention_backward(one["dout"], one["q"], one["k"], one["v"], one["out"], [s], one["dq"], one["dk"], one["dv"], left=99, sinks=3)
        grawa.grawa_head_rotary_forward(one["q"], None, None, None, one["q2"], None, None)
        grawa.grawa_head_rotary_backward(one["dout"], None, one["q"], None, None, None, one["dq2"], None, None, None, None)
    assert torch.equal(*lse)
    for name in at:
        assert torch.equal(own[name], at[name]), name
