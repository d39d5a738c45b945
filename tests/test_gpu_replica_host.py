"""Host side of the replica operators: calls from several threads, and calls that come in the middle of another."""
import threading

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def grawa():
    import paper_2403_04206_b200 as g
    return g


def norm_inputs(rows, cols, kind, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    return dict(dy=[normal(rows, cols).to(kind)], x=[normal(rows, cols).to(kind)], gamma=[normal(cols).to(kind)], mean=[normal(rows) * 0.1], rstd=[1.0 + 0.1 * normal(rows).abs()])


def norm_outputs(d):
    return [[torch.zeros_like(d["x"][0])], [torch.zeros_like(d["gamma"][0])], [torch.zeros_like(d["gamma"][0])]]


def norm_backward(grawa, d, out, **kw):
    grawa.grawa_layernorm_backward(d["dy"], d["x"], d["gamma"], d["mean"], d["rstd"], *out, **kw)


def test_row_lengths_of_one_kernel_from_several_threads(grawa):
    """2048 and 8192 columns of fp32 take the same kernel, with 48 KB of shared memory a CTA and with 192 KB.  The threads call
    the C entry point itself, with tables made beforehand, so that most of their time passes inside it."""
    import ctypes
    lib, threads, turns = grawa.library(), 4, 20000
    cases = [norm_inputs(2, cols, torch.float32, cols) for cols in (2048, 8192)]
    want = []
    for d in cases:
        out = norm_outputs(d)
        norm_backward(grawa, d, out)
        want.append([t[0].clone() for t in out])
    torch.cuda.synchronize()
    wrong, start = [], threading.Barrier(threads)
    outs, streams = [norm_outputs(cases[k % 2]) for k in range(threads)], [torch.cuda.Stream() for _ in range(threads)]

    def work(k):
        d, stream = cases[k % 2], streams[k].cuda_stream
        rows, cols = d["x"][0].shape
        table = [(ctypes.c_void_p * 1)(t[0].data_ptr()) for t in (d["dy"], d["x"], d["gamma"], d["mean"], d["rstd"], *outs[k])]
        start.wait()
        bad = {lib.grawa_layernorm_backward(0, *table, rows, cols, cols, cols, 1, 0, None, 0, stream) for _ in range(turns)}
        if bad != {0}:
            wrong.append(bad)

    workers = [threading.Thread(target=work, args=(k,)) for k in range(threads)]
    for t in workers:
        t.start()
    for t in workers:
        t.join()
    torch.cuda.synchronize()
    assert not wrong, wrong
    for k in range(threads):
        assert all(torch.equal(a[0], b) for a, b in zip(outs[k], want[k % 2]))


def test_a_call_in_the_middle_of_another(grawa, monkeypatch):
    """What Python runs between a call's checks and its launch (a finalizer, for one) may make calls of its own."""
    from paper_2403_04206_b200 import binding
    outer, inner = (norm_inputs(300, 100, torch.bfloat16, seed) for seed in (1, 2))
    want, got, other, extra = (norm_outputs(d) for d in (outer, outer, inner, inner))
    norm_backward(grawa, outer, want)
    norm_backward(grawa, inner, other)
    assert grawa.grawa_layernorm_backward_workspace_bytes(300, 100, 1, aligned=False) > 0
    scratch, nested = binding._scratch, []

    def interrupted(*args):
        if not nested:
            nested.append(True)
            norm_backward(grawa, inner, extra)
        return scratch(*args)

    monkeypatch.setattr(binding, "_scratch", interrupted)
    norm_backward(grawa, outer, got)
    assert nested
    for a, b in zip(want + other, got + extra):
        assert torch.equal(a[0], b[0])
