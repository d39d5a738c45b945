"""Host side of the replica operators: calls from several threads, calls that come in the middle of another, and buffers
that stand between the rows of others."""
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


def test_buffers_in_the_padding_of_others(grawa):
    """Parameters, statistics and gradients that stand between the rows of an output share nothing with it."""
    rows, cols, stride = 9, 40, 200
    gen = torch.Generator(device="cuda").manual_seed(5)
    x, dy = (torch.randn(rows, cols, generator=gen, device="cuda") for _ in range(2))
    gamma, beta = (torch.randn(cols, generator=gen, device="cuda") for _ in range(2))
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
    grawa.grawa_layernorm_forward([x], [gamma], [beta], [y], mean=[mean], rstd=[rstd])
    grawa.grawa_layernorm_backward([dy], [x], [gamma], [mean], [rstd], [dx], [dgamma], [dbeta])

    flat = torch.full((rows, stride), 7.0, device="cuda")      # row 0: y and gamma; row 3: y, beta and mean; last row: y, beta ...
    rows_of = flat[:, :cols]
    g, b, mu, s = flat[0, cols:2 * cols], flat[3, 100:100 + cols], flat[3, 150:150 + rows], flat[7, stride - rows:]
    g.copy_(gamma)
    b.copy_(beta)
    grawa.grawa_layernorm_forward([x], [g], [b], [rows_of], mean=[mu], rstd=[s])
    for got, want in ((rows_of, y), (mu, mean), (s, rstd), (g, gamma), (b, beta)):
        assert torch.equal(got, want)
    flat.fill_(7.0)
    x_rows = flat[:, :cols]
    x_rows.copy_(x)
    dg, db, out = flat[2, cols:2 * cols], flat[2, 2 * cols:3 * cols], flat[:, 148:148 + cols]
    grawa.grawa_layernorm_backward([dy], [x_rows], [gamma], [mean], [rstd], [out], [dg], [db])
    for got, want in ((out, dx), (dg, dgamma), (db, dbeta), (x_rows, x)):
        assert torch.equal(got, want)
    untouched = torch.ones_like(flat, dtype=torch.bool)
    untouched[:, :cols] = untouched[:, 148:148 + cols] = untouched[2, cols:3 * cols] = False
    assert (flat[untouched] == 7.0).all()
    for bad in (flat[2, cols - 1:2 * cols - 1], flat.view(-1)[3 * stride - cols + 1:3 * stride + 1]):
        with pytest.raises(grawa.GrawaError):                 # one element of it in a row, in front or behind
            grawa.grawa_layernorm_forward([x], [bad], [beta], [rows_of])
