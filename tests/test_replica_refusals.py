"""What the replica operators refuse, on the host and before anything is enqueued (fake addresses, no GPU)."""
import ctypes

import pytest

import paper_2403_04206_b200 as grawa

STEP = 1 << 24
OK, BAD, NO_SPACE = 0, -1, -4


def table(first, M=2, step=STEP):
    return (ctypes.c_void_p * M)(*[first + m * step for m in range(M)])


X, R, Y, D, E, F, G, H = (table(0x10_0000_0000 * k) for k in range(1, 9))
NULLS = (ctypes.c_void_p * 2)(0x1000, 0)


def forward_dropout(dtype=1, x=X, r=R, y=Y, n=1000, M=2, p=0.1, seed=1, offset=2, counter=None):
    return grawa.library().grawa_dropout_forward(dtype, x, r, y, n, M, p, seed, offset, counter, None)


def test_dropout_refusals():
    assert forward_dropout(n=0) == OK
    for kw in (dict(dtype=3), dict(dtype=-1), dict(x=None), dict(y=None), dict(M=0), dict(M=65), dict(n=-1), dict(n=(1 << 56) + 1), dict(p=1.0),
               dict(p=-0.1), dict(p=float("nan")), dict(p=float("inf")), dict(x=NULLS), dict(y=NULLS), dict(r=NULLS), dict(counter=0x1004),
               dict(x=table(0x10_0000_0001)),                                    # not aligned to the element size
               dict(x=table(Y[0] + 8)),                                          # partly the same buffer
               dict(x=table(Y[1], 2, -STEP)),                                    # another worker's output
               dict(r=table(Y[0] - 8)), dict(y=table(Y[0], 2, 1998)), dict(counter=Y[0] + 16)):
        assert forward_dropout(**kw) == BAD, kw
    assert grawa.library().grawa_dropout_backward(1, X, None, 10, 2, 0.1, 1, 1, None, None) == BAD
    assert grawa.library().grawa_dropout_backward(1, X, table(X[0] + 4), 10, 2, 0.1, 1, 1, None, None) == BAD


def norm_forward(dtype=1, x=X, gamma=R, beta=D, y=Y, mean=E, rstd=F, rows=10, cols=100, xs=100, ys=100, M=2, eps=1e-5):
    return grawa.library().grawa_layernorm_forward(dtype, x, gamma, beta, y, mean, rstd, rows, cols, xs, ys, M, eps, None)


def test_layernorm_forward_refusals():
    assert norm_forward(rows=0) == OK
    for kw in (dict(dtype=7), dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(M=0), dict(M=65), dict(rows=-1), dict(rows=1 << 31),
               dict(cols=0), dict(cols=-5), dict(cols=1 << 31, xs=1 << 31, ys=1 << 31), dict(xs=99), dict(ys=99), dict(xs=1 << 60), dict(eps=-1e-5),
               dict(eps=float("nan")), dict(eps=float("inf")), dict(x=NULLS), dict(gamma=NULLS), dict(beta=NULLS), dict(y=NULLS), dict(mean=NULLS),
               dict(y=X), dict(y=table(X[0] + 1998)), dict(y=R), dict(y=D), dict(mean=table(Y[0] + 1996)), dict(rstd=E),
               dict(mean=table(0x50_0000_0002)), dict(y=table(0x30_0000_0001)), dict(y=table(Y[0], 2, 198), ys=100),
               dict(y=table(Y[0], 2, 198), ys=200)):                             # rows of two workers overlap by one element
        assert norm_forward(**kw) == BAD, kw


def norm_backward(dtype=1, dy=X, x=R, gamma=D, mean=E, rstd=F, dx=Y, dgamma=G, dbeta=H, rows=1000, cols=100, xs=100, ys=100, M=2, acc=0,
                  ws=0x90_0000_0000, ws_bytes=1 << 30):
    return grawa.library().grawa_layernorm_backward(dtype, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, rows, cols, xs, ys, M, acc, ws, ws_bytes, None)


def test_layernorm_backward_refusals():
    assert norm_backward(rows=0, acc=1) == OK
    size = grawa.grawa_layernorm_backward_workspace_bytes
    need = size(1000, 100, 2)
    assert need > 0 and size(4, 100, 2) == 0 and size(150, 768, 2) > 0 and size(150, 768, 2, aligned=True) == 0
    for bad in ((-1, 100, 2), (10, 0, 2), (10, 100, 0), (10, 100, 65)):
        assert grawa.grawa_layernorm_backward_workspace_bytes(*bad) == 0
    for kw in (dict(ws=None), dict(ws=0x90_0000_0008), dict(ws_bytes=need - 1), dict(ws_bytes=0)):
        assert norm_backward(**kw) == NO_SPACE, kw
    for kw in (dict(dtype=5), dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(dx=None, dgamma=None, dbeta=None), dict(M=65),
               dict(cols=0), dict(xs=99), dict(ys=99), dict(dx=X), dict(dx=R), dict(dgamma=D), dict(dgamma=H), dict(dbeta=NULLS), dict(mean=NULLS),
               dict(ws=X[0] + 16), dict(ws=Y[0] + 16), dict(ws=G[0])):
        assert norm_backward(**kw) == BAD, kw


@pytest.mark.parametrize("rows,cols,M", [(1, 1, 1), (5, 64, 64), (10 ** 6, 768, 8), (10 ** 6, 100_000, 1), (77, 8193, 3)])
def test_workspace_does_not_grow_with_the_rows_without_end(rows, cols, M):
    # at most 16 CTAs an SM's worth of column sums, whatever the rows
    assert grawa.grawa_layernorm_backward_workspace_bytes(rows, cols, M) <= max(148 * 16, M) * 2 * 4 * max(64, 2 * cols)


def ffn_forward(dtype=1, act=0, x=X, wg=R, wu=D, h=Y, gate=E, up=F, rows=64, d_in=64, hidden=64, M=2, ws=None, ws_bytes=0):
    return grawa.library().grawa_gated_ffn_forward(dtype, act, x, wg, wu, h, gate, up, rows, d_in, hidden, M, ws, ws_bytes, None)


def ffn_backward(dtype=1, act=0, dh=X, x=R, wg=D, wu=Y, gate=E, up=F, dx=G, dwg=H, dwu=table(0x90_0000_0000), rows=64, d_in=64, hidden=64, M=2, acc=0,
                 ws=0xa0_0000_0000, ws_bytes=1 << 30):
    return grawa.library().grawa_gated_ffn_backward(dtype, act, dh, x, wg, wu, gate, up, dx, dwg, dwu, rows, d_in, hidden, M, acc, ws, ws_bytes, None)


def test_gated_ffn_refusals():
    size = grawa.grawa_gated_ffn_workspace_bytes
    assert ffn_forward(rows=0) == OK and ffn_backward(rows=0, acc=1) == OK
    assert size(64, 64, 64, 2) == 0 and size(64, 60, 64, 2) > 0 and size(64, 64, 64, 2, aligned=False) > 0
    assert size(64, 64, 64, 2, backward=True) == 2 * 2 * 64 * 64 * 2 and size(0, 64, 64, 2, backward=True) == 0
    assert size(-1, 64, 64, 2, True) == 0 and size(64, 0, 64, 2, True) == 0 and size(64, 64, 64, 65, True) == 0
    for kw in (dict(dtype=0), dict(dtype=3), dict(act=3), dict(act=-1), dict(x=None), dict(wg=None), dict(wu=None), dict(h=None), dict(gate=None),
               dict(up=None), dict(rows=-1), dict(d_in=0), dict(hidden=0), dict(M=0), dict(M=65), dict(rows=1 << 25), dict(d_in=1 << 25),
               dict(d_in=1 << 22, hidden=1 << 22), dict(x=NULLS), dict(wu=NULLS), dict(h=NULLS), dict(up=NULLS), dict(h=X), dict(h=R), dict(gate=Y),
               dict(up=E), dict(x=table(0x10_0000_0001)), dict(h=table(X[1] + 8190))):
        assert ffn_forward(**kw) == BAD, kw
    for kw in (dict(d_in=60), dict(x=table(X[0] + 2)), dict(wg=table(R[0] + 8)), dict(d_in=60, ws=0xa0_0000_0000, ws_bytes=size(64, 60, 64, 2) - 1),
               dict(d_in=60, ws=0xa0_0000_0010, ws_bytes=1 << 30)):
        assert ffn_forward(**kw) == NO_SPACE, kw
    for kw in (dict(dtype=0), dict(act=9), dict(dh=None), dict(gate=None), dict(up=None), dict(dwg=None), dict(dwu=None), dict(dx=None, dwg=None, dwu=None),
               dict(dx=X), dict(dx=R), dict(dwg=D), dict(dwu=H), dict(ws=X[0] - 256), dict(ws=H[0])):
        assert ffn_backward(**kw) == BAD, kw
    for kw in (dict(ws=None), dict(ws_bytes=size(64, 64, 64, 2, True) - 1), dict(ws=0xa0_0000_0080), dict(wu=table(Y[0] + 2), ws_bytes=size(64, 64, 64, 2, True))):
        assert ffn_backward(**kw) == NO_SPACE, kw


def test_the_marshaller_names_the_wrong_table():
    import torch
    from paper_2403_04206_b200 import build
    build.build_marshal()
    from paper_2403_04206_b200 import _marshal
    x = [torch.zeros(4, 8) for _ in range(2)]
    for first, specs, error, word in (
            (x, (("x", x, 4, 8, 1),), ValueError, "current CUDA device"), (x, (("y", None, 4, 8, 0),), TypeError, "y: expected a list"),
            (x, (("y", x[:1], 4, 8, 0),), ValueError, "one entry per worker"), (x, (("y", [1, 2], 4, 8, 0),), TypeError, "expected tensors"),
            (x, (("y", [t.half() for t in x], 4, 8, 0),), TypeError, "expected Float, got Half"),
            ([t.double() for t in x], (), TypeError, "float32, bfloat16 or float16"), ([], (), ValueError, "workers"),
            (x * 40, (), ValueError, "1 to 64 workers"), (7, (), TypeError, "len"), (x, (("y", 3, 4, 8, 0),), TypeError, "list of tensors")):
        with pytest.raises(error, match=word):
            _marshal.tables(first, 0, specs)
    assert _marshal.tables(x, 0, (("r", None, 4, 8, 2),)) == (0, 0, 0)
