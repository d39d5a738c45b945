"""What the attention operators refuse, on the host and before anything is enqueued (fake addresses, no GPU)."""
import ctypes

import pytest
import torch

import paper_2403_04206_b200 as grawa

STEP = 1 << 24
OK, BAD, NO_SPACE = 0, -1, -4


def table(first, M=2, step=STEP):
    return (ctypes.c_void_p * M)(*[first + m * step for m in range(M)])


T = [table(0x10_0000_0000 * k) for k in range(1, 15)]
NULLS = (ctypes.c_void_p * 2)(0x1000, 0)
WS = 0x1000_0000_0000


def head_forward(dtype=1, pairing=0, q=T[0], k=T[1], qw=T[2], kw=T[3], qo=T[4], ko=T[5], pos=T[6], f=0x7000, rows=10, heads=4, kv=2, dim=64, rotary=64,
                 qs=256, ks=128, qos=256, kos=128, period=0, M=2, eps=1e-6):
    return grawa.library().grawa_head_rotary_forward(dtype, pairing, q, k, qw, kw, qo, ko, pos, f, rows, heads, kv, dim, rotary, qs, ks, qos, kos, period, M, eps, None)


def test_head_rotary_forward_refusals():
    assert head_forward(rows=0) == OK
    for kw in (dict(dtype=3), dict(pairing=2), dict(pairing=-1), dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(M=0), dict(M=65), dict(rows=-1),
               dict(rows=1 << 31), dict(heads=0), dict(kv=-1), dict(dim=0), dict(dim=257, rotary=0, qs=2000, ks=2000, qos=2000, kos=2000), dict(rotary=63),
               dict(rotary=66), dict(rotary=-2), dict(qs=255), dict(ks=127), dict(qos=255), dict(kos=127), dict(qs=1 << 60), dict(f=None), dict(f=0x7004),
               dict(pos=None, period=0), dict(pos=table(0x70_0000_0004)), dict(pos=NULLS), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
               dict(q=NULLS), dict(ko=NULLS), dict(qw=NULLS), dict(q=table(0x10_0000_0001)), dict(qo=table(T[0][0] + 2)), dict(qo=T[0], qos=320),
               dict(ko=T[4]), dict(ko=T[2]), dict(qo=table(T[6][0] + 32)), dict(f=T[4][0] + 64), dict(ko=table(T[0][0] + 16))):
        assert head_forward(**kw) == BAD, kw


def head_backward(dtype=1, qo=T[0], ko=T[1], q=T[2], k=T[3], qw=T[4], kw=T[5], dq=T[6], dk=T[7], dqw=T[8], dkw=T[9], pos=T[10], f=0x7000, rows=1000, heads=4, kv=2,
                  dim=64, rotary=64, qs=256, ks=128, qos=256, kos=128, period=0, M=2, eps=1e-6, acc=0, ws=WS, ws_bytes=1 << 30):
    return grawa.library().grawa_head_rotary_backward(dtype, 0, qo, ko, q, k, qw, kw, dq, dk, dqw, dkw, pos, f, rows, heads, kv, dim, rotary, qs, ks, qos, kos,
                                                      period, M, eps, acc, ws, ws_bytes, None)


def test_head_rotary_backward_refusals():
    assert head_backward(rows=0, acc=1) == OK and head_backward(rows=0, dqw=None, dkw=None) == OK
    size = grawa.grawa_head_rotary_backward_workspace_bytes
    need = size(1000, 2)
    assert need > 0 and size(1, 2) == 0 and size(-1, 2) == 0 and size(10, 0) == 0 and size(10, 65) == 0
    for kw in (dict(ws=None), dict(ws=WS + 8), dict(ws_bytes=need - 1)):
        assert head_backward(**kw) == NO_SPACE, kw
    for kw in (dict(dtype=5), dict(qo=None), dict(ko=None), dict(q=None), dict(dq=None, dk=None, dqw=None, dkw=None), dict(kv=0), dict(dq=T[2]), dict(dk=T[2]),
               dict(dqw=T[4]), dict(dqw=T[9]), dict(dkw=NULLS), dict(dq=T[0], qos=264), dict(dq=T[1]), dict(ws=T[0][0]), dict(ws=T[8][0]), dict(rotary=3)):
        assert head_backward(**kw) == BAD, kw


def attention_forward(dtype=1, q=T[0], k=T[1], v=T[2], out=T[3], lse=T[4], off=T[5], seqs=3, period=0, left=5, right=0, sinks=1, rows=10, heads=4, kv=2, dim=64,
                      qs=256, ks=128, vs=128, os=256, M=2, scale=0.1):
    return grawa.library().grawa_window_attention_forward(dtype, q, k, v, out, lse, off, seqs, period, left, right, sinks, rows, heads, kv, dim, qs, ks, vs, os, M,
                                                          scale, None)


SHAPE_REFUSALS = [dict(dtype=0), dict(dtype=3), dict(M=0), dict(M=65), dict(rows=-1), dict(rows=(1 << 31) - 1), dict(heads=0), dict(kv=0), dict(kv=3), dict(kv=8),
                  dict(dim=0), dict(dim=4), dict(dim=63), dict(dim=136, qs=544, ks=272, vs=272, os=544), dict(qs=255), dict(qs=248), dict(ks=120), dict(vs=132),
                  dict(os=257), dict(qs=1 << 60), dict(left=-1), dict(right=-1), dict(sinks=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
                  dict(scale=float("inf")), dict(seqs=-1), dict(off=None), dict(off=table(0x60_0000_0004)), dict(off=NULLS), dict(q=None), dict(k=None), dict(v=None),
                  dict(out=None), dict(q=NULLS), dict(q=table(0x10_0000_0008)), dict(v=table(0x30_0000_0004)), dict(k=table(0x20_0000_0002))]


@pytest.mark.parametrize("kw", SHAPE_REFUSALS + [dict(out=table(0x40_0000_0008)), dict(out=T[0]), dict(out=table(T[1][0] + 16)), dict(lse=table(T[3][0] + 64)),
                                                 dict(lse=table(0x50_0000_0002)), dict(lse=NULLS), dict(out=T[5]), dict(out=table(T[3][0], 2, 4096))], ids=str)
def test_attention_forward_refusals(kw):
    assert attention_forward(**kw) == BAD


def attention_backward(dtype=1, dout=T[6], q=T[0], k=T[1], v=T[2], out=T[3], lse=T[4], dq=T[7], dk=T[8], dv=T[9], off=T[5], seqs=3, period=0, left=5, right=0, sinks=1,
                       rows=10, heads=4, kv=2, dim=64, qs=256, ks=128, vs=128, os=256, M=2, scale=0.1, ws=WS, ws_bytes=1 << 30):
    return grawa.library().grawa_window_attention_backward(dtype, dout, q, k, v, out, lse, dq, dk, dv, off, seqs, period, left, right, sinks, rows, heads, kv, dim, qs, ks,
                                                           vs, os, M, scale, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", SHAPE_REFUSALS + [dict(dout=None), dict(lse=None), dict(dq=None, dk=None, dv=None), dict(dk=None), dict(dv=None), dict(dq=T[0]),
                                                 dict(dk=T[1]), dict(dv=T[8]), dict(dv=T[4]), dict(dq=T[6]), dict(dq=table(0x80_0000_0008)), dict(ws=T[0][0]),
                                                 dict(ws=T[7][0])], ids=str)
def test_attention_backward_refusals(kw):
    assert attention_backward(**kw) == BAD


def test_attention_scratch():
    size = grawa.grawa_window_attention_backward_workspace_bytes
    need = size(10, 4, 2, 64, 1, 2)
    assert need > 0 and size(2000, 4, 2, 64, 1, 2) > size(2000, 4, 2, 64, 0, 2) == size(2000, 4, 2, 64, 129, 2)
    for bad in ((-1, 4, 2, 64, 1, 2), (10, 0, 2, 64, 1, 2), (10, 4, 0, 64, 1, 2), (10, 4, 2, 0, 1, 2), (10, 4, 2, 64, -1, 2), (10, 4, 2, 64, 1, 0),
                (10, 4, 2, 64, 1, 65)):
        assert size(*bad) == 0
    for kw in (dict(ws=None), dict(ws=WS + 16), dict(ws_bytes=need - 1)):
        assert attention_backward(**kw) == NO_SPACE, kw
    assert attention_forward(rows=0) == OK and attention_backward(rows=0, ws=None) == OK


def test_binding_refuses_tensors_it_cannot_pass():
    """CPU tensors, and whatever else is wrong before an address is taken."""
    q = [torch.zeros(4, 2, 64, dtype=torch.bfloat16)]
    for call in (lambda: grawa.grawa_window_attention_forward([q[0].flatten(1)], q, q, q), lambda: grawa.grawa_window_attention_forward(q, q, q, q, offsets=[q[0][:0, 0, 0]]),
                 lambda: grawa.grawa_head_rotary_forward(q, [q[0][:, :0]], None, None, q, None, None)):
        with pytest.raises(ValueError):
            call()
