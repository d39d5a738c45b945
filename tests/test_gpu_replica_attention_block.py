"""An attention sub-layer as a local phase uses it: M workers whose parameters stand in flat bfloat16 vectors run
    z = r + dropout(attention(rotate(norm(q)), rotate(norm(k)), v) Wo),  (q, k, v) = layernorm(r) Wqkv
(the products with Wqkv and Wo are the caller's, library products) forward and backward on two micro-batches of packed texts, with
the gradients added up in the flat gradient vectors, and the averaging step reads those.  Against the whole chain in 64 bits with
torch's own derivatives, and the step against the oracle on the gradients as they stand."""
import numpy as np
import pytest
import torch

import oracle
from attention_util import turn64, visible
from replica_util import keep_mask

pytestmark = pytest.mark.gpu
M, ROWS, HEADS, KV, DIM, P, SEED, EPS, LEFT, SINKS = 3, 150, 4, 2, 32, 0.1, 5, 1e-5, 40, 2
WIDTH, WIDE = HEADS * DIM, (HEADS + 2 * KV) * DIM
# the layers of a worker's vector; an odd one in front, so that everything behind it stands at an odd place
SHAPES = dict(embedding=(7,), gamma=(WIDTH,), beta=(WIDTH,), w_qkv=(WIDE, WIDTH), q_weight=(DIM,), k_weight=(DIM,), w_o=(WIDTH, WIDTH))
OFFSETS = np.cumsum([0] + [int(np.prod(s)) for s in SHAPES.values()])
ENDS = [[0, 60, 61, 150], [0, 0, 149, 150], [0, 10, 100, 150]]
FREQUENCIES = 100.0 ** -torch.linspace(0, 1, DIM // 2, dtype=torch.float64)


def views(flat):
    return {k: [t[a:b].view(s) for t in flat] for (k, s), a, b in zip(SHAPES.items(), OFFSETS, OFFSETS[1:])}


class Pass:
    """One micro-batch on buffers of its own."""

    def __init__(self, r, dz):
        def like(*shape, kind=torch.bfloat16):
            return [torch.empty(shape, dtype=kind, device="cuda") for _ in range(M)]

        self.r, self.dz = r, dz
        self.n, self.mean, self.rstd, self.z = like(ROWS, WIDTH), like(ROWS, kind=torch.float32), like(ROWS, kind=torch.float32), like(ROWS, WIDTH)
        self.qkv, self.dqkv = like(ROWS, HEADS + 2 * KV, DIM), like(ROWS, HEADS + 2 * KV, DIM)
        self.q, self.k, self.o, self.lse = like(ROWS, HEADS, DIM), like(ROWS, KV, DIM), like(ROWS, HEADS, DIM), like(HEADS, ROWS, kind=torch.float32)
        self.dq, self.dk, self.dn, self.dr, self.dout = like(ROWS, HEADS, DIM), like(ROWS, KV, DIM), like(ROWS, WIDTH), like(ROWS, WIDTH), like(ROWS, WIDTH)
        self.offsets = [torch.tensor(e, device="cuda") for e in ENDS]
        self.positions = [torch.arange(ROWS, device="cuda") - torch.tensor(e, device="cuda")[torch.searchsorted(torch.tensor(e, device="cuda"), torch.arange(ROWS, device="cuda"),
                                                                                                                right=True) - 1] for e in ENDS]
        self.f = FREQUENCIES.cuda()

    def run(self, grawa, p, g, offset, first):
        def heads(t):
            return [x[:, :HEADS] for x in t], [x[:, HEADS:HEADS + KV] for x in t], [x[:, HEADS + KV:] for x in t]

        where, mask = dict(positions=self.positions, eps=EPS), dict(offsets=self.offsets, left=LEFT, sinks=SINKS)
        grawa.grawa_layernorm_forward(self.r, p["gamma"], p["beta"], self.n, EPS, mean=self.mean, rstd=self.rstd)
        for m in range(M):
            torch.mm(self.n[m], p["w_qkv"][m].T, out=self.qkv[m].flatten(1))
        q, k, v = heads(self.qkv)
        grawa.grawa_head_rotary_forward(q, k, p["q_weight"], p["k_weight"], self.q, self.k, self.f, **where)
        grawa.grawa_window_attention_forward(self.q, self.k, v, self.o, lse=self.lse, **mask)
        y = [o.flatten(1) @ w.T for o, w in zip(self.o, p["w_o"])]
        grawa.grawa_dropout_forward(y, self.z, P, SEED, offset, residual=self.r)
        # backward
        grawa.grawa_dropout_backward(self.dz, self.dout, P, SEED, offset)
        do = [(t @ w).view(ROWS, HEADS, DIM) for t, w in zip(self.dout, p["w_o"])]
        dq, dk, dv = heads(self.dqkv)
        grawa.grawa_window_attention_backward(do, self.q, self.k, v, self.o, self.lse, self.dq, self.dk, dv, **mask)
        grawa.grawa_head_rotary_backward(self.dq, self.dk, q, k, p["q_weight"], p["k_weight"], dq, dk, g["q_weight"], g["k_weight"], self.f,
                                         accumulate=not first, **where)
        for m in range(M):
            for name, left, right in (("w_o", self.dout[m], self.o[m].flatten(1)), ("w_qkv", self.dqkv[m].flatten(1), self.n[m])):
                dw = left.T @ right
                g[name][m].copy_(dw if first else g[name][m] + dw)
            torch.mm(self.dqkv[m].flatten(1), p["w_qkv"][m], out=self.dn[m])
        grawa.grawa_layernorm_backward(self.dn, self.r, p["gamma"], self.mean, self.rstd, self.dr, g["gamma"], g["beta"], accumulate=not first)


def inputs(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).bfloat16()

    flat = [normal(int(OFFSETS[-1]), scale=WIDTH ** -0.5) for _ in range(M)]
    for k in range(M):
        for name in ("gamma", "q_weight", "k_weight"):
            views(flat)[name][k].add_(1.0)
    return flat, [Pass([normal(ROWS, WIDTH) for _ in range(M)], [normal(ROWS, WIDTH, scale=0.1) for _ in range(M)]) for _ in range(2)]


def test_two_micro_batches_and_the_averaging_step():
    import paper_2403_04206_b200 as grawa
    flat, passes = inputs(1)
    n = int(OFFSETS[-1])
    grads = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(M)]
    for t in grads:
        t[:7] = 0.25
    p, g = views(flat), views(grads)
    for offset, one in enumerate(passes):
        one.run(grawa, p, g, offset, offset == 0)
    assert grawa.grawa_window_attention_status() == 0

    def rms(x):
        return x / (x.square().mean(-1, keepdim=True) + EPS).sqrt()

    for m in range(M):
        wide = {k: v[m].double().requires_grad_() for k, v in p.items()}
        seen = visible(ROWS, list(zip(ENDS[m], ENDS[m][1:])), LEFT, 0, SINKS, "cuda")
        for offset, one in enumerate(passes):
            x = one.r[m].double().requires_grad_()
            centred = x - x.mean(-1, keepdim=True)
            h = centred / (centred.square().mean(-1, keepdim=True) + EPS).sqrt() * wide["gamma"] + wide["beta"]
            q, k, v = (h @ wide["w_qkv"].T).view(ROWS, -1, DIM).split([HEADS, KV, KV], 1)
            q, k = (turn64(rms(t) * wide[w], one.positions[m], one.f, "halves")[0] for t, w in ((q, "q_weight"), (k, "k_weight")))
            q, k, v = (t.transpose(0, 1).repeat_interleave(HEADS // t.shape[1], 0) for t in (q, k, v))
            weights = torch.softmax((q @ k.mT * DIM ** -0.5).masked_fill(~seen, -torch.inf), -1)
            o = (weights @ v).transpose(0, 1).flatten(1) @ wide["w_o"].T
            keep = keep_mask(SEED, offset, m, ROWS * WIDTH, P).view(ROWS, WIDTH).cuda()
            z = x + o * keep / (1.0 - float(np.float32(P)))
            (z * one.dz[m].double()).sum().backward()
            # Each tensor on the way carries one rounding of 2^-8 at most, of itself in the 2-norm, and P and dS one more; a value
            # passes through at most 14 of them, none of which the maps in between make larger by more than 2 here.
            for what, mine, want in (("z", one.z[m], z), ("dr", one.dr[m].double() + one.dz[m].double(), x.grad)):
                assert (mine.double() - want.detach()).norm() <= 28 * 2.0 ** -8 * want.detach().norm(), what
        for k, v in wide.items():
            if k != "embedding":
                assert (g[k][m].double() - v.grad).norm() <= 28 * 2.0 ** -8 * v.grad.norm(), k
    assert all((t[:7] == 0.25).all() for t in grads)

    before, taken = ([t.float().cpu().numpy() for t in v] for v in (flat, grads))
    centre = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    grawa.grawa_step_typed("lgrawa", flat, grads, 0.5, OFFSETS, centre)
    assert grawa.grawa_last_step_status() == 0
    want = oracle.step(before, taken, 0.5, "lgrawa", OFFSETS)
    tol = 2e-6 * max(float(np.abs(t).max()) for t in before)
    for mine, ref in [(centre, want["center"])] + list(zip(flat, want["workers"])):
        assert (np.abs(mine.float().cpu().numpy() - ref) <= tol + 2.0 ** -8 * np.abs(ref)).all()


def test_the_chain_captured_and_replayed_beside_another():
    """Two captured passes, each with scratch of its own, replayed on two streams at once: the same bits as eager ones.  (Each is
    captured on a stream of its own, as the library products' scratch belongs to the stream.)"""
    import paper_2403_04206_b200 as grawa
    flat, passes = inputs(2)
    p = views(flat)
    results, graphs, want = [], [], []
    streams = [torch.cuda.Stream() for _ in passes]
    for i, one in enumerate(passes):
        grads = [torch.zeros(int(OFFSETS[-1]), dtype=torch.bfloat16, device="cuda") for _ in range(M)]
        g = views(grads)
        results.append(one.z + one.dr + one.dqkv + grads)
        one.run(grawa, p, g, i, True)
        want.append([t.clone() for t in results[-1]])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=streams[i]):
            one.run(grawa, p, g, i, True)
        graphs.append(graph)
    for t in results[0] + results[1]:
        t.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for got, ref in zip(results, want):
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_two_host_threads_on_their_own_streams():
    import threading
    import paper_2403_04206_b200 as grawa
    flat, passes = inputs(3)
    p = views(flat)
    grads = [[torch.zeros(int(OFFSETS[-1]), dtype=torch.bfloat16, device="cuda") for _ in range(M)] for _ in passes]
    for i, one in enumerate(passes):
        one.run(grawa, p, views(grads[i]), i, True)
    want = [[t.clone() for t in one.z + one.dr + one.dqkv + g] for one, g in zip(passes, grads)]
    torch.cuda.synchronize()
    errors = []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    passes[i].run(grawa, p, views(grads[i]), i, True)
                torch.cuda.current_stream().synchronize()
        except Exception as e:                                # reported by the main thread
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for one, g, ref in zip(passes, grads, want):
        assert all(torch.equal(a, b) for a, b in zip(one.z + one.dr + one.dqkv + g, ref))
