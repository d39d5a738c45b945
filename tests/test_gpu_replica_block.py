"""The replica operators together, as a local phase uses them: M workers whose parameters stand in flat bfloat16 vectors run
    z = r + dropout(gated_ffn(layernorm(r)) Wd)
(the product with Wd is the caller's, a library product) forward and backward on two micro-batches, with the gradients
added up in the flat gradient vectors, and the averaging step reads those.  Against the whole chain in 64 bits with
torch's own derivatives, and the step against the oracle on the gradients as they stand."""
import numpy as np
import pytest
import torch

import oracle
from replica_util import keep_mask

pytestmark = pytest.mark.gpu
M, ROWS, WIDTH, HIDDEN, P, SEED, EPS = 3, 75, 96, 200, 0.2, 77, 1e-5
# the layers of a worker's vector; an odd one in front, so that everything behind it stands at an odd place
SIZES = dict(embedding=11, gamma=WIDTH, beta=WIDTH, w_gate=HIDDEN * WIDTH, w_up=HIDDEN * WIDTH, w_down=WIDTH * HIDDEN)
SHAPES = dict(gamma=(WIDTH,), beta=(WIDTH,), w_gate=(HIDDEN, WIDTH), w_up=(HIDDEN, WIDTH), w_down=(WIDTH, HIDDEN))
OFFSETS = np.cumsum([0] + list(SIZES.values()))


def views(flat):
    at = dict(zip(SIZES, OFFSETS))
    return {k: [t[at[k]:at[k] + SIZES[k]].view(s) for t in flat] for k, s in SHAPES.items()}


def local_pass(grawa, p, g, r, dz, offset, first):
    """One micro-batch: z, the gradient of r, and the parameters' gradients added to (or, first, put in) g."""
    def like(shape, kind=torch.bfloat16):
        return [torch.empty(shape, dtype=kind, device="cuda") for _ in range(M)]

    n, mean, rstd = like((ROWS, WIDTH)), like(ROWS, torch.float32), like(ROWS, torch.float32)
    grawa.grawa_layernorm_forward(r, p["gamma"], p["beta"], n, EPS, mean=mean, rstd=rstd)
    h, a, u = (like((ROWS, HIDDEN)) for _ in range(3))
    grawa.grawa_gated_ffn_forward(n, p["w_gate"], p["w_up"], h, activation="silu", gate_out=a, up_out=u)
    o = [t @ w.T for t, w in zip(h, p["w_down"])]
    z = like((ROWS, WIDTH))
    grawa.grawa_dropout_forward(o, z, P, SEED, offset, residual=r)
    # backward
    do, dn, dr = (like((ROWS, WIDTH)) for _ in range(3))
    grawa.grawa_dropout_backward(dz, do, P, SEED, offset)
    dh = [t @ w for t, w in zip(do, p["w_down"])]
    for k in range(M):
        dw = do[k].T @ h[k]
        g["w_down"][k].copy_(dw if first else g["w_down"][k] + dw)
    grawa.grawa_gated_ffn_backward(dh, n, p["w_gate"], p["w_up"], a, u, dn, g["w_gate"], g["w_up"], activation="silu", accumulate=not first)
    grawa.grawa_layernorm_backward(dn, r, p["gamma"], mean, rstd, dr, g["gamma"], g["beta"], accumulate=not first)
    return z, [x + y for x, y in zip(dr, dz)]


def test_two_micro_batches_and_the_averaging_step():
    import paper_2403_04206_b200 as grawa
    gen = torch.Generator(device="cuda").manual_seed(1)

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).bfloat16()

    n = int(OFFSETS[-1])
    flat = [normal(n, scale=WIDTH ** -0.5) for _ in range(M)]
    for k in range(M):
        views(flat)["gamma"][k].add_(1.0)
    grads = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(M)]
    for t in grads:
        t[:11] = 0.25
    p, g = views(flat), views(grads)
    batches = [([normal(ROWS, WIDTH) for _ in range(M)], [normal(ROWS, WIDTH, scale=0.1) for _ in range(M)]) for _ in range(2)]
    got = [local_pass(grawa, p, g, r, dz, offset, offset == 0) for offset, (r, dz) in enumerate(batches)]
    assert grawa.grawa_gated_ffn_status() == 0

    for m in range(M):
        wide = {k: v[m].double().requires_grad_() for k, v in p.items()}
        for offset, (r, dz) in enumerate(batches):
            x = r[m].double().requires_grad_()
            centred = x - x.mean(-1, keepdim=True)
            h = centred / (centred.square().mean(-1, keepdim=True) + EPS).sqrt() * wide["gamma"] + wide["beta"]
            a = h @ wide["w_gate"].T
            o = (a * torch.sigmoid(a) * (h @ wide["w_up"].T)) @ wide["w_down"].T
            keep = keep_mask(SEED, offset, m, ROWS * WIDTH, P).view(ROWS, WIDTH).cuda()
            z = x + o * keep / (1.0 - float(np.float32(P)))
            (z * dz[m].double()).sum().backward()
            # Each tensor on the way carries one rounding of 2^-8 at most, of itself in the 2-norm; a value passes
            # through at most 10 of them, none of which the maps in between make larger by more than 2 here.
            for what, mine, want in (("z", got[offset][0][m], z), ("dr", got[offset][1][m], x.grad)):
                assert (mine.double() - want.detach()).norm() <= 20 * 2.0 ** -8 * want.detach().norm(), what
        for k, v in wide.items():
            assert (g[k][m].double() - v.grad).norm() <= 20 * 2.0 ** -8 * v.grad.norm(), k
    assert all((t[:11] == 0.25).all() for t in grads)

    before, taken = ([t.float().cpu().numpy() for t in v] for v in (flat, grads))
    centre = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    grawa.grawa_step_typed("lgrawa", flat, grads, 0.5, OFFSETS, centre)
    assert grawa.grawa_last_step_status() == 0
    want = oracle.step(before, taken, 0.5, "lgrawa", OFFSETS)
    tol = 2e-6 * max(float(np.abs(t).max()) for t in before)
    for mine, ref in [(centre, want["center"])] + list(zip(flat, want["workers"])):
        assert (np.abs(mine.float().cpu().numpy() - ref) <= tol + 2.0 ** -8 * np.abs(ref)).all()


def test_the_chain_captured_and_replayed():
    """The whole pass in one graph: the same bits as eager calls, with a new mask from the device's counter at every replay."""
    import paper_2403_04206_b200 as grawa
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = [torch.randn(ROWS, WIDTH, generator=gen, device="cuda").bfloat16() for _ in range(M)]
    w = [[torch.randn(HIDDEN, WIDTH, generator=gen, device="cuda").bfloat16() for _ in range(M)] for _ in range(2)]
    n, h, y = [torch.empty_like(t) for t in x], [torch.empty(ROWS, HIDDEN, dtype=torch.bfloat16, device="cuda") for _ in range(M)], []
    y = [torch.empty_like(t) for t in h]
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")

    def chain(offset, counter):
        grawa.grawa_layernorm_forward(x, None, None, n, EPS)
        grawa.grawa_gated_ffn_forward(n, w[0], w[1], h, activation="gelu")
        grawa.grawa_dropout_forward(h, y, P, SEED, offset, offset_counter=counter)

    want = []
    for offset in range(3):
        chain(offset, None)
        want.append([t.clone() for t in y])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain(0, counter)
        counter += 1
    counter.zero_()
    for offset in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(y, want[offset]))
    assert grawa.grawa_gated_ffn_status() == 0


def test_two_host_threads_on_their_own_streams():
    """The same calls from two threads at once give the bits that one thread gets."""
    import threading

    import paper_2403_04206_b200 as grawa
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows, width, hidden, turns = 200, 264, 300, 30

    def draw(*shape):
        return [torch.randn(*shape, generator=gen, device="cuda").bfloat16() for _ in range(M)]

    inputs = [dict(x=draw(rows, width), wg=draw(hidden, width), wu=draw(hidden, width), dh=draw(rows, hidden), gamma=draw(width), beta=draw(width)) for _ in range(2)]

    def chain(d):
        n, dx, dn = ([torch.empty_like(t) for t in d["x"]] for _ in range(3))
        h, a, u, y = ([torch.empty_like(t) for t in d["dh"]] for _ in range(4))
        mean, rstd = ([torch.empty(rows, device="cuda") for _ in range(M)] for _ in range(2))
        dwg, dwu, dg, db = ([torch.empty_like(t) for t in d[k]] for k in ("wg", "wu", "gamma", "beta"))
        grawa.grawa_layernorm_forward(d["x"], d["gamma"], d["beta"], n, EPS, mean=mean, rstd=rstd)
        grawa.grawa_gated_ffn_forward(n, d["wg"], d["wu"], h, activation="gelu", gate_out=a, up_out=u)
        grawa.grawa_dropout_forward(h, y, P, SEED, 1, residual=d["dh"])
        grawa.grawa_gated_ffn_backward(d["dh"], n, d["wg"], d["wu"], a, u, dn, dwg, dwu, activation="gelu")
        grawa.grawa_layernorm_backward(dn, d["x"], d["gamma"], mean, rstd, dx, dg, db)
        return n + y + dx + dwg + dwu + dg + db

    want = [chain(d) for d in inputs]
    torch.cuda.synchronize()
    wrong = []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()) as _:
                for _ in range(turns):
                    got = chain(inputs[k])
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(p, q) for p, q in zip(got, want[k])):
                        wrong.append(k)
        except Exception as e:                                # noqa: BLE001  (told to the test's own thread)
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(k,)) for k in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and grawa.grawa_gated_ffn_status() == 0


def test_scratch_and_counters_of_the_caller():
    import paper_2403_04206_b200 as grawa
    rows, width, hidden = 300, 96, 128
    x, dy = ([torch.randn(rows, width, device="cuda").bfloat16()] for _ in range(2))
    stats = [[torch.zeros(rows, device="cuda")], [torch.ones(rows, device="cuda")]]
    dx, dg, db = [torch.empty_like(x[0])], [torch.empty(width, device="cuda").bfloat16()], [torch.empty(width, device="cuda").bfloat16()]
    need = grawa.grawa_layernorm_backward_workspace_bytes(rows, width, 1, aligned=True)
    assert need > 0
    own = torch.full((need,), 255, dtype=torch.uint8, device="cuda")             # NaN everywhere: its contents do not matter
    grawa.grawa_layernorm_backward(dy, x, None, *stats, dx, dg, db, workspace=own)
    first = [t.clone() for t in (dx[0], dg[0], db[0])]
    grawa.grawa_layernorm_backward(dy, x, None, *stats, dx, dg, db)
    assert all(torch.equal(a, b) for a, b in zip(first, (dx[0], dg[0], db[0])))
    with pytest.raises(grawa.GrawaError, match="workspace"):
        grawa.grawa_layernorm_backward(dy, x, None, *stats, dx, dg, db, workspace=own[:need - 16])
    with pytest.raises(ValueError, match="workspace"):
        grawa.grawa_layernorm_backward(dy, x, None, *stats, dx, dg, db, workspace=own.cpu())
    w = [[torch.randn(hidden, width, device="cuda").bfloat16()] for _ in range(2)]
    h = [[torch.randn(rows, hidden, device="cuda").bfloat16()] for _ in range(3)]
    dw = [[torch.empty_like(w[0][0])] for _ in range(2)]
    need = grawa.grawa_gated_ffn_workspace_bytes(rows, width, hidden, 1, backward=True)
    own = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    grawa.grawa_gated_ffn_backward(h[0], x, *w, h[1], h[2], dx, *dw, workspace=own)
    first = [t.clone() for t in (dx[0], dw[0][0], dw[1][0])]
    grawa.grawa_gated_ffn_backward(h[0], x, *w, h[1], h[2], dx, *dw)
    assert all(torch.equal(a, b) for a, b in zip(first, (dx[0], dw[0][0], dw[1][0])))
    y = [torch.empty_like(x[0])]
    for bad, error in ((torch.zeros(1, dtype=torch.int64), ValueError), (torch.zeros(1, device="cuda"), TypeError), (torch.zeros(1, dtype=torch.int32, device="cuda"), TypeError)):
        with pytest.raises(error, match="offset_counter"):
            grawa.grawa_dropout_forward(x, y, P, SEED, offset_counter=bad)
