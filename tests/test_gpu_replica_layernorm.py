"""Layer norm over all workers, both directions, against the definition in 64 bits."""
import pytest
import torch

from replica_util import EPS32, TYPES, check, layernorm64, layernorm_backward64

pytestmark = pytest.mark.gpu
EPS = 1e-5
# one word, ragged words, each kernel's edge (64, 256, 512, 768, 1024, 8192, 16384) and both sides of it
COLS = [1, 2, 7, 8, 63, 64, 65, 72, 255, 256, 258, 500, 512, 513, 768, 770, 776, 1000, 1023, 1024, 1025, 1032, 4100, 8192, 8193, 8200, 16384, 16392, 20001]


@pytest.fixture(scope="module")
def grawa():
    import paper_2403_04206_b200 as g
    return g


def make(M, rows, cols, kind, seed, pad=0, lead=0, shift=0.5, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0, shift=0.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale + shift).to(kind)

    x = normal(M, rows, cols + pad, scale=scale, shift=shift)
    dy = normal(M, rows, cols + pad)
    flat = torch.cat([normal(M, lead), normal(M, cols, scale=0.3, shift=1.0), normal(M, cols)], 1)
    return dict(x=[t[:, :cols] for t in x], dy=[t[:, :cols] for t in dy], gamma=[t[lead:lead + cols] for t in flat], beta=[t[lead + cols:] for t in flat])


def check_forward(grawa, d, kind, pad=0, affine=True, eps=EPS):
    M, (rows, cols) = len(d["x"]), d["x"][0].shape
    full = [torch.full((rows, cols + pad), 3.0, dtype=kind, device="cuda") for _ in range(M)]
    y = [t[:, :cols] for t in full]
    mean, rstd = ([torch.full((rows,), -1.0, device="cuda") for _ in range(M)] for _ in range(2))
    gamma, beta = (d["gamma"], d["beta"]) if affine else (None, None)
    grawa.grawa_layernorm_forward(d["x"], gamma, beta, y, eps, mean=mean, rstd=rstd)
    for m in range(M):
        want, mu, s, compute, dmean = layernorm64(d["x"][m], gamma and gamma[m], beta and beta[m], eps)
        check(y[m], want, kind, compute, f"y of worker {m}")
        check(mean[m], mu, torch.float32, dmean, "mean")
        # half of the relative error of the sum of squares and of the deviations, and the roundings of 1 / sqrt
        check(rstd[m], s, torch.float32, s * (80 * EPS32 + dmean * s), "rstd")
        assert (full[m][:, cols:] == 3.0).all()                                # what is behind a row stays
    return mean, rstd


def check_backward(grawa, d, mean, rstd, kind, pad=0, affine=True, accumulate=False, parts=("dx", "dgamma", "dbeta")):
    M, (rows, cols) = len(d["x"]), d["x"][0].shape
    full = [torch.full((rows, cols + pad), 3.0, dtype=kind, device="cuda") for _ in range(M)]
    dx = [t[:, :cols] for t in full]
    held = [[torch.randn(cols, device="cuda").to(kind) for _ in range(M)] for _ in range(2)]
    out = [[t.clone() for t in h] for h in held]
    gamma = d["gamma"] if affine else None
    grawa.grawa_layernorm_backward(d["dy"], d["x"], gamma, mean, rstd, dx if "dx" in parts else None, out[0] if "dgamma" in parts else None,
                                   out[1] if "dbeta" in parts else None, accumulate=accumulate)
    for m in range(M):
        (wx, ex), *weights = layernorm_backward64(d["dy"][m], d["x"][m], gamma and gamma[m], mean[m], rstd[m])
        if "dx" in parts:
            check(dx[m], wx, kind, ex, f"dx of worker {m}")
            assert (full[m][:, cols:] == 3.0).all()
        else:
            assert (full[m] == 3.0).all()
        for name, o, h, (w, e) in zip(("dgamma", "dbeta"), out, held, weights):
            if name not in parts:
                assert torch.equal(o[m], h[m])
            elif accumulate:
                check(o[m], w + h[m].double(), kind, e + EPS32 * (w.abs() + h[m].double().abs()), name)
            else:
                check(o[m], w, kind, e, name)
    return dx, out


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_row_lengths(grawa, kind, cols):
    d = make(2, 21, cols, kind, cols)
    mean, rstd = check_forward(grawa, d, kind)
    check_backward(grawa, d, mean, rstd, kind)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("rows", [1, 2, 4, 5, 16, 17, 64, 65, 197, 1001])
@pytest.mark.parametrize("cols", [48, 768, 2048])
def test_row_counts_and_accumulation(grawa, kind, rows, cols):
    d = make(3, rows, cols, kind, rows + cols)
    mean, rstd = check_forward(grawa, d, kind)
    check_backward(grawa, d, mean, rstd, kind, accumulate=True)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols,pad,lead", [(768, 8, 0), (768, 3, 11), (770, 2, 1), (1001, 6, 5), (4096, 1, 3), (9000, 8, 1), (20000, 5, 7)])
def test_padded_rows_and_parameters_at_odd_places(grawa, kind, cols, pad, lead):
    d = make(2, 37, cols, kind, cols + pad, pad, lead)
    mean, rstd = check_forward(grawa, d, kind, pad)
    check_backward(grawa, d, mean, rstd, kind, pad)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("cols,pad", [(100, 0), (256, 0), (250, 0), (251, 0), (512, 0), (1025, 1)])
def test_many_short_rows(grawa, kind, cols, pad):
    """Enough rows that every warp takes several, in every way of reading them."""
    d = make(2, 30011, cols, kind, cols, pad)
    mean, rstd = check_forward(grawa, d, kind, pad)
    check_backward(grawa, d, mean, rstd, kind, pad)


def test_most_workers(grawa):
    d = make(64, 9, 72, torch.bfloat16, 3)
    mean, rstd = check_forward(grawa, d, torch.bfloat16)
    check_backward(grawa, d, mean, rstd, torch.bfloat16)


@pytest.mark.parametrize("cols", [40, 768, 3000, 9000])
def test_without_parameters_and_partial_gradients(grawa, cols):
    kind = torch.bfloat16
    d = make(2, 90, cols, kind, cols)
    mean, rstd = check_forward(grawa, d, kind, affine=False)
    check_backward(grawa, d, mean, rstd, kind, affine=False, parts=("dx",))
    check_backward(grawa, d, mean, rstd, kind, parts=("dgamma", "dbeta"))
    check_backward(grawa, d, mean, rstd, kind, parts=("dx", "dbeta"))
    check_backward(grawa, d, mean, rstd, kind, parts=("dgamma",), accumulate=True)
    y, again = ([torch.empty(90, cols, dtype=kind, device="cuda") for _ in range(2)] for _ in range(2))
    grawa.grawa_layernorm_forward(d["x"], d["gamma"], d["beta"], y, EPS, mean=mean, rstd=rstd)
    grawa.grawa_layernorm_forward(d["x"], d["gamma"], d["beta"], again, EPS)     # statistics are optional
    assert all(torch.equal(a, b) for a, b in zip(y, again))


def test_rows_far_from_zero_and_constant_rows(grawa):
    d = make(1, 50, 768, torch.float32, 5, shift=300.0)
    mean, rstd = check_forward(grawa, d, torch.float32)
    check_backward(grawa, d, mean, rstd, torch.float32)
    x = [torch.full((9, 1000), 2.5, dtype=torch.float16, device="cuda")]
    y = [torch.empty_like(x[0])]
    beta = [torch.randn(1000, device="cuda").half()]
    grawa.grawa_layernorm_forward(x, None, beta, y, EPS)
    assert torch.equal(y[0], beta[0].expand(9, -1))                              # deviations are exactly zero


def test_a_bad_row_stays_its_own(grawa):
    d = make(1, 40, 768, torch.bfloat16, 6)
    clean = [torch.empty(40, 768, dtype=torch.bfloat16, device="cuda")]
    grawa.grawa_layernorm_forward(d["x"], d["gamma"], d["beta"], clean, EPS)
    d["x"][0][7, 100] = float("nan")
    d["x"][0][21, 5] = float("inf")
    y = [torch.empty_like(clean[0])]
    grawa.grawa_layernorm_forward(d["x"], d["gamma"], d["beta"], y, EPS)
    good = [r for r in range(40) if r not in (7, 21)]
    assert torch.equal(y[0][good], clean[0][good]) and torch.isnan(y[0][[7, 21]].float()).all()


def test_no_rows(grawa):
    kind = torch.float32
    empty = [torch.empty(0, 16, device="cuda")]
    stats = [torch.empty(0, device="cuda")]
    grawa.grawa_layernorm_forward(empty, None, None, empty, EPS)
    g, b = [torch.ones(16, device="cuda")], [torch.ones(16, device="cuda")]
    grawa.grawa_layernorm_backward(empty, empty, None, stats, stats, None, g, b, accumulate=True)
    assert (g[0] == 1).all() and (b[0] == 1).all()
    grawa.grawa_layernorm_backward(empty, empty, None, stats, stats, None, g, b)
    assert (g[0] == 0).all() and (b[0] == 0).all() and g[0].dtype == kind


def test_interleaved_workers_and_a_second_stream(grawa):
    """All workers' rows in one buffer [rows, M, cols]: rows of one worker lie between the rows of the others."""
    M, rows, cols, kind = 3, 29, 256, torch.bfloat16
    d = make(M, rows, cols, kind, 8)
    joint = torch.stack(d["x"], 1).contiguous()
    out = torch.zeros_like(joint)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    grawa.grawa_layernorm_forward([joint[:, m] for m in range(M)], d["gamma"], d["beta"], [out[:, m] for m in range(M)], EPS, stream=side)
    side.synchronize()
    y = [torch.empty(rows, cols, dtype=kind, device="cuda") for _ in range(M)]
    grawa.grawa_layernorm_forward(d["x"], d["gamma"], d["beta"], y, EPS)
    assert all(torch.equal(out[:, m], y[m]) for m in range(M))
    with pytest.raises(grawa.GrawaError):                                        # overlapping by one element
        flat = out.view(rows, -1)
        grawa.grawa_layernorm_forward(d["x"], None, None, [flat[:, 0:256], flat[:, 255:511], flat[:, 512:768]], EPS)


def test_replayed_graph_gives_the_same_bits(grawa):
    M, rows, cols, kind = 2, 300, 768, torch.float16
    d = make(M, rows, cols, kind, 9)
    y = [torch.empty(rows, cols, dtype=kind, device="cuda") for _ in range(M)]
    dx = [torch.empty_like(t) for t in y]
    mean, rstd = ([torch.empty(rows, device="cuda") for _ in range(M)] for _ in range(2))
    dg, db = ([torch.empty(cols, dtype=kind, device="cuda") for _ in range(M)] for _ in range(2))

    def both():
        grawa.grawa_layernorm_forward(d["x"], d["gamma"], d["beta"], y, EPS, mean=mean, rstd=rstd)
        grawa.grawa_layernorm_backward(d["dy"], d["x"], d["gamma"], mean, rstd, dx, dg, db)

    both()
    want = [t.clone() for t in y + dx + dg + db]
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        both()
    for _ in range(3):
        for t in y + dx + dg + db:
            t.fill_(9.0)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, y + dx + dg + db))


@pytest.mark.parametrize("cols", [24, 100])
def test_gradients_against_differences(grawa, cols):
    """Central differences of sum(y w) in fp32 with steps that make rounding and curvature small beside the tolerance."""
    d = make(1, 6, cols, torch.float32, 10, shift=0.0)
    x, w, gamma, beta = d["x"][0], d["dy"][0], d["gamma"][0], d["beta"][0]
    mean, rstd = check_forward(grawa, d, torch.float32)
    (dx, out) = check_backward(grawa, d, mean, rstd, torch.float32)

    def value(x, gamma, beta):
        y = [torch.empty_like(x)]
        grawa.grawa_layernorm_forward([x], [gamma], [beta], y, EPS)
        return (y[0].double() * w.double()).sum().item()

    # y is rounded to 2^-24 of values below 8 and the sum has 6 cols terms; with a step of 2^-6 that is
    # 6 cols * 8 * 2^-24 / 2^-6 in a difference, and the cubic term is below step^2 * |third derivative| ~ 2^-12 * 40
    step, tol = 2.0 ** -6, 6 * cols * 8 * 2.0 ** -24 * 2.0 ** 6 + 2.0 ** -12 * 40
    for which, grad in ((0, dx[0]), (1, out[0][0]), (2, out[1][0])):
        args = [x, gamma, beta]
        for j in range(0, args[which].numel(), 5):
            v = []
            for sign in (1, -1):
                moved = args[which].clone()
                moved.view(-1)[j] += sign * step
                v.append(value(*[moved if k == which else a for k, a in enumerate(args)]))
            assert abs((v[0] - v[1]) / (2 * step) - grad.reshape(-1)[j].item()) < tol


@pytest.mark.parametrize("apart", [2 ** 31 + 8, 2 ** 31 + 5])                      # whole words, and rows at odd places
def test_rows_further_apart_than_two_to_the_31_elements(grawa, apart):
    rows, cols, kind = 3, 771 - 3 * (apart % 8 == 0), torch.bfloat16

    def far(values=None):
        t = torch.empty((rows - 1) * apart + cols, dtype=kind, device="cuda").as_strided((rows, cols), (apart, 1))
        return t if values is None else t.copy_(values)

    d = make(1, rows, cols, kind, 9)
    x, dy, y = far(d["x"][0]), far(d["dy"][0]), far()
    mean, rstd = ([torch.empty(rows, device="cuda")] for _ in range(2))
    grawa.grawa_layernorm_forward([x], d["gamma"], d["beta"], [y], EPS, mean=mean, rstd=rstd)
    want, _, _, compute, _ = layernorm64(x, d["gamma"][0], d["beta"][0], EPS)
    check(y, want, kind, compute, "y")
    out = [[torch.empty(cols, dtype=kind, device="cuda")] for _ in range(2)]
    dx = y                                                                         # (its values are checked: the buffer serves again)
    grawa.grawa_layernorm_backward([dy], [x], d["gamma"], mean, rstd, [dx], *out)
    (wx, ex), *weights = layernorm_backward64(dy, x, d["gamma"][0], mean[0], rstd[0])
    check(dx, wx, kind, ex, "dx")
    for name, o, (w, e) in zip(("dgamma", "dbeta"), out, weights):
        check(o[0], w, kind, e, name)


def test_workers_that_share_their_inputs(grawa):
    d = make(1, 40, 130, torch.float16, 10)
    d = {k: v * 3 for k, v in d.items()}                                           # the same tensors for three workers
    mean, rstd = check_forward(grawa, d, torch.float16)
    check_backward(grawa, d, mean, rstd, torch.float16)
