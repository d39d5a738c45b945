"""Dropout over all workers: masks bit for bit against Philox4x32-10 in numpy, values against 64 bits."""
import pytest
import torch

from replica_util import EPS32, TYPES, check, dropout64, keep_mask

pytestmark = pytest.mark.gpu
SEED, OFFSET = 0x9E3779B97F4A7C15, (7 << 32) + 5


@pytest.fixture(scope="module")
def grawa():
    import paper_2403_04206_b200 as g
    return g


def values(M, n, kind, seed, lead=0):
    """M vectors of n elements, `lead` elements behind an aligned base."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(n + lead, generator=gen, device="cuda").to(kind)[lead:] for _ in range(M)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("lead", [0, 1])
@pytest.mark.parametrize("n", [1, 3, 4, 5, 7, 8, 9, 31, 255, 2048, 4097, 70003])
def test_forward_and_backward(grawa, kind, lead, n):
    M, p = 3, 0.3
    x, r, dy = values(M, n, kind, 1, lead), values(M, n, kind, 2, lead), values(M, n, kind, 3, lead)
    y, z, dx = ([torch.full_like(t, 7.0) for t in x] for _ in range(3))
    grawa.grawa_dropout_forward(x, y, p, SEED, OFFSET, residual=r)
    grawa.grawa_dropout_forward(x, z, p, SEED, OFFSET)
    grawa.grawa_dropout_backward(dy, dx, p, SEED, OFFSET)
    for m in range(M):
        keep = keep_mask(SEED, OFFSET, m, n, p).cuda()
        for got, v, res in ((y[m], x[m], r[m]), (z[m], x[m], None), (dx[m], dy[m], None)):
            want = dropout64(v, res, keep, p)
            # scale and product, or one fused multiply-add: two roundings of the scaled value, one of the sum
            check(got, want, kind, 2 * EPS32 * (v.double().abs() / 0.7) + EPS32 * want.abs(), f"worker {m}")
            dropped = got[~keep]
            assert torch.equal(dropped, torch.zeros_like(dropped) if res is None else res[~keep])


def test_share_of_kept_elements_and_workers_differ(grawa):
    n = 1 << 20
    x = [torch.ones(n, device="cuda") for _ in range(2)]
    y = [torch.empty(n, device="cuda") for _ in range(2)]
    grawa.grawa_dropout_forward(x, y, 0.25, 3, 0)
    kept = [(t != 0) for t in y]
    for k in kept:
        # binomial: 0.25 * 0.75 / n has a standard deviation of 4.3e-4; six of them
        assert abs(k.double().mean().item() - 0.75) < 6 * (0.25 * 0.75 / n) ** 0.5
    both = (kept[0] & kept[1]).double().mean().item()
    assert abs(both - 0.5625) < 6 * (0.5625 * 0.4375 / n) ** 0.5


@pytest.mark.parametrize("kind", TYPES)
def test_edges_of_p_and_values_in_dropped_places(grawa, kind):
    n = 1003
    x, r = values(1, n, kind, 4), values(1, n, kind, 5)
    y = [torch.empty_like(x[0])]
    grawa.grawa_dropout_forward(x, y, 0.0, 1, 2, residual=r)
    assert torch.equal(y[0], (x[0].float() + r[0].float()).to(kind))           # p = 0: one addition
    grawa.grawa_dropout_forward(x, y, 0.0, 1, 2)
    assert torch.equal(y[0], x[0])
    keep = keep_mask(9, 0, 0, n, 0.5).cuda()
    x[0][~keep] = float("nan")
    x[0][(~keep).nonzero()[::2]] = float("inf")
    grawa.grawa_dropout_forward(x, y, 0.5, 9, 0, residual=r)
    assert torch.isfinite(y[0].float()).all() and torch.equal(y[0][~keep], r[0][~keep])
    largest = 1.0 - 2.0 ** -24                                                  # the largest p of fp32
    grawa.grawa_dropout_backward(r, y, largest, 11, 0)
    keep = keep_mask(11, 0, 0, n, largest).cuda()
    assert torch.equal(y[0] != 0, keep & (r[0] != 0))


def test_in_place_and_many_workers(grawa):
    n, M = 517, 64
    x, r = values(M, n, torch.bfloat16, 6), values(M, n, torch.bfloat16, 7)
    y = [torch.empty_like(t) for t in x]
    grawa.grawa_dropout_forward(x, y, 0.4, SEED, 1, residual=r)
    xs, rs = [t.clone() for t in x], [t.clone() for t in r]
    grawa.grawa_dropout_forward(xs, xs, 0.4, SEED, 1, residual=r)
    grawa.grawa_dropout_forward(x, rs, 0.4, SEED, 1, residual=rs)
    for m in range(M):
        assert torch.equal(xs[m], y[m]) and torch.equal(rs[m], y[m])
    dy = [t.clone() for t in x]
    grawa.grawa_dropout_backward(dy, dy, 0.4, SEED, 1)
    for m in range(M):
        assert torch.equal(dy[m] != 0, keep_mask(SEED, 1, m, n, 0.4).cuda() & (x[m] != 0))


def test_captured_call_takes_a_new_mask_from_the_counter(grawa):
    n = 999
    x, y = values(2, n, torch.float32, 8), [torch.empty(n, device="cuda") for _ in range(2)]
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        grawa.grawa_dropout_forward(x, y, 0.5, SEED, 40, offset_counter=counter)
        counter += 1
    counter.fill_(2 ** 33)
    for step in range(3):
        g.replay()
        torch.cuda.synchronize()
        for m in range(2):
            keep = keep_mask(SEED, 40 + 2 ** 33 + step, m, n, 0.5).cuda()
            assert torch.equal(y[m], torch.where(keep, x[m] * 2, torch.zeros_like(x[m])))


def test_no_elements_and_two_streams_at_once(grawa):
    empty = [torch.empty(0, device="cuda")]
    grawa.grawa_dropout_forward(empty, empty, 0.5, 1, 2, residual=empty)
    streams = [torch.cuda.Stream() for _ in range(2)]
    n, p = 3_000_001, 0.2
    x = values(2, n, torch.bfloat16, 12)
    y = [torch.empty_like(t) for t in x]
    torch.cuda.synchronize()
    for k, s in enumerate(streams):
        grawa.grawa_dropout_forward([x[k]], [y[k]], p, SEED + k, OFFSET, stream=s)
    torch.cuda.synchronize()
    for k in range(2):
        keep = keep_mask(SEED + k, OFFSET, 0, n, p).cuda()
        assert torch.equal(y[k] != 0, keep & (x[k] != 0))


def test_elements_past_two_to_the_31(grawa):
    n, p = 2 ** 31 + 1029, 0.5
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    grawa.grawa_dropout_backward([x], [x], p, SEED, OFFSET)
    import numpy as np
    from replica_util import philox_words
    for first in (0, 2 ** 31 - 512, n - 1029 - 3):
        first -= first % 4
        count = min(1024, n - first)
        words = philox_words(SEED, OFFSET, 0, np.arange(first // 4, first // 4 + (count + 3) // 4)).reshape(-1)[:count]
        want = torch.from_numpy((words >= 2 ** 31).astype(np.float32) * 2)
        assert torch.equal(x[first:first + count].float().cpu(), want)


def test_binding_refuses_wrong_tensors(grawa):
    x, y = values(2, 64, torch.float32, 9), values(2, 64, torch.float32, 10)
    with pytest.raises(ValueError):
        grawa.grawa_dropout_forward(x, [t.cpu() for t in y], 0.1, 1)
    with pytest.raises(TypeError):
        grawa.grawa_dropout_forward(x, [t.half() for t in y], 0.1, 1)
    with pytest.raises(ValueError):
        grawa.grawa_dropout_forward(x, y[:1], 0.1, 1)
    with pytest.raises(ValueError):
        grawa.grawa_dropout_forward(x, [torch.empty(128, device="cuda")[::2]] * 2, 0.1, 1)
    with pytest.raises(grawa.GrawaError):
        grawa.grawa_dropout_forward(x, [y[0], y[0]], 0.1, 1)          # two workers into one buffer
