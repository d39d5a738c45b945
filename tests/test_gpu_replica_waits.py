"""The bounded waits of the gated feed-forward product: one that runs out ends its call with a status, and nothing else."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def grawa():
    import paper_2403_04206_b200 as g
    return g


def forward(grawa, x, w_gate, w_up):
    h = torch.empty(x.shape[0], w_gate.shape[0], dtype=x.dtype, device="cuda")
    grawa.grawa_gated_ffn_forward([x], [w_gate], [w_up], [h], activation="relu")
    return h


def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_right(grawa):
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, w_gate, w_up = (torch.randint(-3, 4, shape, generator=gen, device="cuda").bfloat16() for shape in ((300, 64), (200, 64), (200, 64)))
    want = torch.clamp(x.double() @ w_gate.double().T, min=0) * (x.double() @ w_up.double().T)
    assert torch.equal(forward(grawa, x, w_gate, w_up), want.bfloat16())
    assert grawa.grawa_gated_ffn_status() == 0
    for _ in range(2):
        start = time.perf_counter()
        grawa.grawa_selftest_gated_ffn_wait()
        assert grawa.grawa_gated_ffn_status() == -5 and time.perf_counter() - start < 1.0
        assert grawa.grawa_gated_ffn_status() == 0            # reported once
        assert torch.equal(forward(grawa, x, w_gate, w_up), want.bfloat16())
    assert grawa.grawa_gated_ffn_status() == 0


def test_on_a_stream_between_calls(grawa):
    """Calls in front of it and behind it on the stream, whose launches overlap its own, are not touched by it."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, w_gate, w_up = (torch.randint(-3, 4, shape, generator=gen, device="cuda").bfloat16() for shape in ((700, 128), (512, 128), (512, 128)))
    want = forward(grawa, x, w_gate, w_up)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        first = forward(grawa, x, w_gate, w_up)
        grawa.grawa_selftest_gated_ffn_wait()
        second = forward(grawa, x, w_gate, w_up)
        assert grawa.grawa_gated_ffn_status() == -5
    assert torch.equal(first, want) and torch.equal(second, want)
    grawa.grawa_gated_ffn_status()                            # (tells this stream of it)


def test_every_stream_is_told_once(grawa):
    """One caller's report does not take away another's."""
    streams = [torch.cuda.Stream() for _ in range(3)] + [torch.cuda.current_stream()]
    for s in streams:
        grawa.grawa_gated_ffn_status(s)
    for _ in range(2):
        grawa.grawa_selftest_gated_ffn_wait(stream=streams[0])
        torch.cuda.synchronize()
        assert [grawa.grawa_gated_ffn_status(s) for s in streams] == [-5] * 4
        assert [grawa.grawa_gated_ffn_status(s) for s in streams] == [0] * 4
