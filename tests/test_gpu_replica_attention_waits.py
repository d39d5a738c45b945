"""The bounded waits of the attention kernels: one that runs out ends its call with a status, and nothing else."""
import time

import pytest
import torch

pytestmark = pytest.mark.gpu


def forward(grawa, q, k, v):
    out = torch.empty_like(q)
    grawa.grawa_window_attention_forward([q], [k], [v], [out], left=40)
    return out


def test_a_wait_that_runs_out_is_reported_and_the_calls_around_it_are_right():
    import paper_2403_04206_b200 as grawa
    gen = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(300, 2, 64, generator=gen, device="cuda").bfloat16() for _ in range(3))
    want = forward(grawa, q, k, v)
    assert grawa.grawa_window_attention_status() == 0
    ffn = grawa.grawa_gated_ffn_status()
    for _ in range(2):
        start = time.perf_counter()
        first = forward(grawa, q, k, v)
        grawa.grawa_selftest_window_attention_wait()
        second = forward(grawa, q, k, v)
        assert grawa.grawa_window_attention_status() == -5 and time.perf_counter() - start < 1.0
        assert grawa.grawa_window_attention_status() == 0    # reported once
        assert torch.equal(first, want) and torch.equal(second, want)
    assert ffn == 0 and grawa.grawa_gated_ffn_status() == 0  # the other operator's waits are counted apart
