"""Sizes of the attention operators' scratch for sizes that a call refuses (no GPU)."""
import pytest

import paper_2403_04206_b200 as grawa


@pytest.mark.parametrize("sizes", [(10, 4, 3, 64, 0, 2), (10, 4, 8, 64, 0, 2), (10, 4, 2, 63, 0, 2), (10, 4, 2, 12, 0, 2), (10, 4, 2, 136, 0, 2), ((1 << 31) - 1, 4, 2, 64, 0, 2),
                                   (10, 1 << 15, 1, 64, 0, 2), (1 << 30, 1 << 14, 1, 64, 0, 1), (10, 1 << 62, 1, 8, 0, 1), (10, 4, 1 << 62, 8, 0, 1), (10, 4, 0, 8, 0, 1)], ids=str)
def test_no_scratch_for_what_is_refused(sizes):
    assert grawa.grawa_window_attention_backward_workspace_bytes(*sizes) == 0


def test_scratch_of_what_is_taken():
    for sizes in ((0, 4, 2, 64, 0, 2), (10, 4, 2, 64, 5, 2), (3000, 6, 3, 128, 4, 64)):
        assert grawa.grawa_window_attention_backward_workspace_bytes(*sizes) > 0
