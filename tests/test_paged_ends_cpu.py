"""Sizes at which the paged cache's calls end, without a GPU."""
import ctypes

import pytest

from paper_2403_00835_amd import binding


@pytest.mark.parametrize("vocab", [1, 2048, 2049, 2**30])
@pytest.mark.parametrize("draft", [0, 1])
def test_rows_that_are_counted_in_31_bits(vocab, draft):
    """Statistics are formed by launches of 2^15 rows, the target's and the draft's: their count may pass the last row by a launch."""
    n, most = ctypes.c_size_t(7), (2**30 - 2**14 - 1) // -(-vocab // 2048)
    assert binding.lib().cllm_paged_verify_bytes(most, vocab, draft, ctypes.byref(n)) == 0 and n.value >= 16 * most
    assert binding.lib().cllm_paged_verify_bytes(most + 1, vocab, draft, ctypes.byref(n)) == 3 and n.value == 0
