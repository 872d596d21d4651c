"""Sizes at which the paged cache's calls end, without a GPU."""
import ctypes

import pytest

from paper_2403_00835_amd import binding
from tests.test_paged_binding_cpu import cache  # noqa: F401

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("vocab", [1, 2048, 2049, 2**30])
@pytest.mark.parametrize("draft", [0, 1])
def test_rows_that_are_counted_in_31_bits(vocab, draft):
    """Statistics are formed by launches of 2^15 rows, the target's and the draft's: their count may pass the last row by a launch."""
    n, most = ctypes.c_size_t(7), (2**30 - 2**14 - 1) // -(-vocab // 2048)
    assert binding.lib().cllm_paged_verify_bytes(most, vocab, draft, ctypes.byref(n)) == 0 and n.value >= 16 * most
    assert binding.lib().cllm_paged_verify_bytes(most + 1, vocab, draft, ctypes.byref(n)) == 3 and n.value == 0


@pytest.fixture
def counted(cache):  # noqa: F811
    cache.L.cllm_paged_verify = cache.L.cllm_paged_rotary = lambda *a: cache.calls.append(a) or 0
    cache._float64, cache._logits = torch.float64, {torch.bfloat16: 1, torch.float32: 0}
    return cache


def test_sizes_past_32_bits_are_refused(counted):
    """ctypes takes the low 32 bits of an integer: 2^32 + 3 rows would be three."""
    size = binding.PagedCache.verify_workspace_bytes
    for bad in ((2**32 + 3, 5), (3, 2**32 + 5), (2**31, 1), (3, -2**32 + 5)):
        with pytest.raises(ValueError, match="32 bits"):
            size(*bad, False)

    def verify(rows, n):
        one, many = torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.float64)
        counted.verify(one.expand(rows), torch.zeros(1, 5).expand(rows, 5), one.expand(n), one.expand(n), torch.ones(1).expand(n),
                       many.expand(rows), many.expand(n))

    for rows, n in ((2**32 + 1, 1), (1, 2**32 + 1)):
        with pytest.raises(ValueError, match="32 bits"):
            verify(rows, n)
    assert counted.calls == []
    verify(1, 1)
    for dim in (2**32 + 8, -2**32 + 8):
        with pytest.raises(ValueError, match="32 bits"):
            counted.rotary(dim=dim)
    assert len(counted.calls) == 1
