"""Host-side checks of the paged KV cache's C ABI (no GPU): shapes and NULL arguments are refused
before the device is touched, and the workspace size follows the shape."""
import ctypes

import pytest

from paper_2403_00835_amd import binding

OK = dict(n_heads=32, n_kv_heads=8, head_dim=128, dtype=1, page_size=64, n_pages=100, max_seqs=16, max_ctx=2048,
          max_rows=512, rope_base=10000.0, device=0, stream=None, workspace=None, workspace_bytes=0)


def config(**kw):
    return binding.cllm_paged_config(*[{**OK, **kw}[k] for k, _ in binding.cllm_paged_config._fields_])


def workspace(**kw):
    n = ctypes.c_size_t(7)
    st = binding.lib().cllm_paged_workspace_bytes(ctypes.byref(config(**kw)), ctypes.byref(n))
    return st, n.value


BAD = [dict(n_heads=31), dict(n_heads=0), dict(n_kv_heads=0), dict(n_kv_heads=64), dict(n_heads=2048, n_kv_heads=2048),
       dict(head_dim=48), dict(head_dim=16), dict(dtype=0, head_dim=256), dict(dtype=2), dict(page_size=8),
       dict(page_size=48), dict(page_size=512), dict(n_pages=0), dict(n_pages=1 << 26), dict(max_seqs=0),
       dict(max_seqs=1025), dict(max_ctx=0), dict(max_ctx=(1 << 20) + 1), dict(max_rows=0), dict(max_rows=(1 << 20) + 1),
       dict(rope_base=-1.0), dict(rope_base=float("inf")), dict(rope_base=float("nan"))]


@pytest.mark.parametrize("kw", BAD, ids=[str(k) for k in BAD])
def test_bad_shapes_are_refused(kw):
    assert workspace(**kw) == (1, 0)
    h = ctypes.c_void_p()
    assert binding.lib().cllm_paged_create(ctypes.byref(config(**kw)), ctypes.byref(h)) == 1
    assert not h.value


def test_a_workspace_size_without_a_workspace_is_refused():
    h = ctypes.c_void_p()
    assert binding.lib().cllm_paged_create(ctypes.byref(config(workspace_bytes=1 << 20)), ctypes.byref(h)) == 1


def test_workspace_bytes_follow_the_shape():
    st, base = workspace()
    assert st == 0 and base % 256 == 0
    # at least the books: block table, free list, row arrays
    assert base > 4 * (16 * 32 + 100 + 2 * 512)
    assert workspace(rope_base=0.0)[1] < base  # no rotary factors
    assert workspace(n_pages=100000)[1] > base
    for ok in (dict(dtype=0, head_dim=16), dict(head_dim=256), dict(page_size=16), dict(page_size=256),
               dict(n_heads=7, n_kv_heads=1), dict(max_seqs=1024), dict(max_ctx=1, max_rows=1, max_seqs=1, n_pages=1)):
        assert workspace(**ok)[0] == 0, ok


def test_null_arguments_are_refused():
    L = binding.lib()
    n = ctypes.c_size_t()
    assert L.cllm_paged_workspace_bytes(None, ctypes.byref(n)) == 1
    assert L.cllm_paged_workspace_bytes(ctypes.byref(config()), None) == 1
    assert L.cllm_paged_create(None, None) == 1
    assert L.cllm_paged_plan(None, 1, None, None, None, 0, 0, 0) == 1
    assert L.cllm_paged_append(None, None, 0, None, 0, None, 0, None, 0, None, None) == 1
    assert L.cllm_paged_attn(None, None, 0, None, None, 0.0, None, 0, None) == 1
    assert L.cllm_paged_status(None, None, None) == 1
    assert L.cllm_paged_views_get(None, None) == 1
    assert L.cllm_paged_last_error(None) == b"null cache"
    L.cllm_paged_free(None)
