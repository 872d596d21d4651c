"""Verification of drafted tokens without a GPU: the reference against the rule's own law, sizes and NULL arguments of the C ABI,
and the binding's checks on host tensors."""
import ctypes

import numpy as np
import pytest

from paper_2403_00835_amd import binding
from tests import verify_ref as ref
from tests.test_paged_binding_cpu import cache  # noqa: F401

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("with_q", [True, False])
def test_the_rule_has_the_targets_law(with_q):
    """Over all numbers, the first token has the distribution p: what stands, q(x) min(1, p(x) / q(x)) (a point mass: p(x) of the
    one draft), and what is refused and drawn from the rest."""
    rng = np.random.default_rng(0)
    for _ in range(50):
        n = int(rng.integers(2, 9))
        p, q = (ref.law(rng.standard_normal(n) * 2, 1.0) for _ in range(2))
        out = np.zeros(n)
        for x in range(n):
            weight = q[x] if with_q else float(x == 3 % n)
            stands = min(1.0, p[x] / q[x]) if with_q else p[x]
            out[x] += weight * stands
            rest = ref.left(p, q if with_q else None, x)
            out += weight * (1 - stands) * rest / rest.sum()
        np.testing.assert_allclose(out, p, atol=1e-14)


def test_draws_cut_the_unit_interval():
    p = np.array([0, 0.25, 0, 0.5, 0.25, 0])
    for u, want in ((0, 1), (0.2499, 1), (0.25, 3), (0.7499, 3), (0.75, 4), (0.9999, 4), (1.0, 4), (2.0, 4), (-1.0, 1), (float("nan"), 1)):
        assert ref.draw(p, u) == want


@pytest.mark.parametrize("rows,vocab,draft", [(0, 5, 0), (1, 1, 0), (7, 4096, 1), (7, 4097, 0), (300, 131072, 1)])
def test_workspace_bytes(rows, vocab, draft):
    size = binding.PagedCache.verify_workspace_bytes
    n = size(rows, vocab, draft)
    assert n % 256 == 0 and n >= (16 * rows if vocab > 0 else 0) and size(rows, vocab, 0) <= size(rows, vocab, 1)
    assert size(rows + 300, vocab, draft) > n and size(rows + 1, 100 * vocab, draft) >= n  # it follows rows and vocabulary
    assert n <= 64 * rows * (2 + vocab // 1024) + 256  # and is a small part of the logits


def test_bad_sizes_are_refused():
    n = ctypes.c_size_t(7)
    L = binding.lib()
    assert L.cllm_paged_verify_bytes(1, 1, 0, None) == 1
    for rows, vocab, want in ((-1, 5, 1), (1, 0, 1), (1, -3, 1), (2**20, 2**30, 3), (1, 2**30 + 1, 3), (1, 2**31 - 1, 3), (2**31 - 1, 1, 3)):
        assert L.cllm_paged_verify_bytes(rows, vocab, 1, ctypes.byref(n)) == want and n.value == 0
    with pytest.raises(binding.CllmError, match="ERR_CAPACITY"):
        binding.PagedCache.verify_workspace_bytes(2**31 - 1, 4097, True)
    assert L.cllm_paged_verify(None, 1, None, 1, None, 1, 5, None, 5, None, 0, None, None, None, None, None, None, 0) == 1


@pytest.fixture
def counted(cache):  # noqa: F811
    cache.L.cllm_paged_verify = lambda *a: cache.calls.append(("verify", a)) or 0
    cache._logits, cache._float64 = {torch.bfloat16: 1, torch.float32: 0}, torch.float64
    return cache


def arrays():
    return dict(tokens=torch.zeros(6, dtype=torch.int32), logits=torch.zeros(6, 50), accepted=torch.zeros(2, dtype=torch.int32),
                next_token=torch.zeros(2, dtype=torch.int32), temperature=torch.ones(2), accept_u=torch.zeros(6, dtype=torch.float64),
                sample_u=torch.zeros(2, dtype=torch.float64), row_start=torch.tensor([0, 2, 6], dtype=torch.int32))


def test_what_the_entry_is_given(counted):
    a = arrays()
    before = {k: x._version for k, x in a.items()}
    counted.verify(**a)
    args = counted.calls[-1][1]
    assert args[1] == 2 and args[3] == 6 and args[5:7] == (0, 50) and args[8:11] == (50, None, 0) and args[-1] % 256 == 0
    assert {k for k, x in a.items() if x._version != before[k]} == {"accepted", "next_token"}
    wide, draft = torch.zeros(6, 64).bfloat16()[:, 3:53], torch.zeros(6, 50).bfloat16()
    ws = torch.zeros(4096, dtype=torch.uint8)
    counted.verify(**{**a, "logits": wide, "row_start": None}, draft_logits=draft, workspace=ws)
    args = counted.calls[-1][1]
    assert args[2] is None and args[5:7] == (1, 50) and args[7:11] == (wide.data_ptr(), 64, draft.data_ptr(), 50)
    assert args[-2:] == (ws.data_ptr(), 4096) and ws._version > 0


BAD = [("tokens", lambda x: x.long()), ("tokens", lambda x: x[:5]), ("logits", lambda x: x.half()), ("logits", lambda x: x[:, ::2]),
       ("logits", lambda x: x[0]), ("logits", lambda x: x.requires_grad_()), ("accepted", lambda x: x.long()),
       ("next_token", lambda x: x[:1]), ("temperature", lambda x: x.double()), ("temperature", lambda x: x[:1]),
       ("accept_u", lambda x: x.float()), ("accept_u", lambda x: x[:5]), ("sample_u", lambda x: x.float()), ("sample_u", lambda x: x[:1]),
       ("row_start", lambda x: x[:2]), ("row_start", lambda x: x.long()), ("draft_logits", lambda x: torch.zeros(6, 49)),
       ("draft_logits", lambda x: torch.zeros(6, 50).bfloat16()), ("workspace", lambda x: torch.zeros(4096)),
       ("logits", lambda x: x.to("meta")), ("tokens", lambda x: x.to("meta"))]


@pytest.mark.parametrize("which,change", BAD, ids=range(len(BAD)))
def test_bad_arrays_are_refused(counted, which, change):
    a = arrays()
    a[which] = change(a.get(which))
    with pytest.raises(ValueError):
        counted.verify(**a)
    assert counted.calls == []
