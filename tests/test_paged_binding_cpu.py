"""The checks of binding.PagedCache itself, on host tensors: a cache whose library only counts its calls."""
import types

import pytest

from paper_2403_00835_amd import binding

torch = pytest.importorskip("torch")


@pytest.fixture
def cache():
    c = object.__new__(binding.PagedCache)
    calls = []

    def entry(name):
        return lambda *a: calls.append((name, a)) or 0

    c.L = types.SimpleNamespace(cllm_paged_append=entry("append"), cllm_paged_attn=entry("attn"), cllm_paged_plan=entry("plan"))
    c.h, c.stream, c._current, c.device = 1, 0, lambda: 0, torch.device("cpu")
    c.n_heads, c.n_kv_heads, c.head_dim, c.dtype, c.rows = 4, 2, 32, torch.float32, 3
    c._int32, c._float32 = torch.int32, torch.float32
    c.pool_shape = (5, 2, 16, 32)
    c._ws = torch.zeros(64, dtype=torch.uint8)
    c.calls = calls
    yield c
    c.h = None


def arrays():
    q, k, v, out = (torch.zeros(3, h, 32) for h in (4, 2, 2, 4))
    return dict(q=q, k=k, v=v, out=out, kp=torch.zeros(5, 2, 16, 32), vp=torch.zeros(5, 2, 16, 32), lse=torch.zeros(3, 4))


def call(c, name, a):
    if name == "append":
        c.append(a["q"], a["k"], a["v"], a["out"], a["kp"], a["vp"])
    elif name == "attn":
        c.attn(a["q"], a["kp"], a["vp"], a["out"], lse=a["lse"])
    else:
        n = torch.ones(2, dtype=torch.int32)
        c.plan(n, n, n, rows=3)


@pytest.mark.parametrize("name,which", [("append", x) for x in ("q", "k", "v", "out", "kp", "vp")] +
                         [("attn", x) for x in ("q", "out", "kp", "vp", "lse")])
def test_tensors_that_require_grad_are_refused(cache, name, which):
    a = arrays()
    a[which].requires_grad_()
    with pytest.raises(ValueError, match="grad"):
        call(cache, name, a)
    assert cache.calls == []
    with torch.no_grad():  # as torch's own operators with an output argument have it
        call(cache, name, a)
    with torch.inference_mode():
        call(cache, name, arrays())
    assert [x[0] for x in cache.calls] == [name, name]


@pytest.mark.parametrize("name,written", [("append", ("out", "kp", "vp")), ("attn", ("out", "lse"))])
def test_written_tensors_count_as_changed(cache, name, written):
    """What autograd saved before a call that overwrites it is refused in the backward pass, as after an in-place
    operator of torch's own."""
    a = arrays()
    w = torch.ones(4, 32, requires_grad=True)
    y = (a["out"] * w).sum()  # keeps out for w's gradient
    before = {k: x._version for k, x in a.items()}
    call(cache, name, a)
    assert {k for k, x in a.items() if x._version != before[k]} == set(written)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    rows = torch.zeros(6, 4, 32)  # a view's base too
    a["out"] = rows[1:4]
    before = rows._version
    call(cache, name, a)
    assert rows._version > before
    call(cache, name, dict(a, lse=None) if name == "attn" else a)


def test_the_books_count_as_changed_by_a_plan(cache):
    view = cache._ws[:8].view(torch.int32)
    before = view._version
    call(cache, "plan", None)
    assert view._version > before


@pytest.mark.parametrize("scale", [0, 0.0, -0.0, 1e-46, -1e-50])
def test_a_scale_of_0_in_fp32_is_refused(cache, scale):
    """The library takes 0 for the default scale: what rounds to it must not."""
    a = arrays()
    with pytest.raises(ValueError, match="scale"):
        cache.attn(a["q"], a["kp"], a["vp"], a["out"], scale=scale)
    assert cache.calls == []
    for good in (None, 1e-45, -0.5, 1.0, 3e38):
        cache.attn(a["q"], a["kp"], a["vp"], a["out"], scale=good)
    assert [x[1][5] for x in cache.calls] == [0.0, 1e-45, -0.5, 1.0, 3e38]
