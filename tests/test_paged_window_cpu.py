"""Attention behind a window without a GPU: NULL arguments of the C ABI, and the binding's checks on host tensors."""
import pytest

from paper_2403_00835_amd import binding
from tests.test_paged_binding_cpu import arrays, cache  # noqa: F401

torch = pytest.importorskip("torch")


@pytest.fixture
def counted(cache):  # noqa: F811
    cache.L.cllm_paged_attn_window = lambda *a: cache.calls.append(("window", a)) or 0
    return cache


def test_null_arguments_are_refused():
    assert binding.lib().cllm_paged_attn_window(None, None, 0, None, None, 0.0, 4, 0, None, 0, None) == 1


def test_a_window_chooses_the_entry(counted):
    a = arrays()
    for kw, want in ((dict(), None), (dict(window=1), (1, 0)), (dict(window=2**31 - 1, sinks=7), (2**31 - 1, 7))):
        before = a["out"]._version, a["lse"]._version
        counted.attn(a["q"], a["kp"], a["vp"], a["out"], lse=a["lse"], **kw)
        name, args = counted.calls[-1]
        assert name == ("attn" if want is None else "window")
        assert want is None or args[6:8] == want
        assert args[-1] == a["lse"].data_ptr() and args[-3] == a["out"].data_ptr()
        assert a["out"]._version > before[0] and a["lse"]._version > before[1]


@pytest.mark.parametrize("kw", [dict(window=0), dict(window=-5), dict(window=2**31), dict(window=3, sinks=-1),
                                dict(window=3, sinks=2**31), dict(sinks=2)])
def test_bad_windows_are_refused(counted, kw):
    a = arrays()
    with pytest.raises(ValueError, match="sinks"):
        counted.attn(a["q"], a["kp"], a["vp"], a["out"], **kw)
    assert counted.calls == []


@pytest.mark.parametrize("which", ["q", "out", "kp", "vp", "lse"])
def test_tensors_that_require_grad_are_refused(counted, which):
    a = arrays()
    a[which].requires_grad_()
    with pytest.raises(ValueError, match="grad"):
        counted.attn(a["q"], a["kp"], a["vp"], a["out"], lse=a["lse"], window=4)
    assert counted.calls == []
    with torch.no_grad():
        counted.attn(a["q"], a["kp"], a["vp"], a["out"], lse=a["lse"], window=4)
    assert [x[0] for x in counted.calls] == ["window"]
