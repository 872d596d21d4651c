"""Rotary forms and head norms of the paged KV cache without a GPU: the angles of a spec against their formulas, refusals of
the C ABI, and the binding's checks on host tensors."""
import ctypes
import math

import numpy as np
import pytest

from paper_2403_00835_amd import binding
from tests.test_paged_binding_cpu import arrays, cache  # noqa: F401

torch = pytest.importorskip("torch")

OK = dict(layout=0, dim=0, scaling=0, base=10000.0, factor=4.0, orig_ctx=2048.0, low=1.0, high=4.0, magnitude=0.0, freqs=None)


def freqs(head_dim=64, **kw):
    kw = {**OK, **kw}
    if kw["freqs"] is not None:
        kw["freqs"] = (ctypes.c_double * len(kw["freqs"]))(*kw["freqs"])
    spec = binding.cllm_paged_rotary_spec(*[kw[k] for k, _ in binding.cllm_paged_rotary_spec._fields_])
    out = np.full(128, -7.0)
    st = binding.lib().cllm_paged_rotary_freqs(ctypes.byref(spec), head_dim, out.ctypes.data)
    return st, out


@pytest.mark.parametrize("head_dim,dim", [(64, 0), (64, 24), (16, 2), (256, 0), (128, 64)])
def test_angles_follow_the_formulas(head_dim, dim):
    n = (dim or head_dim) // 2
    theta = [10000.0 ** (-j / n) for j in range(n)]
    st, out = freqs(head_dim, dim=dim)
    assert st == 0 and (out[n:] == -7).all()
    np.testing.assert_allclose(out[:n], theta, rtol=1e-14)
    np.testing.assert_allclose(freqs(head_dim, dim=dim, scaling=1)[1][:n], np.divide(theta, 4), rtol=1e-14)
    by_parts = freqs(head_dim, dim=dim, scaling=2)[1][:n]
    for w, x in zip(theta, by_parts):
        turns = 2048 * w / (2 * math.pi)
        if turns >= 4:
            assert x == w or abs(x / w - 1) < 1e-14
        elif turns <= 1:
            assert abs(4 * x / w - 1) < 1e-14
        else:
            g = (turns - 1) / 3
            assert abs(x - (g * w + (1 - g) * w / 4)) < 1e-14 * w
    own = [0.25 * (j + 1) for j in range(n)]
    np.testing.assert_array_equal(freqs(head_dim, dim=dim, freqs=own, scaling=7, base=-1.0)[1][:n], own)


def test_scaled_angles_reach_every_part():
    """The spec above has pairs that keep their angle, pairs between, and stretched ones."""
    theta = 10000.0 ** (-np.arange(32) / 32)
    share = freqs(scaling=2)[1][:32] / theta
    assert (share > 0.999999).any() and (share < 0.250001).any() and ((share > 0.3) & (share < 0.95)).any()


BAD = [dict(dim=-2), dict(dim=3), dict(dim=66), dict(layout=2), dict(layout=-1), dict(scaling=3), dict(scaling=-1), dict(base=0.0),
       dict(base=-1.0), dict(base=float("inf")), dict(base=float("nan")), dict(scaling=1, factor=0.0), dict(scaling=1, factor=float("nan")),
       dict(scaling=2, factor=-1.0), dict(scaling=2, orig_ctx=0.0), dict(scaling=2, low=4.0), dict(scaling=2, low=float("nan")),
       dict(scaling=2, high=float("inf")), dict(magnitude=float("nan")), dict(magnitude=float("inf")),
       dict(freqs=[0.5] * 31 + [float("nan")]), dict(freqs=[float("inf")] * 32), dict(freqs=[1e301] * 32)]


@pytest.mark.parametrize("kw", BAD, ids=range(len(BAD)))
def test_bad_specs_are_refused(kw):
    st, out = freqs(**kw)
    assert st == 1 and (out == -7).all()


@pytest.mark.parametrize("head_dim", [0, -2, 63, 258])
def test_bad_heads_are_refused(head_dim):
    assert freqs(head_dim)[0] == 1


def test_null_arguments_are_refused():
    L, spec, out = binding.lib(), binding.cllm_paged_rotary_spec(), np.zeros(4)
    assert L.cllm_paged_rotary_freqs(None, 64, out.ctypes.data) == 1
    assert L.cllm_paged_rotary_freqs(ctypes.byref(spec), 64, None) == 1
    assert L.cllm_paged_rotary(None, ctypes.byref(spec)) == 1
    assert L.cllm_paged_append_norm(None, None, 0, None, 0, None, 0, None, 0, None, None, None, None, 0.0) == 1


def counted(c):
    def entry(name):
        return lambda *a: c.calls.append((name, a)) or 0
    c.L.cllm_paged_append_norm, c.L.cllm_paged_rotary = entry("append_norm"), entry("rotary")
    return c


def test_gains_choose_the_entry(cache):  # noqa: F811
    c, a, g = counted(cache), arrays(), torch.ones(32)
    args = a["q"], a["k"], a["v"], a["out"], a["kp"], a["vp"]
    c.append(*args)
    c.append(*args, q_gain=g)
    c.append(*args, k_gain=g, eps=1e-5)
    c.append(None, a["k"], a["v"], None, a["kp"], a["vp"], k_gain=g)
    assert [x[0] for x in c.calls] == ["append"] + 3 * ["append_norm"]
    assert [x[1][-3:] for x in c.calls[1:]] == [(g.data_ptr(), None, 1e-6), (None, g.data_ptr(), 1e-5), (None, g.data_ptr(), 1e-6)]
    before = {k: a[k]._version for k in ("out", "kp", "vp")}
    c.append(*args, q_gain=g)
    assert all(a[k]._version > v for k, v in before.items())


@pytest.mark.parametrize("gain", [torch.ones(31), torch.ones(32).double(), torch.ones(64)[::2], torch.ones(1, 32),
                                  torch.ones(32, device="meta"), torch.ones(32).requires_grad_()])
def test_bad_gains_are_refused(cache, gain):  # noqa: F811
    c, a = counted(cache), arrays()
    for kw in (dict(q_gain=gain), dict(k_gain=gain)):
        with pytest.raises(ValueError, match="gain"):
            c.append(a["q"], a["k"], a["v"], a["out"], a["kp"], a["vp"], **kw)
    assert c.calls == []


def test_rotary_arguments(cache):  # noqa: F811
    c = counted(cache)
    for bad in (dict(layout="whole"), dict(scaling="ntk"), dict(magnitude=0.0), dict(magnitude=1e-50), dict(freqs=[1.0] * 15),
                dict(freqs=[1.0] * 16, scaling="linear", factor=2.0), dict(freqs=[1.0], dim=4)):
        with pytest.raises(ValueError):
            c.rotary(**bad)
    assert c.calls == []
    before = c._ws._version
    c.rotary()
    c.rotary(layout="interleaved", dim=8, scaling="parts", factor=2.0, orig_ctx=64, low=1.0, high=2.0, magnitude=1.1)
    c.rotary(dim=4, freqs=[1.0, 0.5])
    specs = [x[1][1]._obj for x in c.calls]
    assert [(s.layout, s.dim, s.scaling) for s in specs] == [(0, 0, 0), (1, 8, 2), (0, 4, 0)]
    assert [bool(s.freqs) for s in specs] == [False, False, True] and specs[2].freqs[1] == 0.5
    assert c._ws._version > before  # the factors are in the workspace
