"""GPU tests of append with head norms and rotary forms (binding.PagedCache.rotary, append with gains) against plain references
in float64. Tolerances are half steps of the output's type plus bounds of the fp32 arithmetic, derived at their
definitions."""
import math

import numpy as np
import pytest

from tests import paged_ref as ref
from tests.test_gpu_paged import half_step, host, ints, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def binding():
    from paper_2403_00835_amd import binding as b
    return b


def angles(dim, base=10000.0, scaling=None, factor=1.0, orig_ctx=0.0, low=0.0, high=0.0):
    w = base ** (-2.0 * np.arange(dim // 2) / dim)
    if scaling is None:
        return w
    keep = 0 if scaling == "linear" else np.clip((w * orig_ctx / (2 * math.pi) - low) / (high - low), 0, 1)
    return keep * w + (1 - keep) * w / factor


def norm(x, gain, eps):
    return x if gain is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def turn(x, pos, theta, layout, magnitude=1.0):
    """Rows x [R, heads, hd] turned, and |a| + |b| of each element's pair: what rounding errors scale with."""
    n, out, size = len(theta), x.copy(), np.abs(x)
    c, s = (magnitude * f(np.outer(pos, theta))[:, None] for f in (np.cos, np.sin))
    i = np.arange(n)
    a, b = (2 * i, 2 * i + 1) if layout == "interleaved" else (i, i + n)
    out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * max(1.0, abs(magnitude))
    return out, size


def check(got, raw, gain, eps, pos, theta, layout, dtype, magnitude=1.0):
    hd = raw.shape[-1]
    want, size = turn(norm(raw, gain, eps), pos, theta, layout, magnitude)
    # the sum of hd squares, its quotient and root, two products: at most hd + 16 half steps of fp32 of the normalised
    # value (half of them through the root); a factor rounded once, two products and a sum: 4 of |a| + |b|; then the output's half step
    fp32 = ((hd + 16 if gain is not None else 0) + 4) * 2.0**-24 * size
    tol = half_step(dtype) * (np.abs(want) + fp32) + fp32
    d = np.abs(got - want)
    assert (d <= tol).all(), f"off by {np.nanmax(d / tol)} of its bound, {np.isnan(d).sum()} NaN"


FORMS = [  # dtype, heads, kv heads, head dim, page, contexts, new tokens, rotary, norms of (q, k)
    ("bf16", 4, 4, 128, 64, [0, 63, 100], [1, 2, 70], dict(layout="half"), (True, True)),
    ("bf16", 32, 8, 128, 16, [5000], [33], dict(layout="half", scaling="parts", factor=8.0, orig_ctx=2048.0, low=1.0, high=32.0), (True, True)),
    ("bf16", 14, 2, 64, 16, [5], [33], dict(layout="interleaved"), (True, True)),
    ("bf16", 12, 12, 64, 32, [30, 0], [9, 40], dict(layout="half", dim=24, scaling="linear", factor=4.0), (True, True)),
    ("bf16", 3, 1, 32, 32, [0, 0, 31, 64], [0, 5, 1, 0], dict(layout="half", dim=2, base=500000.0), (True, False)),
    ("bf16", 5, 5, 32, 32, [7], [19], dict(layout="interleaved", dim=30), (False, True)),
    ("bf16", 8, 1, 256, 128, [130], [7], dict(layout="half", dim=64), (True, True)),
    ("bf16", 2, 2, 256, 16, [1], [3], dict(layout="interleaved", dim=254, magnitude=1.25), (True, True)),
    ("bf16", 6, 3, 64, 16, [1, 30], [20, 3], None, (True, True)),
    ("bf16", 6, 3, 64, 16, [1, 30], [20, 3], dict(layout="half", dim=32), (False, False)),
    ("bf16", 4, 2, 128, 16, [2], [20], dict(layout="interleaved", dim=64), (False, False)),
    ("f32", 4, 4, 16, 16, [16, 3], [8, 1], dict(layout="interleaved"), (True, True)),
    ("f32", 6, 3, 128, 256, [200], [57], dict(layout="half", dim=96), (True, True)),
    ("f32", 1, 1, 16, 16, [0], [1], dict(layout="half", dim=10), (True, True)),
    ("f32", 2, 1, 32, 16, [2**20 - 5], [5], dict(layout="half", scaling="linear", factor=16.0), (True, True)),
    ("f32", 7, 7, 64, 16, [40], [11], dict(layout="half", dim=44, freqs=[0.01 * (j + 1) for j in range(22)]), (False, True)),
    ("f32", 40, 10, 64, 64, [3, 900], [500, 131], dict(layout="half"), (True, True)),
    # several rows a workgroup, the last one of fewer; two heads a thread, the last one of one
    ("f32", 32, 8, 64, 64, [0, 10], [4000, 101], dict(layout="half", dim=48), (True, True)),
    ("bf16", 9, 3, 64, 64, [40, 0], [200, 101], dict(layout="half", dim=48), (True, True)),
    ("bf16", 5, 5, 128, 64, [40, 0], [300, 1], dict(layout="interleaved", dim=100), (True, False)),
    # pairs of other halves, two heads a thread, from a part of the first vector to all but the last pair
    ("bf16", 9, 3, 64, 16, [40, 0], [300, 9], dict(layout="half", dim=20), (True, True)),
    ("bf16", 7, 7, 256, 64, [3], [260], dict(layout="half", dim=250), (False, True)),
    ("bf16", 3, 1, 32, 16, [0, 7], [280, 1], dict(layout="half", dim=30), (False, False)),
    ("bf16", 4, 4, 128, 32, [100], [257], dict(layout="half", dim=126, magnitude=0.5), (True, False)),
    ("f32", 5, 1, 128, 32, [100], [300], dict(layout="half", dim=6), (True, True))]


@pytest.mark.parametrize("case", FORMS, ids=range(len(FORMS)))
def test_append_forms(binding, case):
    dtype, heads, kv, hd, page, ctx, new, form, norms = case
    n, R, eps = len(new), sum(new), 1e-5
    used = sum(-(-(c + m) // page) for c, m in zip(ctx, new))
    c = make(binding, page=page, n_pages=used + 1, max_seqs=n + 1, max_ctx=max(a + b for a, b in zip(ctx, new)), max_rows=R + 9,
             heads=heads, kv=kv, hd=hd, dtype=dtype, rope_base=0.0 if form is None else 10000.0)
    if form is not None:
        c.rotary(**form)
        kw = {k: v for k, v in form.items() if k not in ("layout", "dim", "freqs", "magnitude")}
        theta = np.array(form["freqs"]) if "freqs" in form else angles(form.get("dim", hd), **kw)
    else:
        theta = np.zeros(0)
    layout, magnitude = (form or {}).get("layout", "half"), (form or {}).get("magnitude", 1.0)
    books, seq = ref.Books(page, used + 1, n + 1), list(range(n, 0, -1))
    rows = books.plan(seq, ctx, new)
    c.plan(ints(seq), ints(ctx), ints(new), rows=R + 2)
    g = torch.Generator(device="cuda").manual_seed(hd + R)
    x = (torch.randn(R + 2, (heads + 2 * kv) * hd + 16, generator=g, device="cuda") * 2.5).to(c.dtype)  # rows of a wider product
    q, k, v = (x[:, a * hd:b * hd] for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
    gains = torch.randn(2 * hd + 1, generator=g, device="cuda")
    qg, kg = (gains[1 + i * hd:1 + (i + 1) * hd] if use else None for i, use in enumerate(norms))  # at any float's address
    kw = dict(q_gain=qg, k_gain=kg, eps=eps)
    was = [torch.randn(c.pool_shape, generator=g, device="cuda").to(c.dtype) for _ in range(2)]
    pools, out = [w.clone() for w in was], torch.full((R + 2, heads, hd), 9.0, device="cuda", dtype=c.dtype)
    c.append(q, k, v, out, *pools, **kw)
    assert c.status()[0] == R
    pos = [p for _, p in rows]
    keys, values = (torch.stack([p[s // page, :, s % page] for s, _ in rows]) for p in pools)
    check(host(out[:R]), host(q[:R]).reshape(R, heads, hd), None if qg is None else host(qg), eps, pos, theta, layout, c.dtype, magnitude)
    check(host(keys), host(k[:R]).reshape(R, kv, hd), None if kg is None else host(kg), eps, pos, theta, layout, c.dtype, magnitude)
    assert torch.equal(values, v[:R].reshape(R, kv, hd))
    assert (out[R:] == 9).all()  # rows behind the last
    for pool, w in zip(pools, was):  # every other slot of the pool
        hit = torch.zeros(c.pool_shape[0], page, dtype=torch.bool)
        for s, _ in rows:
            hit[s // page, s % page] = True
        keep = ~hit.cuda()
        assert torch.equal(pool.transpose(1, 2)[keep], w.transpose(1, 2)[keep])
    # in place, and keys and values alone: the same bits
    again, q2 = [w.clone() for w in was], q.contiguous().clone()
    c.append(q2, k, v, q2, *again, **kw)
    assert torch.equal(q2.view_as(out)[:R], out[:R]) and all(torch.equal(a, b) for a, b in zip(again, pools))
    again = [w.clone() for w in was]
    c.append(None, k, v, None, *again, **{**kw, "q_gain": None})
    assert all(torch.equal(a, b) for a, b in zip(again, pools))


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("f32", 32)])
def test_heads_at_the_ends_of_the_range(binding, dtype, hd):
    """Heads of zeros, of values whose squares pass fp32 or fall below it, and of values that are not finite; their neighbours
    stay as they are."""
    c = make(binding, page=16, n_pages=2, max_seqs=1, max_ctx=32, max_rows=4, heads=8, kv=8, hd=hd, dtype=dtype, rope_base=10000.0)
    c.plan(ints([0]), ints([0]), ints([1]), rows=1)  # position 0: every angle is 0
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(1, 8, hd, generator=g, device="cuda").to(c.dtype)
    x[0, 1] = 0
    x[0, 2] *= 1e30
    x[0, 3] *= 1e-30
    x[0, 4, 5] = float("inf")
    x[0, 5, 7] = float("nan")
    x[0, 6] = 3e38
    gain, eps = torch.ones(hd, device="cuda"), 1e-6
    pools = [torch.zeros(c.pool_shape, device="cuda", dtype=c.dtype) for _ in range(2)]
    out = torch.empty_like(x)
    c.append(x, x, x, out, *pools, q_gain=gain, k_gain=gain, eps=eps)
    assert c.status()[0] == 1
    table = c.block_table[0, 0]
    for got in (out[0], pools[0][table, :, 0]):
        for h in (0, 2, 3, 6, 7):
            check(host(got[None, h:h + 1]), host(x[:, h:h + 1]), host(gain), eps, [0], angles(hd), "half", c.dtype)
        assert (got[1] == 0).all() and got[5].isnan().all()
        # the infinity, over an infinite mean, is NaN, and so is what the rotation pairs with it (0 * NaN); others are 0
        pair = {5, 5 + hd // 2}
        assert all(got[4, i].isnan() if i in pair else got[4, i] == 0 for i in range(hd))
    assert torch.equal(pools[1][table, :, 0].nan_to_num(7), x[0].nan_to_num(7))


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_elements_that_are_not_turned_keep_their_bits(binding, layout):
    """Without a norm, what lies behind the turned part is a copy: infinities, NaN and all."""
    c = make(binding, page=16, n_pages=2, max_seqs=1, max_ctx=32, max_rows=4, heads=2, kv=2, hd=64, rope_base=10000.0)
    c.rotary(layout=layout, dim=18)
    c.plan(ints([0]), ints([9]), ints([2]), rows=2)
    x = torch.randn(2, 2, 64, device="cuda").bfloat16()
    x[0, 0, 18:21] = torch.tensor([float("inf"), float("nan"), -float("inf")])
    pools = [torch.zeros(c.pool_shape, device="cuda", dtype=c.dtype) for _ in range(2)]
    out = torch.empty_like(x)
    c.append(x, x, x, out, *pools)
    assert torch.equal(out[..., 18:].view(torch.int16), x[..., 18:].view(torch.int16))
    check(host(out[..., :18]), host(x[..., :18]), None, 0, [9, 10], angles(18), layout, c.dtype)


def test_the_default_rotation_and_back(binding):
    """Spelled out, the rotation that a cache starts with gives what it gave before, up to its angles' last bits; another form
    and back gives the same bits."""
    c = make(binding, page=16, n_pages=20, max_seqs=1, max_ctx=300, max_rows=40, heads=4, kv=2, hd=64, dtype="f32", rope_base=10000.0)
    c.plan(ints([0]), ints([200]), ints([40]), rows=40)
    q, k = torch.randn(40, 4, 64, device="cuda"), torch.randn(40, 2, 64, device="cuda")
    pools = [torch.zeros(c.pool_shape, device="cuda") for _ in range(2)]
    outs = []
    for form in (None, {}, dict(layout="interleaved", dim=20), {}):
        if form is not None:
            c.rotary(**form)
        out = torch.empty_like(q)
        c.append(q, k, k, out, *pools)
        outs.append(out)
    assert torch.equal(outs[1], outs[3]) and not torch.equal(outs[1], outs[2])
    # a cosine or sine rounded to the other neighbour: 2^-23 of |a| + |b|, and the sums' roundings
    size = turn(host(q), np.zeros(40), np.zeros(32), "half")[1]
    assert (np.abs(host(outs[0]) - host(outs[1])) <= 8 * 2.0**-24 * size).all()


def test_refusals(binding):
    c = make(binding, rope_base=10000.0)
    none = make(binding)
    with pytest.raises(binding.CllmError, match="ERR_STATE.*rope_base"):
        none.rotary()
    for bad in (dict(dim=65), dict(dim=66), dict(base=-1.0), dict(scaling="linear"), dict(scaling="parts", factor=2.0)):
        with pytest.raises(binding.CllmError, match="ERR_ARG"):
            c.rotary(**bad)
    one = ints([1])
    q, kv = torch.zeros(8, 4, 64, device="cuda").bfloat16(), torch.zeros(8, 2, 64, device="cuda").bfloat16()
    pools = [torch.zeros(c.pool_shape, device="cuda").bfloat16() for _ in range(2)]
    gain = torch.ones(64, device="cuda")
    with pytest.raises(binding.CllmError, match="ERR_STATE"):
        c.append(q, kv, kv, q, *pools, q_gain=gain)  # no plan yet
    c.plan(one, one, one, rows=8)
    for eps in (0.0, -1.0, 1e-39, float("inf"), float("nan")):
        with pytest.raises(binding.CllmError, match="eps"):
            c.append(q, kv, kv, q, *pools, k_gain=gain, eps=eps)
    with pytest.raises(binding.CllmError, match="q_gain without q"):
        c.append(None, kv, kv, None, *pools, q_gain=gain)
    with pytest.raises(ValueError, match="gain"):
        c.append(q, kv, kv, q, *pools, q_gain=gain.cpu())
    L, p, z = binding.lib(), [x.data_ptr() for x in pools], np.ones(64, np.float32)
    args = (c.h, q.data_ptr(), 256, kv.data_ptr(), 128, kv.data_ptr(), 128, q.data_ptr(), 256, *p)
    assert L.cllm_paged_append_norm(*args, z.ctypes.data, None, 1e-6) == 1  # host memory
    assert L.cllm_paged_append_norm(*args, gain.data_ptr() + 2, None, 1e-6) == 1  # not a float's address
    with torch.cuda.stream(torch.cuda.Stream()):
        with pytest.raises(ValueError, match="stream"):
            c.rotary()
    c.close()
    with pytest.raises(ValueError, match="closed"):
        c.rotary()


def test_captured_appends(binding):
    """A captured append replayed for other plans and values, with other eager work between; the factors of a later form of
    the same layout reach it."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = make(binding, page=16, n_pages=30, max_seqs=2, max_ctx=200, max_rows=24, heads=4, kv=2, hd=64, dtype="f32", rope_base=10000.0)
        seq, ctx, new = ints([0, 1]), ints([0, 0]), ints([0, 0])
        q, k = torch.zeros(24, 4, 64, device="cuda"), torch.zeros(24, 2, 64, device="cuda")
        out, gain = torch.zeros_like(q), torch.randn(64, device="cuda")
        pools = [torch.zeros(c.pool_shape, device="cuda") for _ in range(2)]

        def step():
            c.plan(seq, ctx, new, rows=24, max_new=16)
            c.append(q, k, k, out, *pools, q_gain=gain, k_gain=gain)

        c.rotary(dim=32, scaling="linear", factor=2.0)
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
            with pytest.raises(binding.CllmError, match="ERR_STATE.*captured"):
                c.rotary(dim=16)
        for i, (a, m, factor) in enumerate([([0, 0], [3, 5], 2.0), ([3, 5], [16, 8], 2.0), ([19, 13], [1, 0], 4.0), ([20, 13], [2, 2], 4.0)]):
            c.rotary(dim=32, scaling="linear", factor=factor)
            for x, v in ((ctx, a), (new, m)):
                x.copy_(ints(v))
            q.normal_()
            k.normal_()
            graph.replay()
            R = sum(m)
            assert c.status()[0] == R
            pos = [p for b in range(2) for p in range(a[b], a[b] + m[b])]
            check(host(out[:R]), host(q[:R]), host(gain), 1e-6, pos, angles(32, scaling="linear", factor=factor), "half", c.dtype)
            keys = pools[0].transpose(1, 2).reshape(-1, 2, 64)[c.row_slot[:R].long()]
            check(host(keys), host(k[:R]), host(gain), 1e-6, pos, angles(32, scaling="linear", factor=factor), "half", c.dtype)
