"""GPU tests of the paged KV cache (binding.PagedCache) against the plain references of
tests/paged_ref.py: the pool's books, rotary append, attention of chunks of new tokens, refusals, and a
run of the three as a decoder makes it. Tolerances are half steps of the output's type plus bounds of
the fp32 arithmetic, derived at their definitions."""
import random

import numpy as np
import pytest

from tests import paged_ref as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def binding():
    from paper_2403_00835_amd import binding as b
    return b


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def make(binding, page=16, n_pages=64, max_seqs=8, max_ctx=512, max_rows=256, heads=4, kv=2, hd=64, **kw):
    return binding.PagedCache(heads, kv, hd, page, n_pages, max_seqs, max_ctx, max_rows, **kw)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def host(x):
    return x.double().cpu().numpy()


# ------------------------------------------------------------------------------------------ plan
def check_books(c, books, n_pages):
    table = c.block_table.cpu().numpy()
    for s, pages in enumerate(books.table):
        want = np.full(table.shape[1], -1)
        want[:len(pages)] = pages
        np.testing.assert_array_equal(table[s], want)
    np.testing.assert_array_equal(c.seq_pages.cpu().numpy(), [len(t) for t in books.table])
    np.testing.assert_array_equal(c.free_list[:len(books.free)].cpu().numpy(), books.free)


def check_rows(c, rows, new):
    start = np.concatenate([[0], np.cumsum(new)])
    np.testing.assert_array_equal(c.row_start[:len(new) + 1].cpu().numpy(), start)
    np.testing.assert_array_equal(c.row_slot[:len(rows)].cpu().numpy(), [s for s, _ in rows])
    np.testing.assert_array_equal(c.row_pos[:len(rows)].cpu().numpy(), [p for _, p in rows])


@pytest.mark.parametrize("page,slots,max_ctx,seed", [(16, 1, 100, 0), (16, 7, 300, 1), (64, 64, 1000, 2), (256, 65, 700, 3),
                                                     (32, 1024, 90, 4)])
def test_plan_follows_the_books(binding, page, slots, max_ctx, seed):
    rng = random.Random(seed)
    n_pages = max(2, slots * max_ctx // page // 2)
    c = make(binding, page=page, n_pages=n_pages, max_seqs=slots, max_ctx=max_ctx, max_rows=max(max_ctx, 40 * slots))
    books = ref.Books(page, n_pages, slots)
    refused = 0
    for _ in range(12):
        n = rng.randint(1, slots)
        seq = rng.sample(range(slots), n)
        total = [rng.choice([0, 1, page, page + 1, rng.randint(0, max_ctx), max_ctx]) for _ in seq]
        new = [min(t, rng.choice([0, 0, 1, 2, 39, 40])) for t in total]
        ctx = [t - m for t, m in zip(total, new)]
        rows = books.plan(seq, ctx, new)
        c.plan(ints(seq), ints(ctx), ints(new), rows=max(sum(new), 1), max_new=max(new))
        if rows is None:
            refused += 1
            with pytest.raises(binding.CllmError, match="ERR_CAPACITY.*pages"):
                c.status()
        else:
            assert c.status() == (len(rows), len(books.free))
            check_rows(c, rows, new)
        check_books(c, books, n_pages)
    assert refused < 12


def test_undoing_a_plan_restores_the_free_list(binding):
    c = make(binding, max_seqs=3, max_rows=400)
    seq, base = ints([2, 0, 1]), ints([40, 0, 17])
    c.plan(seq, base, ints([0, 0, 0]), rows=0)
    before = c.free_list.clone(), c.block_table.clone(), c.status()
    c.plan(seq, base, ints([60, 100, 1]), rows=400)
    assert c.status() == (161, 64 - 7 - 7 - 2)
    c.plan(seq, base, ints([0, 0, 0]), rows=0)
    assert c.status() == before[2]
    n = before[2][1]
    assert torch.equal(c.free_list[:n], before[0][:n]) and torch.equal(c.block_table, before[1])


REFUSED = [  # slots, contexts, new tokens, bounds, what the status says
    ([0, 0], [1, 2], [1, 1], {}, "ERR_ARG"), ([8, 0], [1, 2], [1, 1], {}, "ERR_ARG"),
    ([-1, 0], [1, 2], [1, 1], {}, "ERR_ARG"), ([1, 0], [-1, 2], [1, 1], {}, "ERR_ARG"),
    ([1, 0], [1, 2], [1, -1], {}, "ERR_ARG"), ([1, 0], [512, 2], [1, 1], {}, "ERR_ARG"),
    ([1, 0], [2**31 - 1, 2], [1, 1], {}, "ERR_ARG"), ([1, 0], [1, 2], [1, 9], dict(max_new=8), "ERR_ARG"),
    ([1, 0], [1, 90], [1, 1], dict(max_len=90), "ERR_ARG"), ([1, 0], [1, 2], [8, 9], dict(rows=16), "ERR_CAPACITY.*rows"),
    ([1, 0], [2, 510], [1, 2], dict(rows=16), "ERR_CAPACITY.*pages")]


@pytest.mark.parametrize("case", REFUSED, ids=range(len(REFUSED)))
def test_a_refused_plan_changes_nothing_and_has_no_rows(binding, case):
    seq, ctx, new, bounds, says = case
    c = make(binding, n_pages=32)
    c.plan(ints([3, 0]), ints([20, 5]), ints([4, 0]), rows=4)
    free = c.status()[1]
    keep = [x.clone() for x in (c.block_table, c.seq_pages, c.free_list)]
    c.plan(ints(seq), ints(ctx), ints(new), **{"rows": 64, **bounds})
    with pytest.raises(binding.CllmError, match=says):
        c.status()
    assert all(torch.equal(a, b) for a, b in zip(keep, (c.block_table, c.seq_pages, c.free_list)))
    q, kv = torch.zeros(64, 4, 64, device="cuda").bfloat16(), torch.ones(64, 2, 64, device="cuda").bfloat16()
    pools = [torch.full(c.pool_shape, 7.0, device="cuda").bfloat16() for _ in range(2)]
    out = torch.full_like(q, 5.0)
    c.append(q, kv, kv, q, *pools)
    c.attn(q, *pools, out)
    assert (out == 5).all() and (q == 0).all() and all((p == 7).all() for p in pools)
    c.plan(ints([1]), ints([0]), ints([3]), rows=3)  # the next one is served
    assert c.status() == (3, free - 1)


def test_calls_are_refused_before_the_device(binding):
    c = make(binding)
    q, kv = torch.zeros(8, 4, 64, device="cuda").bfloat16(), torch.zeros(8, 2, 64, device="cuda").bfloat16()
    pools = [torch.zeros(c.pool_shape, device="cuda").bfloat16() for _ in range(2)]
    for call in (lambda: c.append(None, kv, kv, None, *pools), lambda: c.attn(q, *pools, q)):
        with pytest.raises(binding.CllmError, match="ERR_STATE"):
            call()  # no plan yet
    one = ints([1])
    for kw, err in ((dict(rows=-1), "ERR_ARG"), (dict(rows=257), "ERR_CAPACITY"), (dict(rows=4, max_new=5), "ERR_ARG"),
                    (dict(rows=4, max_len=513), "ERR_CAPACITY"), (dict(rows=4, max_len=-1), "ERR_ARG")):
        with pytest.raises(binding.CllmError, match=err):
            c.plan(one, one, one, **kw)
    with pytest.raises(binding.CllmError, match="ERR_ARG"):
        c.plan(ints([0] * 9), ints([0] * 9), ints([0] * 9), rows=1)  # more requests than slots
    for bad in ((one.long(), one, one), (one, ints([1, 2]), one), (one, one, one.cpu()), (one, one, ints([1, 2])[::2][:0])):
        with pytest.raises(ValueError):
            c.plan(*bad, rows=4)
    c.plan(one, one, one, rows=8)
    wide = torch.zeros(8, 8, 128, device="cuda").bfloat16()
    for bad in (q[:4], q.float(), wide[:, :4, ::2], q[:, :2], q.cpu(), q.transpose(0, 1)):
        with pytest.raises(ValueError):
            c.attn(bad, *pools, q)
        with pytest.raises(ValueError):
            c.append(bad, kv, kv, bad, *pools)
    with pytest.raises(ValueError):
        c.append(q, kv, kv, None, *pools)
    with pytest.raises(ValueError):
        c.attn(q, pools[0][:-1], pools[1], q)
    with pytest.raises(ValueError):
        c.attn(q, *pools, q, lse=torch.zeros(8, 4, device="cuda").half())
    odd = torch.zeros(8 * 256 + 8, device="cuda").bfloat16()
    with pytest.raises(binding.CllmError, match="aligned"):
        c.attn(odd[1:8 * 256 + 1].view(8, 4, 64), *pools, q)
    with pytest.raises(binding.CllmError, match="stride"):
        c.attn(torch.zeros(8, 257, device="cuda").bfloat16()[:, :256], *pools, q)
    with pytest.raises(binding.CllmError, match="scale"):
        c.attn(q, *pools, q, scale=float("inf"))
    L, p, z = binding.lib(), [x.data_ptr() for x in pools], np.zeros(1 << 16, np.uint16)
    assert L.cllm_paged_attn(c.h, z.ctypes.data & ~15, 256, *p, 0.0, q.data_ptr(), 256, None) == 1  # host memory
    assert L.cllm_paged_attn(c.h, q.data_ptr(), 256, *p, 0.0, q.data_ptr(), 264, None) == 1  # out = q, other stride
    with torch.cuda.stream(torch.cuda.Stream()):
        with pytest.raises(ValueError, match="stream"):
            c.attn(q, *pools, q)
    c.close()
    with pytest.raises(ValueError, match="closed"):
        c.attn(q, *pools, q)


def test_scales_at_the_ends_of_their_range(binding):
    """A scale whose product with log2(e) is above fp32's range is refused; the smallest gives equal weights, and not
    those of the default."""
    c = make(binding, page=16, n_pages=4, max_seqs=1, max_ctx=40, max_rows=2, heads=2, kv=1, hd=32)
    books = ref.Books(16, 4, 1)
    books.plan([0], [30], [2])
    c.plan(ints([0]), ints([30]), ints([2]), rows=2)
    kp, vp = fill(c, books, [0], [32], seed=9)
    q, out = torch.randn(2, 2, 32, device="cuda").bfloat16(), torch.full((2, 2, 32), 5.0, device="cuda").bfloat16()
    for bad in (3e38, -3.4e38, 2.4e38, 1e39, float("nan")):
        with pytest.raises(binding.CllmError, match="ERR_ARG.*scale"):
            c.attn(q, kp, vp, out, scale=bad)
    for bad in (1e-46, 0.0):
        with pytest.raises(ValueError, match="scale"):
            c.attn(q, kp, vp, out, scale=bad)
    assert (out == 5).all()
    v = ref.gather(host(vp), books.table[0], 32)[0]
    for scale in (1e-45, -1e-45, 1e-38):  # scores of at most 2^-100: every weight is 1
        c.attn(q, kp, vp, out, scale=scale)
        for i in range(2):
            want = v[:31 + i].mean(0)
            assert (np.abs(host(out[i]) - want) <= 2.0**-8 * np.abs(want) + 2.0**-17).all()


# ---------------------------------------------------------------------------------------- append
@pytest.mark.parametrize("dtype,heads,kv,hd,page,ctx,new,base", [
    ("bf16", 4, 4, 128, 64, [0, 63, 100], [1, 2, 70], 10000.0), ("bf16", 14, 2, 64, 16, [5], [33], 10000.0),
    ("bf16", 3, 1, 32, 32, [0, 0, 31, 64], [0, 5, 1, 0], 500000.0), ("bf16", 8, 1, 256, 128, [130], [7], 10000.0),
    ("f32", 4, 4, 16, 16, [16, 3], [8, 1], 10000.0), ("f32", 6, 3, 128, 256, [200], [57], 10000.0),
    ("bf16", 2, 2, 64, 16, [1, 30], [20, 3], 0.0), ("f32", 2, 1, 32, 16, [2**20 - 5], [5], 10000.0)])
def test_append(binding, dtype, heads, kv, hd, page, ctx, new, base):
    n, R = len(new), sum(new)
    used = sum(-(-(c + m) // page) for c, m in zip(ctx, new))
    c = make(binding, page=page, n_pages=used + 1, max_seqs=n + 1, max_ctx=max(c + m for c, m in zip(ctx, new)),
             max_rows=R + 9, heads=heads, kv=kv, hd=hd, dtype=dtype, rope_base=base)
    books, seq = ref.Books(page, used + 1, n + 1), list(range(n, 0, -1))
    rows = books.plan(seq, ctx, new)
    c.plan(ints(seq), ints(ctx), ints(new), rows=R + 2)
    g = torch.Generator(device="cuda").manual_seed(hd)
    x = torch.randn(R + 2, (heads + 2 * kv) * hd + 16, generator=g, device="cuda").to(c.dtype)  # rows of a wider product
    q, k, v = (x[:, a * hd:b * hd] for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
    was = [torch.randn(c.pool_shape, generator=g, device="cuda").to(c.dtype) for _ in range(2)]
    pools, out = [w.clone() for w in was], torch.full((R + 2, heads, hd), 9.0, device="cuda", dtype=c.dtype)
    c.append(q, k, v, out, *pools)
    assert c.status()[0] == R
    pos = [p for _, p in rows]
    step = half_step(c.dtype)
    for got, src, h in ((out[:R], q[:R], heads), (None, k[:R], kv), (None, v[:R], kv)):
        raw = host(src).reshape(R, h, hd)
        turned = src.data_ptr() != v.data_ptr() and base > 0
        want = ref.rotate(raw, pos, base) if turned else raw
        if got is None:
            got = torch.stack([pools[src.data_ptr() == v.data_ptr()][s // page, :, s % page] for s, _ in rows])
        # cos and sin rounded once, two products and a sum in fp32: three half steps of |a| + |b| at most,
        # then the output's half step
        size = np.abs(raw) + np.abs(np.roll(raw, hd // 2, -1))
        tol = (step * (np.abs(want) + 4 * 2.0**-24 * size) + 4 * 2.0**-24 * size) if turned else 0 * size
        assert (np.abs(host(got) - want) <= tol).all()
    assert (out[R:] == 9).all()  # rows behind the last
    for pool, w in zip(pools, was):  # every other slot of the pool
        hit = torch.zeros(c.pool_shape[0], page, dtype=torch.bool)
        for s, _ in rows:
            hit[s // page, s % page] = True
        keep = ~hit.cuda()
        assert torch.equal(pool.transpose(1, 2)[keep], w.transpose(1, 2)[keep])
    # in place, and keys and values alone: the same bits
    again, q2 = [w.clone() for w in was], q.contiguous().clone()
    c.append(q2, k, v, q2, *again)
    assert torch.equal(q2.view_as(out)[:R], out[:R]) and all(torch.equal(a, b) for a, b in zip(again, pools))
    again = [w.clone() for w in was]
    c.append(None, k, v, None, *again)
    assert all(torch.equal(a, b) for a, b in zip(again, pools))


# ------------------------------------------------------------------------------------- attention
def fill(c, books, seq, total, seed, scatter=float("nan")):
    """Pools that hold `scatter` everywhere but in the requests' tokens."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    pools = []
    for _ in range(2):
        x = torch.randn(c.pool_shape, generator=g, device="cuda").to(c.dtype)
        keep = torch.zeros(c.pool_shape[0], c.pool_shape[2], dtype=torch.bool)
        for s, t in zip(seq, total):
            for i, p in enumerate(books.table[s]):
                keep[p, :max(0, min(t - i * books.page, books.page))] = True
        pools.append(torch.where(keep.cuda()[:, None, :, None], x, torch.full_like(x, scatter)))
    return pools


def tolerance(c, q, k, want, lse, mag, scale, keys):
    """Bounds of |out - want| and |lse - want|. Scores are sums of hd products of exact inputs in fp32:
    off by (hd + 8) 2^-23 of sum |q k| (with the scale and the exponent's argument), which is the
    relative error of a weight; sums over the keys add keys 2^-23; a weight's two bf16 planes 2^-17. The
    weights' errors reach the output times sum p |v|, once through the numerator and once through the
    denominator; then the output's half step. The weights of long bf16 chunks (more than 64 rows x heads of
    a group) are rounded to bf16 in the numerator: a half step, 2^-8, of each."""
    group = want.shape[1] // k.shape[0]
    hd = q.shape[-1]
    size = np.stack([np.abs(q[:, h]) @ np.abs(k[h // group]).T for h in range(q.shape[1])], 1).max(-1) * abs(scale)
    w = (hd + 8) * 2.0**-23 * size + (keys + 8) * 2.0**-23
    bf16 = c.dtype == torch.bfloat16
    arith = (2 * (w + (2.0**-17 if bf16 else 0))[..., None] + (2.0**-8 if bf16 and len(q) * group > 64 else 0)) * mag
    return half_step(c.dtype) * (np.abs(want) + arith) + arith, w + 2.0**-22 * np.abs(lse)


def check_attn(c, books, seq, ctx, new, seed, scale=None, bounds=None, strided=False):
    R, H, hd = sum(new), c.n_heads, c.head_dim
    total = [a + b for a, b in zip(ctx, new)]
    assert books.plan(seq, ctx, new) is not None
    c.plan(ints(seq), ints(ctx), ints(new), **{"rows": R + 1, **(bounds or {})})
    kp, vp = fill(c, books, seq, total, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    q = (torch.randn(R + 1, H + (1 if strided else 0), hd, generator=g, device="cuda") * 1.5).to(c.dtype)[:, :H]
    out = torch.full((R + 1, H + (2 if strided else 0), hd), 3.0, device="cuda", dtype=c.dtype)[:, :H]
    lse = torch.full((R + 1, H), 3.0, device="cuda")
    c.attn(q, kp, vp, out, scale=scale, lse=lse)
    assert c.status()[0] == R
    sc = scale if scale is not None else hd ** -0.5
    kh, vh, qh = host(kp), host(vp), host(q)
    r = 0
    for s, a, m in zip(seq, ctx, new):
        if m == 0:
            continue
        k, v = (ref.gather(x, books.table[s], a + m) for x in (kh, vh))
        want, wl, mag = ref.attend(qh[r:r + m], k, v, a, sc)
        tol, tl = tolerance(c, qh[r:r + m], k, want, wl, mag, sc, a + m)
        d, dl = np.abs(host(out[r:r + m]) - want), np.abs(host(lse[r:r + m]) - wl)
        assert (d <= tol).all(), f"request {s}: output off by {np.nanmax(d / tol)} of its bound, {np.isnan(d).sum()} NaN"
        assert (dl <= tl).all(), f"request {s}: lse off by {np.nanmax(dl / tl)} of its bound"
        r += m
    assert (out[R:] == 3).all() and (lse[R:] == 3).all()
    return q, kp, vp, out, lse


ATTN = [  # dtype, heads, kv heads, head dim, page, contexts, new tokens
    ("bf16", 4, 4, 128, 64, [0], [1]), ("bf16", 4, 4, 128, 64, [511], [1]), ("bf16", 4, 4, 128, 64, [512, 1], [1, 1]),
    ("bf16", 8, 2, 128, 16, [700, 3, 0, 64], [1, 1, 1, 1]), ("bf16", 14, 2, 64, 32, [17, 0, 130], [5, 64, 0]),
    ("bf16", 2, 2, 128, 64, [690], [16]), ("bf16", 2, 2, 128, 128, [1100, 40], [32, 31]),
    ("bf16", 2, 2, 128, 64, [1215], [64]), ("bf16", 8, 1, 64, 16, [63, 62], [8, 3]), ("bf16", 3, 1, 32, 256, [255, 256], [2, 9]),
    ("bf16", 1, 1, 256, 32, [100, 700], [17, 1]), ("bf16", 4, 2, 256, 16, [33], [40]),
    ("bf16", 8, 2, 128, 64, [900], [65]), ("bf16", 4, 2, 64, 16, [0, 1000], [300, 129]), ("bf16", 7, 1, 128, 32, [333, 0], [77, 1]),
    ("bf16", 4, 4, 32, 64, [20], [200]), ("bf16", 2, 1, 256, 64, [65], [140]), ("bf16", 16, 1, 128, 128, [5, 600, 90], [4, 5, 128]),
    ("bf16", 1, 1, 128, 64, [0], [129]), ("bf16", 32, 8, 128, 64, [1500], [40]), ("bf16", 2, 2, 128, 16, [0, 3000], [640, 100]),
    ("bf16", 8, 1, 32, 16, [2500, 10], [9, 1]), ("bf16", 6, 2, 256, 64, [1300, 0, 7], [30, 500, 2]),
    ("bf16", 64, 1, 64, 16, [300, 0], [1, 3]), ("f32", 2, 2, 64, 64, [900], [130]),
    ("f32", 4, 4, 16, 16, [16], [8]), ("f32", 12, 12, 64, 32, [5, 700, 301], [41, 3, 17]), ("f32", 4, 1, 128, 64, [1030, 1], [30, 1]),
    ("f32", 6, 2, 32, 16, [0, 15], [130, 1]), ("f32", 2, 2, 128, 256, [513], [70])]


@pytest.mark.parametrize("case", ATTN, ids=["-".join(str(x) for x in a[:5]) + f"-ctx{a[5]}-new{a[6]}" for a in ATTN])
def test_attention(binding, case):
    dtype, heads, kv, hd, page, ctx, new = case
    n, total = len(new), [a + b for a, b in zip(ctx, new)]
    n_pages = sum(-(-t // page) for t in total) + 2
    c = make(binding, page=page, n_pages=n_pages, max_seqs=n + 2, max_ctx=max(total), max_rows=sum(new) + 1, heads=heads, kv=kv,
             hd=hd, dtype=dtype)
    books, seq = ref.Books(page, n_pages, n + 2), list(range(n + 1, 1, -1))
    half = [t // 2 for t in total]  # pages interleaved: the requests grew in turn
    books.plan(seq, half, [0] * n)
    c.plan(ints(seq), ints(half), ints([0] * n), rows=0)
    check_attn(c, books, seq, ctx, new, seed=hd + n)
    # the tightest bounds, strided rows, another scale; then in place: the same bits
    q, kp, vp, out, _ = check_attn(c, books, seq, ctx, new, seed=hd, scale=-0.11, strided=True,
                                     bounds=dict(max_new=max(new), max_len=max(total)))
    c.attn(q, kp, vp, q, scale=-0.11)
    assert torch.equal(q[:sum(new)], out[:sum(new)])


@pytest.mark.parametrize("heads,kv,hd,page,n,lo,hi", [(8, 8, 128, 64, 68, 17, 64), (16, 8, 64, 16, 68, 9, 32), (32, 16, 32, 32, 36, 9, 32),
                                                      (4, 4, 256, 64, 132, 17, 40), (8, 8, 128, 16, 63, 17, 64)])
def test_many_requests_of_a_block_each(binding, heads, kv, hd, page, n, lo, hi):
    """Enough blocks to fill the device (all but the last case), one request of a token, one of none and one long
    chunk among them: the formula, and each block's bits as in a plan of its own, with values that are not finite
    in tokens that some rows see."""
    rng = random.Random(hd)
    new = [rng.randint(lo, hi) for _ in range(n)]
    ctx = [rng.randint(250, 500) for _ in range(n)]
    new[3], new[7], new[11], ctx[12], ctx[13] = 1, 0, 70, 0, 256 - new[13]
    total = [a + b for a, b in zip(ctx, new)]
    n_pages = sum(-(-t // page) for t in total) + 1
    c = make(binding, page=page, n_pages=n_pages, max_seqs=n, max_ctx=max(total), max_rows=sum(new) + 1, heads=heads, kv=kv, hd=hd)
    books, seq = ref.Books(page, n_pages, n), list(range(n))
    q, kp, vp, out, lse = check_attn(c, books, seq, ctx, new, seed=hd)
    start = np.concatenate([[0], np.cumsum(new)])
    mine = [0, 3, 12, 13, 14, n - 1]

    def alone(s):
        c.plan(ints([s]), ints([ctx[s]]), ints([new[s]]), rows=new[s])
        o, ls = torch.empty_like(q[:new[s]]), torch.empty_like(lse[:new[s]])
        c.attn(q[start[s]:start[s + 1]], kp, vp, o, lse=ls)
        return o, ls

    for s in mine:
        o, ls = alone(s)
        assert torch.equal(o, out[start[s]:start[s + 1]]) and torch.equal(ls, lse[start[s]:start[s + 1]])
    for s in mine:  # a token in the midst of the new ones, and one of the first
        for t, d, value in ((ctx[s] + new[s] // 2, 5, float("inf")), (ctx[s] + new[s] // 3, hd - 1, float("nan")),
                            (total[s] // 9, 6, -float("inf"))):
            vp[books.table[s][t // page], :, t % page, d] = value
    c.plan(ints(seq), ints(ctx), ints(new), rows=sum(new))
    odd = torch.empty_like(out)
    c.attn(q, kp, vp, odd)
    for s in mine:
        a, b = alone(s)[0], odd[start[s]:start[s + 1]]
        same = (a == b) | (torch.isnan(a) & torch.isnan(b))
        assert same.all()
        at = new[s] // 2
        assert torch.isfinite(b[:at, :, 5]).all() and (b[at:, :, 5] == float("inf")).all()
        assert torch.isnan(b[new[s] // 3:, :, hd - 1]).all() and torch.isfinite(b[:new[s] // 3, :, hd - 1]).all()
        keep = [d for d in range(hd) if d not in (5, 6, hd - 1)]
        assert torch.equal(b[..., keep], out[start[s]:start[s + 1]][..., keep])


@pytest.mark.parametrize("dtype,heads,kv,hd,ctx,m", [("bf16", 4, 4, 128, 500, 40), ("bf16", 8, 2, 64, 70, 16),
                                                     ("bf16", 4, 2, 128, 120, 90), ("f32", 2, 2, 64, 60, 30)])
def test_unseen_tokens_do_not_reach_a_row(binding, dtype, heads, kv, hd, ctx, m):
    """NaN and infinities in tokens of the chunk: the rows before them keep their bits, the rows that
    see them are what the products make of them."""
    total, page = ctx + m, 32
    n_pages = -(-total // page) + 1
    c = make(binding, page=page, n_pages=n_pages, max_seqs=1, max_ctx=total, max_rows=m, heads=heads, kv=kv, hd=hd, dtype=dtype)
    books = ref.Books(page, n_pages, 1)
    books.plan([0], [ctx], [m])
    c.plan(ints([0]), ints([ctx]), ints([m]), rows=m)
    kp, vp = fill(c, books, [0], [total], seed=5)
    q = torch.randn(m, heads, hd, device="cuda").to(c.dtype)
    want = torch.empty_like(q)
    c.attn(q, kp, vp, want)
    assert torch.isfinite(want).all()
    at = m // 3  # the first row that sees the value

    def run(pool, value, d=slice(None)):
        pools = [kp.clone(), vp.clone()]
        t = ctx + at
        pools[pool][books.table[0][t // page], :, t % page, d] = value
        out = torch.empty_like(q)
        c.attn(q, *pools, out)
        assert torch.equal(out[:at], want[:at])
        return out[at:]

    nan = float("nan")
    assert torch.isnan(run(0, nan)).all()
    assert torch.isnan(run(1, nan)).all()
    out = run(1, nan, 3)
    assert torch.isnan(out[..., 3]).all() and torch.isfinite(out[..., :3]).all() and torch.isfinite(out[..., 4:]).all()
    for value in (float("inf"), -float("inf")):
        out = run(1, value, 7)
        assert (out[..., 7] == value).all() and torch.isfinite(out[..., 8:]).all()


def test_infinite_values_of_both_signs(binding):
    c = make(binding, page=16, n_pages=4, max_seqs=1, max_ctx=48, max_rows=8, heads=1, kv=1, hd=32)
    books = ref.Books(16, 4, 1)
    books.plan([0], [40], [8])
    c.plan(ints([0]), ints([40]), ints([8]), rows=8)
    kp, vp = fill(c, books, [0], [48], seed=1)
    page = books.table[0][2]
    vp[page, 0, 10, 0], vp[page, 0, 12, 0] = float("inf"), -float("inf")  # positions 42 and 44
    q = torch.randn(8, 1, 32, device="cuda").bfloat16()
    out = torch.empty_like(q)
    c.attn(q, kp, vp, out)
    first = out[:, 0, 0].float()
    assert torch.isfinite(first[:2]).all() and (first[2:4] == float("inf")).all() and torch.isnan(first[4:]).all()
    assert torch.isfinite(out[:, 0, 1:]).all()


@pytest.mark.parametrize("heads,kv,hd,ctx,m,at", [
    (2, 2, 64, 0, 140, 10), (8, 1, 128, 0, 130, 3), (8, 1, 128, 0, 130, 40), (2, 1, 32, 0, 70, 0), (1, 1, 256, 0, 129, 63),
    (2, 2, 128, 30, 100, 50), (4, 4, 128, 40, 80, 20), (1, 1, 64, 250, 100, 252), (8, 1, 64, 700, 66, 705)])
def test_infinities_in_the_first_chunk_that_a_tile_walks(binding, heads, kv, hd, ctx, m, at):
    """Long chunks whose tiles begin (from context 0, or in a range of keys that starts at the new tokens) with a chunk
    of keys that only some of the rows see: values that are not finite reach the rows that see them as they are."""
    total, page = ctx + m, 16
    n_pages = -(-total // page) + 1
    c = make(binding, page=page, n_pages=n_pages, max_seqs=1, max_ctx=total, max_rows=m, heads=heads, kv=kv, hd=hd)
    books = ref.Books(page, n_pages, 1)
    books.plan([0], [ctx], [m])
    c.plan(ints([0]), ints([ctx]), ints([m]), rows=m)
    kp, vp = fill(c, books, [0], [total], seed=hd)
    q = torch.randn(m, heads, hd, generator=torch.Generator(device="cuda").manual_seed(m), device="cuda").bfloat16()
    want, out = torch.empty_like(q), torch.empty_like(q)
    c.attn(q, kp, vp, want)
    assert torch.isfinite(want).all()
    inf, nan = float("inf"), float("nan")
    put = [(at, 3, inf), (at, 4, -inf), (at, 5, nan), (at, 6, inf), (at + 2, 6, -inf), (at + 1, hd - 1, inf)]
    for t, d, value in put:
        vp[books.table[0][t // page], :, t % page, d] = value
    c.attn(q, kp, vp, out)
    keep = [d for d in range(hd) if d not in (3, 4, 5, 6, hd - 1)]
    assert torch.equal(out[..., keep], want[..., keep])
    for d in (3, 4, 5, 6, hd - 1):
        for i in range(m):
            seen = [value for t, e, value in put if e == d and t <= ctx + i]
            if not seen:
                assert torch.equal(out[i, :, d], want[i, :, d])
            elif sum(seen) != sum(seen):
                assert torch.isnan(out[i, :, d]).all(), (i, d)
            else:
                assert (out[i, :, d] == seen[0]).all(), (i, d, out[i, :, d])


def test_scores_far_apart_and_all_the_same(binding):
    """A row whose one key outweighs the others by more than fp32's range, and rows of equal scores."""
    c = make(binding, page=16, n_pages=80, max_seqs=2, max_ctx=1200, max_rows=4, heads=2, kv=1, hd=64)
    books = ref.Books(16, 80, 2)
    books.plan([0], [1100], [2])
    c.plan(ints([0]), ints([1100]), ints([2]), rows=2)
    kp, vp = fill(c, books, [0], [1102], seed=3)
    q = torch.full((2, 2, 64), 1.0, device="cuda").bfloat16()
    out = torch.empty_like(q)
    kp[books.table[0][50], :, 3] = 100.0  # position 803: score 800, the others a few
    c.attn(q, kp, vp, out)
    assert torch.equal(out, vp[books.table[0][50], 0, 3].expand_as(out))
    q.zero_()
    lse = torch.empty(2, 2, device="cuda")
    c.attn(q, kp, vp, out, lse=lse)
    v = ref.gather(host(vp), books.table[0], 1102)[0]
    for i in range(2):
        np.testing.assert_allclose(host(lse[i]), np.log(1101 + i), rtol=2.0**-22)
        # weights are exact (1): sums of 1101 values in fp32, then the half step
        assert (np.abs(host(out[i]) - v[:1101 + i].mean(0)) <= 2.0**-8 * np.abs(v[:1101 + i].mean(0)) + 2.0**-13).all()


@pytest.mark.parametrize("dtype,heads,kv,hd,page,ctx,m", [("bf16", 2, 2, 128, 64, 1000, 64), ("bf16", 8, 2, 64, 16, 505, 16),
                                                          ("f32", 2, 1, 64, 32, 700, 30)])
def test_a_rows_bits_do_not_depend_on_the_call(binding, dtype, heads, kv, hd, page, ctx, m):
    """One chunk; its tokens one by one; among many other requests (no split); in other pages."""
    total, others = ctx + m, 600
    n_pages = -(-total // page) + others * 2 + 4
    c = make(binding, page=page, n_pages=n_pages, max_seqs=others + 1, max_ctx=total, max_rows=m + others, heads=heads, kv=kv,
             hd=hd, dtype=dtype)
    books = ref.Books(page, n_pages, others + 1)
    books.plan([0], [ctx], [m])
    c.plan(ints([0]), ints([ctx]), ints([m]), rows=m, max_len=total)
    kp, vp = fill(c, books, [0], [total], seed=8)
    q = torch.randn(m, heads, hd, device="cuda").to(c.dtype)
    want, lse = torch.empty_like(q), torch.empty(m, heads, device="cuda")
    c.attn(q, kp, vp, want, lse=lse)
    one, l1 = torch.empty_like(q), torch.empty_like(lse)
    for i in range(m):
        c.plan(ints([0]), ints([ctx + i]), ints([1]), rows=1)
        c.attn(q[i:i + 1], kp, vp, one[i:i + 1], lse=l1[i:i + 1])
    assert torch.equal(one, want) and torch.equal(l1, lse)
    # in pieces of unequal length
    r = 0
    while r < m:
        k = min(m - r, 7)
        c.plan(ints([0]), ints([ctx + r]), ints([k]), rows=k, max_new=k)
        c.attn(q[r:r + k], kp, vp, one[r:r + k])
        r += k
    assert torch.equal(one, want)
    # other pages, in the midst of other requests
    old = list(books.table[0])
    seq = list(range(1, others // 2)) + [0] + list(range(others // 2, others + 1))
    at = seq.index(0)
    ctxs, news = [ctx if s == 0 else s % 9 for s in seq], [m if s == 0 else 1 for s in seq]
    books.plan([0], [0], [0])
    c.plan(ints([0]), ints([0]), ints([0]), rows=0)
    books.plan(seq, ctxs, news)
    c.plan(ints(seq), ints(ctxs), ints(news), rows=m + others)
    assert books.table[0] != old
    kp2, vp2 = (torch.zeros_like(p).index_copy_(0, torch.tensor(books.table[0], device="cuda"), p[old]) for p in (kp, vp))
    q2 = torch.randn(m + others, heads, hd, device="cuda").to(c.dtype)
    q2[at:at + m] = q
    out = torch.empty_like(q2)
    c.attn(q2, kp2, vp2, out)
    assert c.status()[0] == m + others
    assert torch.equal(out[at:at + m], want)
    c.attn(q2, kp2, vp2, q2)  # in place
    assert torch.equal(q2, out)


@pytest.mark.parametrize("heads,kv,hd,page,ctx,m", [(32, 8, 128, 64, 900, 16), (24, 8, 64, 16, 505, 21), (8, 1, 128, 32, 250, 8),
                                                    (14, 2, 64, 16, 0, 9), (64, 1, 32, 16, 700, 1), (8, 2, 256, 64, 300, 16)])
def test_blocks_of_grouped_heads_at_the_limit(binding, heads, kv, hd, page, ctx, m):
    """Blocks of 64 / group tokens, the most whose rows' bits do not depend on the call."""
    assert (m + 1) * heads // kv > 64 >= m * heads // kv
    test_a_rows_bits_do_not_depend_on_the_call(binding, "bf16", heads, kv, hd, page, ctx, m)


@pytest.mark.parametrize("heads,kv,hd,m", [(32, 8, 128, 64), (8, 1, 64, 30), (64, 2, 32, 5)])
def test_a_longer_block_of_grouped_heads_in_steps(binding, heads, kv, hd, m):
    """A block above the limit, run in steps of 64 / group tokens beside other requests: the bits of its tokens one by one.
    As one chunk it has the long chunks' weights, one bf16 plane."""
    ctx, others, page, k = 700, 9, 32, 64 * kv // heads
    total, n = ctx + m, others + 1
    n_pages = -(-total // page) + others * -(-(400 + m) // page)
    g = torch.Generator(device="cuda").manual_seed(hd)
    x = torch.randn(m, heads + 2 * kv, hd, generator=g, device="cuda").bfloat16()
    first = [torch.randn(n_pages, kv, page, hd, generator=g, device="cuda").bfloat16() for _ in range(2)]

    def run(step, beside):
        c = make(binding, page=page, n_pages=n_pages, max_seqs=n, max_ctx=total, max_rows=m * n, heads=heads, kv=kv, hd=hd,
                 rope_base=10000.0)
        pools, out, r = [p.clone() for p in first], torch.empty(m, heads, hd, device="cuda").bfloat16(), 0
        c.plan(ints([0]), ints([ctx]), ints([0]), rows=0)  # the context: the first pages
        while r < m:
            j = min(step, m - r)
            new, ctxs = [j] + [step] * beside, [ctx + r] + [40 * b + r for b in range(beside)]
            y = torch.randn(sum(new), heads + 2 * kv, hd, generator=g, device="cuda").bfloat16()
            y[:j] = x[r:r + j]
            q, o = y[:, :heads], torch.empty(sum(new), heads, hd, device="cuda").bfloat16()
            c.plan(ints(list(range(1 + beside))), ints(ctxs), ints(new), rows=sum(new))
            c.append(q, y[:, heads:heads + kv], y[:, heads + kv:], q, *pools)
            c.attn(q, *pools, o)
            out[r:r + j] = o[:j]
            r += j
        assert c.status()[0] == sum(new)
        return out

    want = run(1, 0)
    assert torch.equal(run(k, 0), want) and torch.equal(run(k, others), want)
    # against the tokens: two half steps of the output and the half step of the weights, of values up to 6
    assert (run(m, 0).float() - want.float()).abs().max() <= 2.0**-8 * 3 * 6


@pytest.mark.parametrize("dtype,heads,kv,hd,page,n,hi,lo_ctx,hi_ctx,far", [
    ("bf16", 32, 32, 32, 64, 64, 16, 1000, 4000, 0), ("bf16", 64, 32, 32, 16, 48, 8, 200, 9000, 0),
    ("bf16", 32, 32, 32, 64, 101, 60, 800, 2500, 9000), ("bf16", 16, 16, 128, 64, 96, 1, 3000, 5000, 0),
    ("f32", 32, 32, 16, 32, 99, 40, 500, 2500, 9000)])
def test_full_plans_give_a_workgroup_several_spans(binding, dtype, heads, kv, hd, page, n, hi, lo_ctx, hi_ctx, far):
    """Row blocks whose spans of all key heads are above 16384: a workgroup takes several, one after another, the last
    one of a request fewer. The formula for some requests, and the bits of a plan of its own."""
    rng = random.Random(hd + n)
    new = [rng.randint(1, hi) for _ in range(n)]
    ctx = [rng.randint(lo_ctx, hi_ctx) for _ in range(n)]
    if far:  # a request of more than twice the mean keys, so that none is taken whole
        ctx[5], new[5] = far, hi
    total = [a + b for a, b in zip(ctx, new)]
    n_pages = sum(-(-t // page) for t in total)
    c = make(binding, page=page, n_pages=n_pages, max_seqs=n, max_ctx=max(total), max_rows=sum(new), heads=heads, kv=kv, hd=hd,
             dtype=dtype)
    rows = 16 if hd * (2 if dtype == "bf16" else 4) >= 512 else 32
    blocks = [-(-m * heads // kv // rows) for m in new]
    spans = [(t - 1) // 256 + 1 for t in total]
    units = sum(b * s for b, s in zip(blocks, spans))
    per = -(-units * kv // 16384)
    assert per > 1 and units * kv % 16384 and any(s % per for s in spans)
    g = torch.Generator(device="cuda").manual_seed(n)
    kp, vp = (torch.randn(c.pool_shape, generator=g, device="cuda").to(c.dtype) for _ in range(2))
    q = (torch.randn(sum(new), heads, hd, generator=g, device="cuda") * 1.5).to(c.dtype)
    out, lse = torch.empty_like(q), torch.empty(sum(new), heads, device="cuda")
    c.plan(ints(list(range(n))), ints(ctx), ints(new), rows=sum(new))
    took = int(c._ws[:64].view(torch.int32)[4])  # the plan's units: a word of the status block
    assert took == sum(b * -(-s // per) for b, s in zip(blocks, spans))
    c.attn(q, kp, vp, out, lse=lse)
    start = np.concatenate([[0], np.cumsum(new)])
    for s in (0, 5, n // 2, n - 1):
        c.plan(ints([s]), ints([ctx[s]]), ints([new[s]]), rows=new[s])
        qs, o, ls = q[start[s]:start[s + 1]], torch.empty_like(q[:new[s]]), torch.empty_like(lse[:new[s]])
        c.attn(qs, kp, vp, o, lse=ls)
        assert torch.equal(o, out[start[s]:start[s + 1]]) and torch.equal(ls, lse[start[s]:start[s + 1]])
        pages = c.block_table[s, :-(-total[s] // page)].long()
        k, v = (ref.gather(host(p[pages]), range(len(pages)), total[s]) for p in (kp, vp))
        for i in {0, new[s] - 1}:
            t = ctx[s] + i + 1
            want, wl, mag = ref.attend(host(qs[i:i + 1]), k[:, :t], v[:, :t], t - 1, hd ** -0.5)
            tol, tl = tolerance(c, host(qs[i:i + 1]), k[:, :t], want, wl, mag, hd ** -0.5, t)
            assert (np.abs(host(o[i]) - want[0]) <= tol[0]).all() and (np.abs(host(ls[i]) - wl[0]) <= tl[0]).all()


@pytest.mark.parametrize("new", [1, 130], ids=["token", "chunk"])
def test_offsets_past_32_bits(binding, new):
    """A request in the last pages of pools of more than 2^31 elements."""
    heads, hd, page, far = 32, 128, 256, 1 << 19
    n_pages = far // page + 4
    c = make(binding, page=page, n_pages=n_pages, max_seqs=2, max_ctx=far, max_rows=256, heads=heads, kv=heads, hd=hd)
    books = ref.Books(page, n_pages, 2)
    books.plan([0], [far], [0])
    c.plan(ints([0]), ints([far]), ints([0]), rows=0)
    ctx = 600
    books.plan([1], [ctx], [new])
    c.plan(ints([1]), ints([ctx]), ints([new]), rows=new)
    assert min(books.table[1]) * heads * page * hd >= 2**31
    pools = [torch.empty(c.pool_shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for p in pools:
        p[books.table[1]] = torch.randn(len(books.table[1]), *c.pool_shape[1:], device="cuda").bfloat16()
    k, v = (torch.randn(new, heads, hd, device="cuda").bfloat16() for _ in range(2))
    c.append(None, k, v, None, *pools)
    for i in (0, new - 1):
        t = ctx + i
        for p, x in zip(pools, (k, v)):
            assert torch.equal(p[books.table[1][t // page], :, t % page], x[i])
    q = torch.randn(new, heads, hd, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty(new, heads, device="cuda")
    c.attn(q, *pools, out, lse=lse)
    kh, vh = (ref.gather(host(p[books.table[1]]), range(len(books.table[1])), ctx + new) for p in pools)
    pick = [0, new - 1] if new > 1 else [0]
    for i in pick:
        want, wl, mag = ref.attend(host(q[i:i + 1]), kh[:, :ctx + i + 1], vh[:, :ctx + i + 1], ctx + i, hd ** -0.5)
        tol, _ = tolerance(c, host(q[i:i + 1]), kh[:, :ctx + i + 1], want, wl, mag, hd ** -0.5, ctx + i + 1)
        tol = tol + (2.0**-8 * mag if new > 64 else 0)  # a long chunk's weights
        assert (np.abs(host(out[i:i + 1]) - want) <= tol).all()


def joined(c):
    """Row blocks of the last plan whose spans are joined: those of requests that are split over several workgroups
    (word 9 of the status block, the first words of the cache's memory)."""
    return int(c._ws[:64].view(torch.int32)[9])


@pytest.mark.parametrize("heads,kv,chunk", [(1, 1, 200), (1, 1, 2000), (8, 2, 90)])
def test_a_long_fp32_chunk_leaves_the_others_their_split(binding, heads, kv, chunk):
    """Tokens and a block over long contexts are worked on by many workgroups also beside a chunk that has more
    partial states than the cache holds, wherever in the plan that is, with the bits of a plan of their own."""
    page, hd, n = 64, 32, 4
    seq, ctx, new = [3, 1, 0, 2], [5000, 9000, 3000, 4100], [1, chunk, 16, 1]
    total = [a + b for a, b in zip(ctx, new)]
    n_pages = sum(-(-t // page) for t in total)
    c = make(binding, page=page, n_pages=n_pages, max_seqs=n, max_ctx=max(total), max_rows=sum(new), heads=heads, kv=kv, hd=hd,
             dtype="f32")
    g = torch.Generator(device="cuda").manual_seed(chunk)
    pools = [torch.randn(c.pool_shape, generator=g, device="cuda") for _ in range(2)]
    q = torch.randn(sum(new), heads, hd, generator=g, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(sum(new), heads, device="cuda")
    c.plan(ints(seq), ints(ctx), ints(new), rows=sum(new))  # all pages are taken
    whole = joined(c)
    c.attn(q, *pools, out, lse=lse)
    few, r = 0, 0
    for s, a, m in zip(seq, ctx, new):
        c.plan(ints([s]), ints([a]), ints([m]), rows=m)
        few += joined(c) if m < chunk else 0
        o, ls = torch.empty_like(q[:m]), torch.empty_like(lse[:m])
        c.attn(q[r:r + m], *pools, o, lse=ls)
        assert torch.equal(o, out[r:r + m]) and torch.equal(ls, lse[r:r + m])
        pages = c.block_table[s, :-(-(a + m) // page)].cpu().numpy()
        k, v = (ref.gather(host(p), pages, a + m) for p in pools)
        for i in (0, m - 1):  # against the formula
            want, wl, mag = ref.attend(host(q[r + i:r + i + 1]), k[:, :a + i + 1], v[:, :a + i + 1], a + i, hd ** -0.5)
            tol, tl = tolerance(c, host(q[r + i:r + i + 1]), k[:, :a + i + 1], want, wl, mag, hd ** -0.5, a + i + 1)
            assert (np.abs(host(out[r + i]) - want[0]) <= tol[0]).all() and (np.abs(host(lse[r + i]) - wl[0]) <= tl[0]).all()
        r += m
    assert few >= 3 and whole >= few


# ---------------------------------------------------------------------------------- run together
class Layers:
    """Two attention layers with random projections, in fp32: what a decoder does around the operators."""

    def __init__(self, c, d, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        H, KV, hd = c.n_heads, c.n_kv_heads, c.head_dim
        self.c, self.wqkv = c, [torch.randn(d, (H + 2 * KV) * hd, generator=g, device="cuda") / d ** 0.5 for _ in range(2)]
        self.wo = [torch.randn(H * hd, d, generator=g, device="cuda") / (H * hd) ** 0.5 for _ in range(2)]
        self.pools = [[torch.full(c.pool_shape, float("nan"), device="cuda") for _ in range(2)] for _ in range(2)]

    def step(self, x):
        c = self.c
        H, KV, hd = c.n_heads, c.n_kv_heads, c.head_dim
        for wqkv, wo, (kp, vp) in zip(self.wqkv, self.wo, self.pools):
            y = x @ wqkv
            q, k, v = y[:, :H * hd], y[:, H * hd:(H + KV) * hd], y[:, (H + KV) * hd:]
            c.append(q, k, v, q, kp, vp)
            out = torch.empty(x.shape[0], H * hd, device="cuda")
            c.attn(q, kp, vp, out)
            x = x + out @ wo
        return x

    def plain(self, x, base):
        """One whole sequence in float64."""
        c, n = self.c, x.shape[0]
        H, KV, hd = c.n_heads, c.n_kv_heads, c.head_dim
        x = host(x)
        for wqkv, wo in zip(self.wqkv, self.wo):
            y = (x @ host(wqkv)).reshape(n, H + 2 * KV, hd)
            t = ref.rotate(y[:, :H + KV], range(n), base)
            o, _, _ = ref.attend(t[:, :H], t[:, H:].transpose(1, 0, 2), y[:, H + KV:].transpose(1, 0, 2), 0, hd ** -0.5)
            x = x + o.reshape(n, -1) @ host(wo)
        return x


def test_ragged_steps_with_rejected_tokens_and_ended_requests(binding):
    """Requests that come and go in blocks of ragged length, each step keeping a part of its block, as
    Jacobi decoding does: the kept rows are those of one pass over each whole sequence."""
    rng, base, d, slots = random.Random(2), 10000.0, 48, 5
    c = make(binding, page=16, n_pages=40, max_seqs=slots, max_ctx=200, max_rows=200, heads=6, kv=2, hd=32, dtype="f32",
             rope_base=base)
    net = Layers(c, d, 3)
    done, live = [], {}
    for step in range(30):
        for s in range(slots):
            if s not in live and rng.random() < 0.5:
                n = rng.randint(3, 120)
                live[s] = dict(x=torch.randn(n, d, device="cuda"), y=torch.empty(n, d, device="cuda"), ctx=0)
        seq = [s for s in live if rng.random() < 0.8]
        if not seq:
            continue
        rng.shuffle(seq)
        new = [min(rng.choice([0, 1, 8, 40]), live[s]["x"].shape[0] - live[s]["ctx"]) for s in seq]
        ctx = [live[s]["ctx"] for s in seq]
        c.plan(ints(seq), ints(ctx), ints(new), rows=sum(new), max_new=max(new))
        keep = [rng.randint(1, m) if m else 0 for m in new]
        # the tail of each block is a wrong guess
        x = [live[s]["x"][a:a + m].clone() for s, a, m in zip(seq, ctx, new)]
        for t, k in zip(x, keep):
            t[k:] = 1e3
        if sum(new):
            y = net.step(torch.cat(x))
            r = 0
            for s, m, k in zip(seq, new, keep):
                e = live[s]
                e["y"][e["ctx"]:e["ctx"] + k] = y[r:r + k]
                e["ctx"] += k
                r += m
        assert c.status()[0] == sum(new)
        over = [s for s in seq if live[s]["ctx"] == live[s]["x"].shape[0]]
        if over:
            c.plan(ints(over), ints([0] * len(over)), ints([0] * len(over)), rows=0)
            done += [live.pop(s) for s in over]
    assert len(done) == 7  # what this seed ends; the host alone decides it
    for e in done:
        want = net.plain(e["x"], base)
        # two layers of fp32 products of 48 and 192 terms and attention over 120 keys on values near 1
        np.testing.assert_allclose(host(e["y"]), want, rtol=0, atol=2e-4)


def test_captured_steps(binding):
    """A step captured once and replayed for other lengths, tokens and pages; two graphs on one cache;
    a replay behind a plan with other bounds does nothing and says so."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = make(binding, page=16, n_pages=60, max_seqs=3, max_ctx=900, max_rows=64, heads=4, kv=2, hd=64, rope_base=10000.0)
        pools = [torch.zeros(c.pool_shape, device="cuda").bfloat16() for _ in range(2)]
        seq, ctx, new = ints([0, 1, 2]), ints([0, 0, 0]), ints([0, 0, 0])
        x = torch.zeros(48, 8 * 64, device="cuda").bfloat16()
        q = torch.zeros(48, 4, 64, device="cuda").bfloat16()
        out = torch.zeros(2, 48, 4, 64, device="cuda").bfloat16()

        def step(rows, o):
            c.plan(seq, ctx, new, rows=rows, max_new=16, max_len=900)
            c.append(x[:, :256], x[:, 256:384], x[:, 384:], q, *pools)
            c.attn(q, *pools, o)

        step(48, out[0])
        side.synchronize()
        graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
        for g, rows, o in zip(graphs, (48, 40), out):
            with torch.cuda.graph(g, stream=side):
                step(rows, o)
        attn_only = torch.cuda.CUDAGraph()
        with torch.cuda.graph(attn_only, stream=side):
            c.attn(q, *pools, out[1])
        eager = torch.zeros_like(out[0])
        for i, (cs, ms) in enumerate([([0, 700, 30], [16, 1, 3]), ([16, 701, 33], [16, 16, 8]), ([5, 0, 600], [1, 0, 16]),
                                      ([880, 0, 0], [16, 0, 0]), ([0, 0, 0], [1, 1, 1])]):
            ctx.copy_(ints(cs))
            new.copy_(ints(ms))
            x.normal_()
            out.fill_(7)
            for which in (i % 2, 1 - i % 2):
                graphs[which].replay()
            assert c.status()[0] == sum(ms)
            side.synchronize()
            eager.fill_(7)
            step(48, eager)
            side.synchronize()
            assert torch.equal(out[0], eager) and torch.equal(out[1], eager)
        out.fill_(7)
        attn_only.replay()  # made for 40 rows, behind a plan for 48
        with pytest.raises(binding.CllmError, match="ERR_STATE"):
            c.status()
        assert (out == 7).all()
        c.plan(seq, ctx, new, rows=40, max_new=16, max_len=900)
        attn_only.replay()
        assert c.status()[0] == 3
        assert torch.equal(out[1][:3], eager[:3]) and (out[1][3:] == 7).all()
        side.synchronize()
        del graphs, attn_only


def test_a_captured_call_behind_plans_of_more_requests(binding):
    """Attention captured behind a plan of one request; the same bounds then hold many, whole or a long one among them."""
    side = torch.cuda.Stream()
    n, m, kv = 70, 20, 8
    with torch.cuda.stream(side):
        c = make(binding, page=16, n_pages=1400, max_seqs=n, max_ctx=3000, max_rows=n * m, heads=kv, kv=kv, hd=64)
        bounds = dict(rows=n * m, max_new=m, max_len=3000)
        pools = [torch.randn(c.pool_shape, device="cuda").bfloat16() for _ in range(2)]
        q = torch.randn(n * m, kv, 64, device="cuda").bfloat16()
        out, eager = torch.empty_like(q), torch.empty_like(q)
        c.plan(ints([0]), ints([100]), ints([m]), **bounds)
        c.attn(q, *pools, out)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.attn(q, *pools, out)
        for first in (100, 2900, 250):
            ctx = [first] + [90 + s for s in range(1, n)]
            c.plan(ints(list(range(n))), ints(ctx), ints([m] * n), **bounds)
            out.fill_(7)
            graph.replay()
            c.attn(q, *pools, eager)
            assert c.status()[0] == n * m
            assert torch.equal(out, eager) and (eager != 7).any()
        side.synchronize()
        del graph


def test_two_caches_side_by_side(binding):
    """Two caches on two streams: neither's partials or books are the other's."""
    got = []
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for run in range(2):
        caches = []
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                g = torch.Generator(device="cuda").manual_seed(i)
                c = make(binding, page=32, n_pages=80, max_seqs=1, max_ctx=2100, max_rows=4, heads=8, kv=8, hd=128)
                pools = [torch.randn(c.pool_shape, generator=g, device="cuda").bfloat16() for _ in range(2)]
                q = torch.randn(4, 8, 128, generator=g, device="cuda").bfloat16()
                c.plan(ints([0]), ints([2000 + i]), ints([4]), rows=4)
                caches.append((c, pools, q, torch.empty_like(q)))
        if run:
            torch.cuda.synchronize()
        for _ in range(20):
            for s, (c, pools, q, out) in zip(streams, caches):
                with torch.cuda.stream(s):
                    c.attn(q, *pools, out)
            if run:
                torch.cuda.synchronize()  # one after another
        torch.cuda.synchronize()
        got.append([x[3].clone() for x in caches])
        for c, *_ in caches:
            c.close()
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_cache_made_for_a_stream_that_is_not_current(binding):
    """stream= at creation: the calls are made with that stream current, and refused with any other. The memory of the
    books is told of that stream and no other (the default one has the address 0)."""
    side, default, got = torch.cuda.Stream(), torch.cuda.default_stream(), []
    for now, stream in ((default, None), (default, side), (side, default)):
        told, record = [], torch.Tensor.record_stream
        with torch.cuda.stream(now), pytest.MonkeyPatch.context() as patch:
            patch.setattr(torch.Tensor, "record_stream", lambda x, s: (told.append(s.cuda_stream), record(x, s)))
            c = make(binding, page=16, n_pages=30, max_seqs=2, max_ctx=200, max_rows=8, heads=4, kv=2, hd=64, rope_base=10000.0,
                     stream=None if stream is None else stream.cuda_stream)
            assert told == ([] if stream is None else [stream.cuda_stream])
            if stream is not None:
                with pytest.raises(ValueError, match="stream"):
                    c.plan(ints([0]), ints([0]), ints([1]), rows=1)
        with torch.cuda.stream(stream or default):
            g = torch.Generator(device="cuda").manual_seed(4)
            pools = [torch.randn(c.pool_shape, generator=g, device="cuda").bfloat16() for _ in range(2)]
            x, out = torch.randn(8, 8, 64, generator=g, device="cuda").bfloat16(), torch.empty(8, 4, 64, device="cuda").bfloat16()
            c.plan(ints([1, 0]), ints([150, 20]), ints([3, 5]), rows=8)
            c.append(x[:, :4], x[:, 4:6], x[:, 6:], x[:, :4], *pools)
            c.attn(x[:, :4], *pools, out)
            assert c.status() == (8, 30 - 10 - 2)
            got.append(out.clone())
            torch.cuda.current_stream().synchronize()
        c.close()
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])


def test_a_cache_that_ends_while_a_graph_is_captured(binding):
    """Closing a cache, or dropping it, waits for nothing: another cache's step can be in capture meanwhile."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        kw = dict(page=16, n_pages=30, max_seqs=2, max_ctx=200, max_rows=8, heads=4, kv=2, hd=64)
        c, old = make(binding, **kw), [make(binding, **kw) for _ in range(2)]
        pools = [torch.randn(c.pool_shape, device="cuda").bfloat16() for _ in range(2)]
        q = torch.randn(8, 4, 64, device="cuda").bfloat16()
        want, out = torch.empty_like(q), torch.empty_like(q)
        for x in [c] + old:
            x.plan(ints([0, 1]), ints([150, 20]), ints([3, 5]), rows=8)
            x.attn(q, *pools, want)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            old.pop().close()
            c.attn(q, *pools, out)
            old.pop()
        for _ in range(3):
            out.zero_()
            graph.replay()
            side.synchronize()
            assert torch.equal(out, want)
        del graph
