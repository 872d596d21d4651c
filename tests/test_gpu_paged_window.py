"""GPU tests of attention behind a window with sinks (binding.PagedCache.attn with window) against a plain reference in float64:
sizes and masks at the ends of pages, chunks, spans and tiles, values that are not finite in places that a row does not
see, bits that do not depend on the call, graphs, refusals. Tolerances are those of the attention without a window."""
import random

import numpy as np
import pytest

from tests import paged_ref as ref
from tests.test_gpu_paged import fill, host, ints, make, tolerance

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def binding():
    from paper_2403_00835_amd import binding as b
    return b


def seen(pos, window, sinks):
    t = np.arange(pos + 1)
    return t[(t > pos - window) | (t < sinks)]


def attend(q, k, v, ctx, scale, window, sinks):
    """(out, lse, sum p |v|) of rows q [m, H, hd] at positions ctx.. over k, v [KV, ctx + m, hd], row by row over what it sees."""
    m, H, hd = q.shape
    group = H // k.shape[0]
    out, lse, mag = np.empty((m, H, hd)), np.empty((m, H)), np.empty((m, H, hd))
    for i in range(m):
        at = seen(ctx + i, window, sinks)
        kk, vv = np.repeat(k[:, at], group, 0), np.repeat(v[:, at], group, 0)
        s = (kk @ q[i][:, :, None])[..., 0] * scale
        t = s.max(-1, keepdims=True)
        p = np.exp(s - t)
        lse[i] = (t + np.log(p.sum(-1, keepdims=True)))[:, 0]
        p /= p.sum(-1, keepdims=True)
        out[i], mag[i] = (p[:, None] @ vv)[:, 0], (p[:, None] @ np.abs(vv))[:, 0]
    return out, lse, mag


def hide(c, books, seq, ctx, new, window, sinks, pools):
    """NaN and infinities where no row of the step sees."""
    for s, a, m in zip(seq, ctx, new):
        if m == 0:
            continue
        gone = np.setdiff1d(np.arange(a + m), np.concatenate([seen(a, window, sinks), np.arange(a, a + m)]))
        for j, t in enumerate(gone):
            for pool in pools:
                pool[books.table[s][t // books.page], :, t % books.page] = (float("nan"), float("inf"), -float("inf"))[j % 3]


def check(c, books, seq, ctx, new, window, sinks, seed, scale=None, bounds=None, strided=False, rows=None):
    R, H, hd = sum(new), c.n_heads, c.head_dim
    total = [a + b for a, b in zip(ctx, new)]
    assert books.plan(seq, ctx, new) is not None
    c.plan(ints(seq), ints(ctx), ints(new), **{"rows": R + 1, **(bounds or {})})
    kp, vp = fill(c, books, seq, total, seed)
    hide(c, books, seq, ctx, new, window, sinks, (kp, vp))
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    q = (torch.randn(R + 1, H + (1 if strided else 0), hd, generator=g, device="cuda") * 1.5).to(c.dtype)[:, :H]
    out = torch.full((R + 1, H + (2 if strided else 0), hd), 3.0, device="cuda", dtype=c.dtype)[:, :H]
    lse = torch.full((R + 1, H), 3.0, device="cuda")
    c.attn(q, kp, vp, out, scale=scale, lse=lse, window=window, sinks=sinks)
    assert c.status()[0] == R
    sc = scale if scale is not None else hd ** -0.5
    qh, r = host(q), 0
    for s, a, m in zip(seq, ctx, new):
        if m == 0:
            continue
        pages = torch.tensor(books.table[s], device="cuda")
        k, v = (np.nan_to_num(ref.gather(host(p[pages]), range(len(pages)), a + m), nan=0.0, posinf=0.0, neginf=0.0) for p in (kp, vp))
        want, wl, mag = attend(qh[r:r + m], k, v, a, sc, window, sinks)
        tol, tl = tolerance(c, qh[r:r + m], k, want, wl, mag, sc, min(a + m, window + sinks))
        d, dl = np.abs(host(out[r:r + m]) - want), np.abs(host(lse[r:r + m]) - wl)
        assert (d <= tol).all(), f"request {s}: output off by {np.nanmax(d / tol)} of its bound, {np.isnan(d).sum()} NaN"
        assert (dl <= tl).all(), f"request {s}: lse off by {np.nanmax(dl / tl)} of its bound"
        r += m
    assert (out[R:] == 3).all() and (lse[R:] == 3).all()
    return q, kp, vp, out, lse


CASES = [  # dtype, heads, kv heads, head dim, page, contexts, new tokens, window, sinks
    ("bf16", 4, 4, 128, 64, [0], [1], 1, 0), ("bf16", 4, 4, 128, 64, [511], [1], 1, 0), ("bf16", 4, 4, 128, 64, [512, 1], [1, 1], 1, 1),
    ("bf16", 8, 2, 128, 16, [700, 3, 0, 64], [1, 1, 1, 1], 64, 4), ("bf16", 8, 2, 128, 16, [1700, 300], [1, 2], 257, 3),
    ("bf16", 4, 4, 128, 64, [2000], [1], 256, 0), ("bf16", 4, 4, 128, 64, [2047], [1], 512, 256), ("bf16", 2, 2, 128, 64, [2048], [1], 513, 257),
    ("bf16", 14, 2, 64, 32, [17, 0, 1300], [5, 64, 0], 33, 2), ("bf16", 2, 2, 128, 64, [1690], [16], 100, 0),
    ("bf16", 2, 2, 128, 128, [1100, 40], [32, 31], 300, 70), ("bf16", 2, 2, 128, 64, [1215], [64], 5, 1),
    ("bf16", 8, 1, 64, 16, [763, 62], [8, 3], 129, 64), ("bf16", 3, 1, 32, 256, [255, 1256], [2, 9], 1000, 30),
    ("bf16", 1, 1, 256, 32, [100, 700], [17, 1], 90, 5), ("bf16", 4, 2, 256, 16, [533], [32], 31, 400),
    ("bf16", 8, 2, 128, 64, [900], [65], 200, 4), ("bf16", 4, 2, 64, 16, [0, 1000], [300, 129], 100, 1),
    ("bf16", 7, 1, 128, 32, [333, 0], [77, 1], 1, 0), ("bf16", 4, 4, 32, 64, [20], [200], 63, 65),
    ("bf16", 2, 1, 256, 64, [65], [140], 64, 0), ("bf16", 16, 1, 128, 128, [5, 600, 90], [4, 5, 128], 40, 7),
    ("bf16", 1, 1, 128, 64, [0], [129], 128, 1), ("bf16", 32, 8, 128, 64, [1500], [40], 700, 130),
    ("bf16", 2, 2, 128, 16, [0, 3000], [640, 100], 500, 3), ("bf16", 8, 1, 32, 16, [2500, 10], [9, 1], 2000, 600),
    ("bf16", 6, 2, 256, 64, [1300, 0, 7], [30, 500, 2], 333, 9), ("bf16", 2, 2, 64, 64, [3000], [1], 4, 2900),
    ("bf16", 64, 1, 64, 16, [300, 0], [1, 3], 20, 20), ("f32", 2, 2, 64, 64, [900], [130], 70, 3),
    ("f32", 4, 4, 16, 16, [16], [8], 3, 1), ("f32", 12, 12, 64, 32, [5, 700, 301], [41, 3, 17], 101, 1),
    ("f32", 4, 1, 128, 64, [1030, 1], [30, 1], 600, 0), ("f32", 6, 2, 32, 16, [0, 15], [130, 1], 1, 200),
    ("f32", 2, 2, 128, 256, [1513], [70], 900, 258)]


@pytest.mark.parametrize("case", CASES, ids=["-".join(str(x) for x in a[:5]) + f"-ctx{a[5]}-new{a[6]}-w{a[7]}-s{a[8]}" for a in CASES])
def test_window(binding, case):
    dtype, heads, kv, hd, page, ctx, new, window, sinks = case
    n, total = len(new), [a + b for a, b in zip(ctx, new)]
    n_pages = sum(-(-t // page) for t in total) + 2
    c = make(binding, page=page, n_pages=n_pages, max_seqs=n + 2, max_ctx=max(max(total), window + 1), max_rows=sum(new) + 1, heads=heads,
             kv=kv, hd=hd, dtype=dtype)
    books, seq = ref.Books(page, n_pages, n + 2), list(range(n + 1, 1, -1))
    half = [t // 2 for t in total]  # pages interleaved: the requests grew in turn
    books.plan(seq, half, [0] * n)
    c.plan(ints(seq), ints(half), ints([0] * n), rows=0)
    check(c, books, seq, ctx, new, window, sinks, seed=hd + n)
    # the tightest bounds, strided rows, another scale; then in place: the same bits
    q, kp, vp, out, _ = check(c, books, seq, ctx, new, window, sinks, seed=hd, scale=-0.11, strided=True,
                              bounds=dict(max_new=max(new), max_len=max(total)))
    c.attn(q, kp, vp, q, scale=-0.11, window=window, sinks=sinks)
    assert torch.equal(q[:sum(new)], out[:sum(new)])


def run(c, q, kp, vp, **kw):
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    c.attn(q, kp, vp, out, lse=lse, **kw)
    return out, lse


SHAPES = [("bf16", 2, 2, 128, 64, 1000, 64), ("bf16", 8, 2, 64, 16, 505, 16), ("bf16", 4, 4, 256, 32, 300, 40), ("bf16", 24, 8, 32, 16, 900, 21),
          ("f32", 3, 3, 64, 32, 700, 45), ("f32", 8, 2, 16, 16, 250, 70), ("f32", 2, 1, 128, 64, 600, 9)]


@pytest.mark.parametrize("dtype,heads,kv,hd,page,ctx,m", SHAPES)
def test_a_rows_bits_do_not_depend_on_the_call(binding, dtype, heads, kv, hd, page, ctx, m):
    """Blocks of few rows, and fp32: a row's bits are those of a token of its own, in pieces, and beside other requests; behind
    a window that holds its whole past, and where the sinks do, those without one."""
    total, others = ctx + m, 9
    n_pages = -(-total // page) + others * -(-(50 + m) // page)
    c = make(binding, page=page, n_pages=n_pages, max_seqs=others + 1, max_ctx=total + 100, max_rows=m + others, heads=heads, kv=kv,
             hd=hd, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(hd)
    kp, vp = (torch.randn(c.pool_shape, generator=g, device="cuda").to(c.dtype) for _ in range(2))
    q = torch.randn(m, heads, hd, generator=g, device="cuda").to(c.dtype)
    for window, sinks in ((1, 0), (7, 3), (64, 64), (300, 4), (511, 0), (total - 1, 0), (total, 0), (5, total), (total + 50, 9)):
        kw = dict(window=window, sinks=sinks)
        c.plan(ints([0]), ints([ctx]), ints([m]), rows=m)
        want, lse = run(c, q, kp, vp, **kw)
        if window >= total or sinks >= total:
            full = run(c, q, kp, vp)
            assert torch.equal(want, full[0]) and torch.equal(lse, full[1])
        r = 0
        for k in [1] * 3 + [7] * m:
            k = min(k, m - r)
            if k == 0:
                break
            c.plan(ints([0]), ints([ctx + r]), ints([k]), rows=k, max_new=k)
            out, l1 = run(c, q[r:r + k], kp, vp, **kw)
            assert torch.equal(out, want[r:r + k]) and torch.equal(l1, lse[r:r + k])
            r += k
        seq = list(range(1, 5)) + [0] + list(range(5, others + 1))
        q2 = torch.randn(m + others, heads, hd, generator=g, device="cuda").to(c.dtype)
        q2[4:4 + m] = q
        c.plan(ints(seq), ints([ctx if s == 0 else s * 5 for s in seq]), ints([m if s == 0 else 1 for s in seq]), rows=m + others)
        out, l1 = run(c, q2, kp, vp, **kw)
        assert c.status()[0] == m + others
        assert torch.equal(out[4:4 + m], want) and torch.equal(l1[4:4 + m], lse)
        c.plan(ints(seq[:4] + seq[5:]), ints([0] * others), ints([0] * others), rows=0)


@pytest.mark.parametrize("heads,kv,hd,ctx,m", [(8, 1, 128, 700, 66), (2, 2, 64, 300, 140), (1, 1, 256, 0, 129), (4, 4, 32, 100, 300)])
def test_long_chunks_behind_a_window_of_everything(binding, heads, kv, hd, ctx, m):
    total = ctx + m
    c = make(binding, page=16, n_pages=-(-total // 16), max_seqs=1, max_ctx=total + 10, max_rows=m, heads=heads, kv=kv, hd=hd)
    kp, vp = (torch.randn(c.pool_shape, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(m, heads, hd, device="cuda").bfloat16()
    c.plan(ints([0]), ints([ctx]), ints([m]), rows=m)
    want, lse = run(c, q, kp, vp)
    for kw in (dict(window=total), dict(window=total + 5, sinks=3), dict(window=total + 10), dict(window=2**31 - 1, sinks=2**31 - 1)):
        out, l1 = run(c, q, kp, vp, **kw)
        assert torch.equal(out, want) and torch.equal(l1, lse)


@pytest.mark.parametrize("heads,kv,hd,page,n,lo,hi", [(8, 8, 128, 64, 68, 17, 64), (16, 8, 64, 16, 68, 9, 32), (32, 16, 32, 32, 36, 9, 32),
                                                      (4, 4, 256, 64, 132, 17, 40)])
@pytest.mark.parametrize("window,sinks", [(100, 4), (300, 0), (1, 70)])
def test_many_requests_of_a_block_each(binding, heads, kv, hd, page, n, lo, hi, window, sinks):
    """Enough blocks to be taken whole, one request of a token, one of none and one long chunk among them: the formula for some,
    and the bits of a plan of their own."""
    rng = random.Random(hd)
    new, ctx = [rng.randint(lo, hi) for _ in range(n)], [rng.randint(250, 700) for _ in range(n)]
    new[3], new[7], new[11], ctx[12], ctx[13] = 1, 0, 70, 0, 256 - new[13]
    total = [a + b for a, b in zip(ctx, new)]
    n_pages = sum(-(-t // page) for t in total)
    c = make(binding, page=page, n_pages=n_pages, max_seqs=n, max_ctx=max(total), max_rows=sum(new), heads=heads, kv=kv, hd=hd)
    g = torch.Generator(device="cuda").manual_seed(n)
    kp, vp = (torch.randn(c.pool_shape, generator=g, device="cuda").bfloat16() for _ in range(2))
    q = (torch.randn(sum(new), heads, hd, generator=g, device="cuda") * 1.5).bfloat16()
    c.plan(ints(list(range(n))), ints(ctx), ints(new), rows=sum(new))
    kw = dict(window=window, sinks=sinks)
    out, lse = run(c, q, kp, vp, **kw)
    assert c.status()[0] == sum(new)
    start = np.concatenate([[0], np.cumsum(new)])
    for s in (0, 3, 12, 13, 14, n - 1):
        at = slice(start[s], start[s + 1])
        c.plan(ints([s]), ints([ctx[s]]), ints([new[s]]), rows=new[s])
        o, ls = run(c, q[at], kp, vp, **kw)
        assert torch.equal(o, out[at]) and torch.equal(ls, lse[at])
        pages = c.block_table[s, :-(-total[s] // page)].long()
        k, v = (ref.gather(host(p[pages]), range(len(pages)), total[s]) for p in (kp, vp))
        want, wl, mag = attend(host(q[at]), k, v, ctx[s], hd ** -0.5, window, sinks)
        tol, tl = tolerance(c, host(q[at]), k, want, wl, mag, hd ** -0.5, min(total[s], window + sinks))
        assert (np.abs(host(o) - want) <= tol).all() and (np.abs(host(ls) - wl) <= tl).all()


@pytest.mark.parametrize("dtype,heads,kv,hd,page,n,hi", [
    ("bf16", 32, 8, 128, 16, 64, 1), ("bf16", 32, 4, 64, 64, 40, 2), ("bf16", 8, 8, 128, 32, 30, 64), ("bf16", 6, 2, 32, 16, 70, 9),
    ("bf16", 16, 8, 256, 64, 40, 16), ("bf16", 64, 64, 64, 16, 9, 20), ("f32", 4, 4, 64, 16, 60, 30), ("f32", 6, 2, 16, 16, 90, 9),
    ("f32", 8, 1, 128, 64, 30, 90), ("f32", 3, 3, 32, 32, 70, 70)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 4), (200, 70), (600, 300)])
def test_few_rows_give_the_same_bits_alone_and_beside_others(binding, dtype, heads, kv, hd, page, n, hi, window, sinks):
    """Requests of few rows (fp32: any) with bounds that say so, with values that are not finite where some rows see them: many of
    them, which a workgroup each takes, give the bits that each has alone, where spans share it; and so in a graph of one plan
    behind another."""
    rng = random.Random(n + window)
    new, ctx = [rng.randint(1, hi) for _ in range(n)], [rng.randint(0, 900) for _ in range(n)]
    new[2], new[4], ctx[4], ctx[5] = 0, hi, 0, 256
    total = [a + b for a, b in zip(ctx, new)]
    n_pages = sum(-(-t // page) for t in total)
    R, bounds = sum(new), dict(max_new=hi, max_len=max(total))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = make(binding, page=page, n_pages=n_pages, max_seqs=n, max_ctx=max(total), max_rows=R, heads=heads, kv=kv, hd=hd, dtype=dtype)
        g = torch.Generator(device="cuda").manual_seed(n)
        kp, vp = (torch.randn(c.pool_shape, generator=g, device="cuda").to(c.dtype) for _ in range(2))
        q = (torch.randn(R, heads, hd, generator=g, device="cuda") * 1.5).to(c.dtype)
        plan = lambda k, rows: c.plan(ints(list(range(k))), ints(ctx[:k]), ints(new[:k]), rows=rows, **bounds)
        plan(n, R)
        for s in (3, n - 1):  # (some rows see it, and the first ones of a block may not)
            vp[int(c.block_table[s, max(ctx[s] - window // 2, 0) // page]), :, 3, 7 + s % 2] = float("nan") if s == 3 else float("inf")
        kw = dict(window=window, sinks=sinks)
        out, lse = run(c, q, kp, vp, **kw)
        assert c.status()[0] == R
        start = np.concatenate([[0], np.cumsum(new)])
        for s in range(0, n, 1 if n < 32 else 3):
            at = slice(start[s], start[s + 1])
            c.plan(ints([s]), ints([ctx[s]]), ints([new[s]]), rows=new[s], max_len=max(total))
            o, ls = run(c, q[at], kp, vp, **kw)
            assert torch.equal(o.view(torch.uint8), out[at].view(torch.uint8)) and torch.equal(ls, lse[at])
        plan(n // 2, R)
        again = torch.empty_like(q)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.attn(q, kp, vp, again, **kw)
        for k in (n // 2, n, 1, n):
            plan(k, R)
            again.fill_(7)
            graph.replay()
            assert c.status()[0] == start[k]
            assert torch.equal(again[:start[k]].view(torch.uint8), out[:start[k]].view(torch.uint8)) and (again[start[k]:] == 7).all()
        del graph


@pytest.mark.parametrize("dtype,heads,kv,hd,ctx,m,n", [
    ("bf16", 4, 4, 128, 500, 40, 1), ("bf16", 8, 2, 64, 70, 16, 1), ("bf16", 8, 8, 64, 500, 40, 66), ("bf16", 4, 2, 128, 120, 90, 1),
    ("bf16", 1, 1, 256, 300, 130, 1), ("bf16", 2, 2, 32, 0, 200, 1), ("f32", 2, 2, 64, 60, 30, 1), ("f32", 2, 1, 16, 300, 40, 1)])
@pytest.mark.parametrize("window,sinks", [(20, 3), (64, 0), (9, 90), (130, 1)])
def test_values_that_are_not_finite(binding, dtype, heads, kv, hd, ctx, m, n, window, sinks):
    """NaN and infinities in single values of tokens that some rows see and others do not, because the token is behind them, or
    in front of their window: each row's output is what the tokens that it sees make of it, its other columns keep their bits."""
    page, total = 16, ctx + m
    n_pages = -(-total // page) * n
    c = make(binding, page=page, n_pages=n_pages, max_seqs=n, max_ctx=total, max_rows=m * n, heads=heads, kv=kv, hd=hd, dtype=dtype)
    c.plan(ints(list(range(n))), ints([ctx] * n), ints([m] * n), rows=m * n, max_new=m)
    g = torch.Generator(device="cuda").manual_seed(hd)
    kp, vp = (torch.randn(c.pool_shape, generator=g, device="cuda").to(c.dtype) for _ in range(2))
    q = torch.randn(m * n, heads, hd, generator=g, device="cuda").to(c.dtype)
    kw = dict(window=window, sinks=sinks)
    want = run(c, q, kp, vp, **kw)[0]
    assert torch.isfinite(want).all()
    inf, nan, lo = float("inf"), float("nan"), max(0, ctx - window)
    # before the first row's window, in it, and among the new tokens; two of opposite signs a window apart and close
    put = [(0, 1, inf), (max(sinks - 1, 0), 2, -inf), (sinks, 3, nan), (lo, 4, inf), (lo + 1, 5, -inf), (lo + 1, 6, nan),
           (ctx + m // 3, 7, inf), (ctx + m // 3, 8, nan), (ctx + m // 2, 9, inf), (ctx + m // 2 + 2, 9, -inf), (lo + 2, 10, inf),
           (min(lo + 2 + window, total - 1), 10, -inf), (total - 1, 11, -inf)]
    put = [(t, d, x) for t, d, x in put if t < total]
    s = n - 1
    for t, d, x in put:
        vp[int(c.block_table[s, t // page]), :, t % page, d] = x
    out = run(c, q, kp, vp, **kw)[0]
    assert torch.equal(out[:-m], want[:-m])
    out, want = out[-m:], want[-m:]
    cols = {d for _, d, _ in put}
    keep = [d for d in range(hd) if d not in cols]
    assert torch.equal(out[..., keep], want[..., keep])
    for d in cols:
        for i in range(m):
            sum_ = sum(x for t, e, x in put if e == d and t in seen(ctx + i, window, sinks))
            got = out[i, :, d].float()
            if sum_ == 0:
                assert torch.equal(out[i, :, d], want[i, :, d])
            else:
                assert torch.isnan(got).all() if sum_ != sum_ else (got == sum_).all()


@pytest.mark.parametrize("dtype,m", [("bf16", 1), ("bf16", 100), ("f32", 20)])
def test_keys_that_are_not_finite_and_unseen(binding, dtype, m):
    ctx, page = 400, 32
    c = make(binding, page=page, n_pages=-(-(ctx + m) // page), max_seqs=1, max_ctx=ctx + m, max_rows=m, heads=4, kv=2, hd=64, dtype=dtype)
    c.plan(ints([0]), ints([ctx]), ints([m]), rows=m)
    kp, vp = (torch.randn(c.pool_shape, device="cuda").to(c.dtype) for _ in range(2))
    q = torch.randn(m, 4, 64, device="cuda").to(c.dtype)
    want = run(c, q, kp, vp, window=50, sinks=2)[0]
    for t in (2, 100, ctx - 50):  # the last one: the first that no row sees
        kp[int(c.block_table[0, t // page]), :, t % page] = float("nan")
    assert torch.equal(run(c, q, kp, vp, window=50, sinks=2)[0], want)
    kp[int(c.block_table[0, (ctx - 49) // page]), :, (ctx - 49) % page] = float("nan")  # the first row's first
    out = run(c, q, kp, vp, window=50, sinks=2)[0]
    assert torch.isnan(out[0]).all() and torch.equal(out[1:], want[1:])


@pytest.mark.parametrize("new", [1, 130], ids=["token", "chunk"])
def test_offsets_past_32_bits_and_a_long_past(binding, new):
    """A request of half a million tokens in pools of more than 2^31 elements: only its window is read."""
    heads, hd, page, far, window, sinks = 32, 128, 256, 1 << 19, 700, 5
    n_pages = far // page + 4
    c = make(binding, page=page, n_pages=n_pages, max_seqs=1, max_ctx=far + 1000, max_rows=256, heads=heads, kv=heads, hd=hd)
    ctx = far + 100
    c.plan(ints([0]), ints([ctx]), ints([new]), rows=new)
    table = c.block_table[0].cpu().numpy()
    assert int(table[(ctx + new - 1) // page]) * heads * page * hd >= 2**31
    pools = [torch.empty(c.pool_shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    first, last = (ctx - window) // page, (ctx + new - 1) // page
    used = [0] + list(range(first, last + 1))
    for p in pools:
        p[table[used]] = torch.randn(len(used), *c.pool_shape[1:], device="cuda").bfloat16()
    q = torch.randn(new, heads, hd, device="cuda").bfloat16()
    out, lse = run(c, q, *pools, window=window, sinks=sinks)
    assert c.status()[0] == new
    near = [host(p[table[used]]).transpose(1, 0, 2, 3).reshape(heads, -1, hd) for p in pools]
    for i in {0, new - 1}:
        at = seen(ctx + i, window, sinks)
        at = np.where(at < page, at, at - first * page + page)
        kk, vv = (x[:, at] for x in near)
        # every token of the gathered ones is seen: as a context of its own
        want, wl, mag = attend(host(q[i:i + 1]), kk, vv, kk.shape[1] - 1, hd ** -0.5, 10**6, 0)
        tol, tl = tolerance(c, host(q[i:i + 1]), kk, want, wl, mag, hd ** -0.5, kk.shape[1])
        tol = tol + (2.0**-8 * mag if new > 64 else 0)  # a long chunk's weights
        assert (np.abs(host(out[i:i + 1]) - want) <= tol).all() and (np.abs(host(lse[i:i + 1]) - wl) <= tl).all()


def test_captured_behind_plans_of_more_requests(binding):
    """Attention captured behind a plan of one request; the same bounds then hold many, whole or a long one among them; behind a
    plan with other bounds a replay does nothing and says so."""
    side = torch.cuda.Stream()
    n, m, kv = 70, 20, 8
    kw = dict(window=333, sinks=4)
    with torch.cuda.stream(side):
        c = make(binding, page=16, n_pages=1400, max_seqs=n, max_ctx=3000, max_rows=n * m, heads=kv, kv=kv, hd=64)
        bounds = dict(rows=n * m, max_new=m, max_len=3000)
        pools = [torch.randn(c.pool_shape, device="cuda").bfloat16() for _ in range(2)]
        q = torch.randn(n * m, kv, 64, device="cuda").bfloat16()
        out, eager = torch.empty_like(q), torch.empty_like(q)
        c.plan(ints([0]), ints([100]), ints([m]), **bounds)
        c.attn(q, *pools, out, **kw)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.attn(q, *pools, out, **kw)
        for first in (100, 2900, 250):
            ctx = [first] + [90 + s for s in range(1, n)]
            c.plan(ints(list(range(n))), ints(ctx), ints([m] * n), **bounds)
            out.fill_(7)
            graph.replay()
            c.attn(q, *pools, eager, **kw)
            assert c.status()[0] == n * m
            assert torch.equal(out, eager) and (eager != 7).any()
        c.plan(ints([0]), ints([100]), ints([m]), **{**bounds, "max_len": 2999})
        out.fill_(7)
        graph.replay()
        with pytest.raises(binding.CllmError, match="ERR_STATE"):
            c.status()
        assert (out == 7).all()
        side.synchronize()
        del graph


def test_refusals(binding):
    c = make(binding)
    q = torch.zeros(8, 4, 64, device="cuda").bfloat16()
    pools = [torch.zeros(c.pool_shape, device="cuda").bfloat16() for _ in range(2)]
    with pytest.raises(binding.CllmError, match="ERR_STATE"):
        c.attn(q, *pools, q, window=4)  # no plan yet
    one = ints([1])
    c.plan(one, one, one, rows=8)
    for bad in (dict(window=0), dict(window=-1), dict(window=2**31), dict(window=4, sinks=-1), dict(window=4, sinks=2**31), dict(sinks=1)):
        with pytest.raises(ValueError, match="sinks"):
            c.attn(q, *pools, q, **bad)
    L, args = binding.lib(), (c.h, q.data_ptr(), 256, *[x.data_ptr() for x in pools], 0.0)
    for window, sinks in ((0, 0), (-1, 0), (1, -1)):
        assert L.cllm_paged_attn_window(*args, window, sinks, q.data_ptr(), 256, None) == 1
    assert L.cllm_paged_attn_window(*args, 4, 0, None, 256, None) == 1
    c.plan(one, one, one, rows=64)
    c.plan(ints([9]), one, one, rows=8)  # refused on the device: attention does nothing
    q.fill_(5)
    c.attn(q, *pools, q, window=4)
    assert (q == 5).all()
