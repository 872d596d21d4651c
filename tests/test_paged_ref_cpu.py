"""The references of the paged KV cache's tests (tests/paged_ref.py), each against a second form of the same formula."""
import random

import numpy as np
import pytest

from tests import paged_ref as ref


@pytest.mark.parametrize("page,slots,seed", [(16, 1, 0), (16, 9, 1), (64, 40, 2)])
def test_books_own_every_page_once_and_undo_a_plan(page, slots, seed):
    rng = random.Random(seed)
    n_pages, length = 3 * slots + 2, [0] * slots
    books = ref.Books(page, n_pages, slots)
    for _ in range(40):
        seq = rng.sample(range(slots), rng.randint(1, slots))
        ctx = [rng.randint(0, length[s]) for s in seq]
        new = [rng.randint(0, 2 * page) for _ in seq]
        free, table = list(books.free), [list(t) for t in books.table]
        rows = books.plan(seq, ctx, new)
        if rows is None:
            assert books.free == free and books.table == table
            continue
        for s, c, m in zip(seq, ctx, new):
            length[s] = c + m
        assert sorted(books.free + sum(books.table, [])) == list(range(n_pages))
        assert [len(t) for t in books.table] == [-(-n // page) for n in length]
        assert [p for _, p in rows] == [p for c, m in zip(ctx, new) for p in range(c, c + m)]
        assert len({s for s, _ in rows}) == len(rows)  # no two rows in one slot of the pool
        kept = list(books.free), [list(t) for t in books.table]
        more = [length[s] + rng.randint(0, page) for s in seq]
        if books.plan(seq, more, [0] * len(seq)) is not None:
            books.plan(seq, [length[s] for s in seq], [0] * len(seq))
            assert (books.free, books.table) == kept


def test_rotate_is_a_complex_product():
    x, pos, base = np.random.default_rng(0).standard_normal((5, 3, 16)), [0, 1, 7, 1000, 2**20 - 1], 10000.0
    wave = np.exp(-np.log(base) * np.arange(8) / 8)
    z = (x[..., :8] + 1j * x[..., 8:]) * np.exp(1j * np.outer(pos, wave))[:, None]
    # both angles are rounded in float64: off by a few 2^-53 of 2^20
    np.testing.assert_allclose(ref.rotate(x, pos, base), np.concatenate([z.real, z.imag], -1), rtol=0, atol=2.0**-28)


@pytest.mark.parametrize("heads,kv,m,ctx", [(4, 4, 1, 0), (6, 2, 5, 9), (8, 1, 3, 40)])
def test_attend_is_a_masked_softmax(heads, kv, m, ctx):
    rng = np.random.default_rng(heads)
    q, k, v = rng.standard_normal((m, heads, 8)), rng.standard_normal((kv, ctx + m, 8)), rng.standard_normal((kv, ctx + m, 8))
    out, lse, mag = ref.attend(q, k, v, ctx, 0.3)
    kk, vv = np.repeat(k, heads // kv, 0), np.repeat(v, heads // kv, 0)
    e = np.exp(0.3 * np.einsum("mhd,htd->mht", q, kk)) * (np.arange(ctx + m) <= ctx + np.arange(m)[:, None])[:, None]
    np.testing.assert_allclose(lse, np.log(e.sum(-1)), rtol=1e-12, atol=1e-12)
    p = e / e.sum(-1, keepdims=True)
    np.testing.assert_allclose(out, np.einsum("mht,htd->mhd", p, vv), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(mag, np.einsum("mht,htd->mhd", p, np.abs(vv)), rtol=1e-12)


def test_gather_follows_the_pages():
    pool = np.arange(5 * 2 * 4 * 3).reshape(5, 2, 4, 3)
    x = ref.gather(pool, [3, 0], 6)
    assert x.shape == (2, 6, 3)
    for t in range(6):
        np.testing.assert_array_equal(x[:, t], pool[[3, 0][t // 4], :, t % 4])
