"""GPU tests of the verification of drafted tokens (binding.PagedCache.verify) against the plain reference of
tests/verify_ref.py. Results are whole numbers and have to be equal: sums in 64 bits on both sides put a draw to another token
with a probability of some 2^-50 V."""
import random

import numpy as np
import pytest

from tests import verify_ref as ref
from tests.test_gpu_paged import ints, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def binding():
    from paper_2403_00835_amd import binding as b
    return b


@pytest.fixture(scope="module")
def cache(binding):
    return make(binding, max_seqs=1024)


def f64(v):
    return torch.tensor(v, dtype=torch.float64, device="cuda")


def run(c, start, tokens, logits, draft, temperature, accept_u, sample_u, **kw):
    n = len(temperature)
    accepted, following = ints([77] * (n + 1)), ints([77] * (n + 1))
    c.verify(ints(tokens), logits, accepted[:n], following[:n], torch.tensor(temperature, dtype=torch.float32, device="cuda"),
             f64(accept_u), f64(sample_u), **{"row_start": ints(start), "draft_logits": draft, **kw})
    assert accepted[n] == 77 and following[n] == 77
    return accepted[:n].tolist(), following[:n].tolist()


def check(c, start, tokens, logits, draft, temperature, accept_u, sample_u, **kw):
    got = run(c, start, tokens, logits, draft, temperature, accept_u, sample_u, **kw)
    want = ref.verify(start, tokens, logits.double().cpu().numpy(), None if draft is None else draft.double().cpu().numpy(), temperature,
                      accept_u, sample_u)
    assert got == tuple(want)
    return got


def place(x, dtype, pad, shift):
    """Rows of x in a wider array, from element `shift` on."""
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), device="cuda").to(dtype)
    wide[:, shift:shift + x.shape[1]] = torch.tensor(x, device="cuda").to(dtype)
    return wide[:, shift:shift + x.shape[1]]


def problem(rng, new, vocab, with_draft, close=0.7):
    """Logits with a favoured token a row; drafts of the draft's distribution or mostly favoured."""
    g = np.random.default_rng(rng.randint(0, 2**31))
    start = [0] + list(np.cumsum(new))
    R, n = start[-1], len(new)
    x = g.standard_normal((R, vocab)) * 1.5
    liked = g.integers(0, vocab, R)
    x[np.arange(R), liked] += g.uniform(3, 12, R)
    draft = x + g.standard_normal((R, vocab)) * close if with_draft else None
    temperature = [rng.choice([0.0, 0.3, 1.0, 1.0, 2.5]) for _ in range(n)]
    tokens = [int(t) for t in g.integers(0, vocab, R)]
    for b in range(n):
        for r in range(start[b], start[b + 1] - 1):
            if with_draft:
                tokens[r + 1] = ref.draw(ref.law(draft[r], temperature[b]), g.random())
            elif g.random() < 0.8:
                tokens[r + 1] = int(liked[r])
    return [int(s) for s in start], tokens, x, draft, temperature, list(g.random(R)), list(g.random(n))


SHAPES = [  # rows of the requests, vocabulary, padding and first element of a row
    ([1], 1, 0, 0), ([3, 1], 1, 3, 1), ([5], 2, 0, 0), ([2, 0, 4, 1], 7, 0, 0), ([1] * 30, 100, 0, 0), ([9, 1, 0, 17], 513, 5, 3), ([5], 4095, 1, 1),
    ([4, 4], 4096, 0, 0), ([4, 3], 4097, 0, 0), ([2, 5], 8192, 8, 0), ([6, 1, 2], 32000, 0, 0), ([3, 2], 70001, 0, 0), ([40, 70, 33], 300, 0, 0),
    ([1, 2] * 50, 33, 2, 1), ([2], 300007, 9, 5)]


@pytest.mark.parametrize("shape", SHAPES, ids=range(len(SHAPES)))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("with_draft", [False, True])
def test_verify(cache, shape, dtype, with_draft):
    new, vocab, pad, shift = shape
    rng = random.Random(vocab * 2 + with_draft)
    for _ in range(2 if vocab > 20000 else 6):
        start, tokens, x, draft, *rest = problem(rng, new, vocab, with_draft)
        check(cache, start, tokens, place(x, dtype, pad, shift), None if draft is None else place(draft, dtype, pad + 1, shift), *rest)


def test_many_requests_and_long_ones(cache):
    """As many requests as a cache has slots, some of none; a request of more rows than the waves of a workgroup, all standing."""
    rng = random.Random(5)
    start, tokens, x, draft, *rest = problem(rng, [rng.choice([0, 1, 1, 2, 5]) for _ in range(1024)], 40, True)
    check(cache, start, tokens, place(x, torch.float32, 0, 0), place(draft, torch.float32, 0, 0), *rest)
    start, tokens, x, draft, temperature, au, su = problem(rng, [1, 100, 3], 50, False)
    x[:, :] -= 30
    for r in range(1, 104):
        x[r - 1, tokens[r]] = 30
    a, _ = check(cache, start, tokens, place(x, torch.bfloat16, 0, 0), None, temperature, au, su)
    assert a == [1, 100, 3]


@pytest.mark.parametrize("stop", [0, 15, 16, 18, 19])
@pytest.mark.parametrize("with_draft", [False, True])
def test_where_a_long_request_over_many_chunks_stops(cache, stop, with_draft):
    """The row of any wave, in its first or its second turn, or the last row, with more chunks than a wave has lanes."""
    rng = random.Random(stop)
    start, tokens, x, draft, _, au, su = problem(rng, [2, 20, 1], 140000, with_draft)
    for r in range(2, 21):  # drafts that stand, up to the row
        x[r, tokens[r + 1]] = 25.0 if r < 2 + stop else -25.0
    for low in (None, 139999, 3):  # the refused draft is anywhere, or in the last chunk, or in the first
        if low is not None and stop < 19:
            x[2 + stop, tokens[3 + stop]] = 0.0
            tokens[3 + stop] = low
            x[2 + stop, low] = 1.0
            au[2 + stop] = 1 - 2.0 ** -40
        a, _ = check(cache, start, tokens, place(x, torch.float32, 0, 0), None if draft is None else place(draft, torch.float32, 0, 0),
                     [0.8, 1.0, 1.0], au, su)
        assert a[1] == stop + 1 or with_draft


@pytest.mark.parametrize("vocab", [5000, 32768])
@pytest.mark.parametrize("with_draft", [False, True])
def test_where_a_longer_request_over_few_chunks_stops(cache, vocab, with_draft):
    """Rows of a wave's four, of any wave and any turn, greedy and not."""
    rng = random.Random(vocab)
    start, tokens, x, draft, _, au, su = problem(rng, [1, 150, 2], vocab, with_draft)
    base = x.copy()
    for stop in (0, 1, 31, 32, 63, 64, 67, 130, 148, 149):
        x[:] = base
        for r in range(1, 150):
            x[r, tokens[r + 1]] = 25.0 if r < 1 + stop else -25.0
        for t in (0.0, 0.7):
            a, _ = check(cache, start, tokens, place(x, torch.bfloat16, 0, 0), None if draft is None else place(draft, torch.bfloat16, 0, 0),
                         [1.0, t, 0.0], au, su)
            assert a[1] == stop + 1 or with_draft and t


def test_the_drawn_tokens_have_the_targets_law(cache):
    """1024 requests of two rows at a time, all of one p and q: the first token that stands or is drawn is distributed as p, within five
    standard deviations of each count."""
    g = np.random.default_rng(3)
    V, n, times = 9, 1024, 40
    x, y = g.standard_normal((1, V)) * 1.3, g.standard_normal((1, V)) * 1.3
    p, q = ref.law(np.float32(x[0]), 1.0), ref.law(np.float32(y[0]), 1.0)
    logits, draft = (place(np.repeat(z, 2 * n, 0), torch.float32, 0, 0) for z in (x, y))
    count = np.zeros(V)
    start = list(range(0, 2 * n + 1, 2))
    for _ in range(times):
        drafts = g.choice(V, n, p=q)
        tokens = np.zeros(2 * n, int)
        tokens[1::2] = drafts
        a, t = run(cache, start, list(tokens), logits, draft, [1.0] * n, list(g.random(2 * n)), list(g.random(n)))
        count += np.bincount(np.where(np.array(a) == 2, drafts, np.array(t)), minlength=V)
    N = n * times
    assert (np.abs(count - N * p) <= 5 * np.sqrt(N * p * (1 - p))).all()


def test_greedy_is_the_acceptance_of_a_jacobi_block(cache):
    """Temperature 0: 1 + the leading guesses that are the predictions before them, ties to the lowest index, whatever the numbers."""
    g = np.random.default_rng(1)
    x = g.integers(-3, 3, (64, 5000)).astype(float)  # many ties
    best = x.argmax(1)
    for keep in (0, 1, 7, 15):
        tokens = g.integers(0, 5000, 64)
        for b in range(4):
            tokens[16 * b + 1:16 * b + 1 + keep] = best[16 * b:16 * b + keep]
            if keep < 15:
                tokens[16 * b + 1 + keep] = (best[16 * b + keep] + 1) % 5000
        for draft in (None, place(g.standard_normal((64, 5000)), torch.bfloat16, 0, 0)):
            a, t = check(cache, [0, 16, 32, 48, 64], list(tokens), place(x, torch.bfloat16, 0, 0), draft, [0.0] * 4, [0.999] * 64, [0.5] * 4)
            assert a == [keep + 1] * 4 and t == [best[16 * b + keep] for b in range(4)]


def test_numbers_at_the_ends(cache):
    """Equal weights, whose running sums are exact: every border falls to the token behind it; numbers outside [0, 1)."""
    V = 8192
    x = np.full((1, V), -np.inf)
    x[0, 5::8] = 2.5  # 1024 tokens of weight 1
    logits = place(x, torch.float32, 0, 0)
    for u, want in ((0.0, 0), (-0.0, 0), (-3.0, 0), (float("nan"), 0), (1 / 1024, 1), (np.nextafter(1 / 1024, 0), 0), (0.5, 512), (512.5 / 1024, 512),
                    (1023 / 1024, 1023), (np.nextafter(1, 0), 1023), (1.0, 1023), (float("inf"), 1023)):
        assert check(cache, [0, 1], [0], logits, None, [0.8], [0.0], [u]) == ([1], [5 + 8 * want])
    # the refused draft is taken out, the acceptance is strict
    two = place(np.repeat(x, 2, 0), torch.float32, 0, 0)
    for u, want in ((1 / 1024, 1), (np.nextafter(1 / 1024, 0), 2), (0.0, 2), (float("nan"), 1)):
        a, t = check(cache, [0, 2], [0, 13], two, None, [1.0], [u, 0.0], [1 / 1023])
        assert a == [want] and (t == [5 + 8 * 2] if want == 1 else t == [13])
    assert check(cache, [0, 2], [0, 12], two, None, [1.0], [0.0, 0.0], [0.0])[0] == [1]  # weight 0: u 1 < 0 does not hold


def test_masked_tokens_are_never_drawn(cache):
    g = np.random.default_rng(8)
    x = np.full((256, 9000), -np.inf)
    for r in range(256):
        x[r, g.choice(9000, 3, replace=False)] = g.standard_normal(3)
    tokens = list(g.integers(0, 9000, 256))
    _, t = check(cache, list(range(0, 257, 2)), tokens, place(x, torch.float32, 0, 0), None, [1.0] * 128, list(g.random(256)), list(g.random(128)))
    # a refused draft is the only token of its row that may be drawn from nothing left: here each has three
    assert all(np.isfinite(x[2 * b:2 * b + 2, t[b]]).any() for b in range(128))


def test_the_same_distribution_takes_every_draft(cache):
    g = np.random.default_rng(2)
    x = g.standard_normal((64, 3001)) * 3
    logits = place(x, torch.bfloat16, 0, 0)
    tokens = list(g.integers(0, 3001, 64))
    a, _ = check(cache, [0, 64], tokens, logits, logits.clone(), [0.7], [np.nextafter(1, 0)] * 64, [0.3])
    assert a == [64]


def test_a_rest_of_nothing_is_drawn_from_p(cache):
    """A refusal (by a number above 1) where p and q are the same, or p has its draft alone."""
    x = np.array([[1.0, 2, 3], [0, 0, 0]])
    logits = place(x, torch.float32, 0, 0)
    for u in (0.01, 0.2, 0.9):
        check(cache, [0, 2], [0, 1], logits, logits, [1.0], [5.0, 0], [u])
    alone = place(np.array([[-np.inf, 2.0, -np.inf], [0, 0, 0]]), torch.float32, 0, 0)
    assert check(cache, [0, 2], [0, 1], alone, None, [1.0], [5.0, 0], [0.5]) == ([1], [1])


def test_rows_without_a_distribution(cache):
    inf, nan = float("inf"), float("nan")
    g = np.random.default_rng(4)
    for V in (10, 5000):
        for at, value, t in ((3, nan, 1.0), (3, inf, 1.0), (None, None, 1.0), (3, nan, 0.0), (3, inf, 0.0), (None, None, 0.0), (V - 1, nan, 2.0)):
            for row in range(3):
                x = g.standard_normal((6, V))
                if at is None:
                    x[row] = -inf
                else:
                    x[row, at] = value
                tokens = [0] + [int(v) for v in x[:5].argmax(1)]
                tokens[3] = 0
                for r in range(2):
                    tokens[r + 1] = int(np.nan_to_num(x[r], nan=-9).argmax())
                a, tok = check(cache, [0, 3, 6], tokens, place(x, torch.float32, 0, 0), None, [t, t], [0.0] * 6, [0.4] * 2)
                assert a[0] == row + 1 and tok[0] == -1 and tok[1] >= 0
    x = place(g.standard_normal((3, 20)), torch.float32, 0, 0)
    for t in (-1.0, inf, nan, -inf):
        assert check(cache, [0, 3], [0, 1, 2], x, None, [t], [0.0] * 3, [0.4]) == ([1], [-1])
    for t in (1e-45, 1e-38, 3e38):  # the ends of the temperatures
        check(cache, [0, 3], [0, 1, 2], x, None, [t], [0.0] * 3, [0.4])
    # a draft's row without one counts as no draft logits; a draft that is no token does not stand
    y = g.standard_normal((3, 20))
    y[0, 4] = nan
    for draft in (place(y, torch.float32, 0, 0), None):
        for u in (0.0, 0.3, 0.9):
            for tokens in ([0, 1, 2], [0, -1, 2], [0, 20, 2], [0, 2**31 - 1, 1], [0, -2**31, 1]):
                check(cache, [0, 3], tokens, x, draft, [1.0], [u] * 3, [0.6])


def test_far_logits(cache):
    """Logits up to the ends of their type, and weights that fall below 2^-1000."""
    for dtype, big in ((torch.float32, 3e38), (torch.bfloat16, 3.3e38)):
        x = np.array([[big, -big, 0, big], [-big, -big, -big, -3e38], [1000, 300, 999, -1e30], [0, -690, -700, -800]])
        for u in (0.0, 0.3, 0.75, 0.999999):
            check(cache, [0, 1, 2, 3, 4], [0] * 4, place(x, dtype, 0, 0), None, [1.0, 0.5, 1.0, 1.0], [0.5] * 4, [u] * 4)


def test_chunks_far_apart(cache):
    """Parts of a long row at very different heights: weights of one of them are all that counts, wherever the number falls, and
    sums relative to different logits are joined."""
    g = np.random.default_rng(12)
    V = 150000  # more chunks of any size up to 2048 than a wave has lanes
    base = g.standard_normal((1, V))
    for heights, t in (((0, -2000, 3000), 1.0), ((-5000, -5000, -9000), 1.0), ((650, 600, -700), 1.0), ((0, 0, 5000), 0.3), ((-620, 0, 620), 1.0),
                       ((1e4, 1e4 + 3, 1e4 - 3), 2.0)):
        x = base.copy()
        for i, h in enumerate(heights):
            x[0, i * 50000:(i + 1) * 50000] += h
        x[0, 70000:74096] = -np.inf  # a masked stretch
        for u in (0.0, 1e-9, 0.4, 0.9, np.nextafter(1, 0), 1.0):
            a, tok = check(cache, [0, 1], [0], place(x, torch.float32, 0, 0), None, [t], [0.0], [u])
        two = np.repeat(x, 2, 0)
        for draft in (int(x[0].argmax()), 5, 70001, 120000):
            for u in (0.0, 0.2, 0.999):
                check(cache, [0, 2], [0, draft], place(two, torch.float32, 0, 0), None, [t], [u, 0], [0.37])
                check(cache, [0, 2], [0, draft], place(two, torch.float32, 0, 0), place(np.roll(two, 3, 1), torch.float32, 0, 0), [t], [u, 0], [0.37])


def test_rows_of_nobody(cache):
    """row_start that leaves the rows' bounds, or falls: those requests have nothing, the others what they have alone."""
    g = np.random.default_rng(9)
    x, tokens = place(g.standard_normal((8, 60)), torch.float32, 0, 0), [int(v) for v in g.integers(0, 60, 8)]
    au, su = list(g.random(8)), list(g.random(3))
    for start in ([0, 3, 8, 9], [0, 0, 0, 0], [2, 5, 5, 6], [-1, 3, 6, 8], [8, 9, 2**31 - 1, 2**31 - 1], [0, 8, 8, 8]):
        check(cache, start, tokens, x, None, [1.0] * 3, au, su)
    assert run(cache, [5, 4, 3, 2], tokens, x, None, [1.0] * 3, au, su) == ([0] * 3, [-1] * 3)
    none = torch.zeros(0, 60, device="cuda")
    assert run(cache, [0, 0, 0], [], none, None, [1.0] * 2, [], [0.5] * 2) == ([0, 0], [-1, -1])


def test_the_last_plans_rows(binding):
    c = make(binding, max_seqs=4, n_pages=20)
    g = np.random.default_rng(6)
    x = place(g.standard_normal((12, 300)), torch.bfloat16, 0, 0)
    tokens, au, su = [int(v) for v in g.integers(0, 300, 12)], list(g.random(12)), list(g.random(3))
    with pytest.raises(binding.CllmError, match="ERR_STATE"):
        run(c, [0], tokens, x, None, [1.0] * 3, au, su, row_start=None)
    new = [5, 0, 4]
    c.plan(ints([2, 0, 3]), ints([7, 0, 30]), ints(new), rows=12)
    got = run(c, [0], tokens, x, None, [1.0] * 3, au, su, row_start=None)
    want = ref.verify([0, 5, 5, 9], tokens, x.double().cpu().numpy(), None, [1.0] * 3, au, su)
    assert got == tuple(want)
    # more requests than the plan's; then a plan that is refused: nobody has rows
    got = run(c, [0], tokens, x, None, [1.0] * 4, au, su + [0.5], row_start=None)
    assert got == (want[0] + [0], want[1] + [-1])
    c.plan(ints([2, 2, 3]), ints([7, 0, 30]), ints(new), rows=12)
    assert run(c, [0], tokens, x, None, [1.0] * 3, au, su, row_start=None) == ([0] * 3, [-1] * 3)


def test_offsets_past_32_bits(cache):
    """Rows of a stride that takes the last of them past 2^32 bytes."""
    V, stride, R = 1000, (1 << 30) + 1, 4
    flat = torch.empty((R - 1) * stride + V, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((R, V), (stride, 1))
    g = np.random.default_rng(2)
    x.copy_(torch.tensor(g.standard_normal((R, V)) * 2, device="cuda"))
    tokens = [0] + [int(v) for v in x[:3].float().argmax(1)]
    for draft in (None, x):
        check(cache, [0, R], tokens, x, draft, [0.5], [0.01] * R, [0.7])


def test_captured(binding):
    """Captured with a workspace of its own and with one of the caller's, shared by two graphs on the stream; every replay against the
    eager call, with eager work between."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = make(binding, max_seqs=8)
        rng = random.Random(0)
        new, V = [3, 1, 5, 0, 2], 9001
        start, tokens, x, draft, temperature, au, su = problem(rng, new, V, True)
        logits, dl = place(x, torch.bfloat16, 0, 0), place(draft, torch.bfloat16, 0, 0)
        tok, st, tp, a_u, s_u = ints(tokens), ints(start), torch.tensor(temperature, device="cuda"), f64(au), f64(su)
        out = [[ints([9] * 5), ints([9] * 5)] for _ in range(3)]
        ws = torch.empty(binding.PagedCache.verify_workspace_bytes(11, V, True), dtype=torch.uint8, device="cuda")

        def step(o, **kw):
            c.verify(tok, logits, *o, tp, a_u, s_u, row_start=st, draft_logits=dl, **kw)

        step(out[0])
        side.synchronize()
        graphs = []
        for o, kw in zip(out, ({}, dict(workspace=ws), dict(workspace=ws))):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                step(o, **kw)
        seen = set()
        for i in range(6):
            start, tokens, x, draft, temperature, au, su = problem(rng, new, V, True)
            for dst, src in ((logits, x), (dl, draft), (tok, tokens), (tp, temperature), (a_u, au), (s_u, su)):
                dst.copy_(torch.tensor(src))
            for o in out:
                o[0].fill_(9), o[1].fill_(9)
            for k in (i % 3, (i + 1) % 3, (i + 2) % 3):
                graphs[k].replay()
            eager = [ints([9] * 5), ints([9] * 5)]
            step(eager, workspace=ws)
            want = ref.verify(start, tokens, logits.double().cpu().numpy(), dl.double().cpu().numpy(), temperature, au, su)
            assert [y.tolist() for y in eager] == list(want)
            for o in out:
                assert torch.equal(o[0], eager[0]) and torch.equal(o[1], eager[1])
            seen.add(tuple(want[0]))
        assert len(seen) > 1
        side.synchronize()
        del graphs


def test_refusals(binding, cache):
    c, V = cache, 64
    x = torch.zeros(4, V, device="cuda")
    i4, d4, one = ints([0] * 4), f64([0.0] * 4), torch.ones(1, device="cuda")
    ws = torch.empty(1024, dtype=torch.uint8, device="cuda")
    L = binding.lib()
    good = dict(n=1, row_start=i4.data_ptr(), rows=4, tokens=i4.data_ptr(), dtype=0, vocab=V, logits=x.data_ptr(), stride=V, draft=None,
                draft_stride=0, temperature=one.data_ptr(), accept_u=d4.data_ptr(), sample_u=d4.data_ptr(), accepted=i4.data_ptr(),
                next_token=i4.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=1024)
    assert L.cllm_paged_verify(c.h, *good.values()) == 0
    hostmem = np.zeros(4096, np.float64)
    bad = [dict(n=0), dict(n=1025), dict(rows=-1), dict(vocab=0), dict(dtype=2), dict(stride=V - 1), dict(stride=(1 << 40) + 1),
           dict(draft=x.data_ptr(), draft_stride=V - 1), dict(draft=x.data_ptr() + 2, draft_stride=V), dict(logits=x.data_ptr() + 1),
           dict(accept_u=d4.data_ptr() + 4), dict(workspace=ws.data_ptr() + 128)]
    bad += [{k: v} for k in ("tokens", "logits", "temperature", "accept_u", "sample_u", "accepted", "next_token", "workspace")
            for v in (None, hostmem.ctypes.data // 256 * 256 + 256)]
    bad += [dict(row_start=hostmem.ctypes.data)]
    for kw in bad:
        assert L.cllm_paged_verify(c.h, *{**good, **kw}.values()) == 1, kw
    for kw in (dict(workspace_bytes=63), dict(draft=x.data_ptr(), draft_stride=V, workspace_bytes=159), dict(rows=2**30)):
        assert L.cllm_paged_verify(c.h, *{**good, **kw}.values()) == 3, kw
    with torch.cuda.stream(torch.cuda.Stream()):
        with pytest.raises(ValueError, match="stream"):
            run(c, [0, 4], [0] * 4, x, None, [1.0], [0.0] * 4, [0.0])
    shut = make(binding)
    shut.close()
    with pytest.raises(ValueError, match="closed"):
        run(shut, [0, 4], [0] * 4, x, None, [1.0], [0.0] * 4, [0.0])
