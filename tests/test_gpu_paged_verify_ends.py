"""GPU tests of PagedCache.verify at the ends of what a call may be: for more requests than the last plan has (row_start None), as a
program that verifies for all of its slots does, behind a plan of more requests, whose starts the array still holds; for
requests of very many rows. Results are whole numbers and have to be equal to those of tests/verify_ref.py."""
import random

import numpy as np
import pytest

from tests import verify_ref as ref
from tests.test_gpu_paged import ints, make
from tests.test_gpu_paged_verify import f64, place, problem

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

VOCAB = 700
PLANS = {8: [[1] * 8, [4, 4], [7], [2, 0, 3], [0, 0, 8]],  # max_seqs: new tokens of one plan after another
         200: [[1] * 200, [60, 0, 130], [199], [3] * 66, [1, 2] * 20, [0] * 150 + [5, 6]]}


@pytest.fixture(scope="module")
def binding():
    from paper_2403_00835_amd import binding as b
    return b


def rows_of(rng, new, n, rows, with_draft):
    """A problem of the plan's requests, with no tokens for the others and rows of nobody behind them."""
    start, tokens, x, draft, temperature, au, su = problem(rng, new + [0] * (n - len(new)), VOCAB, with_draft)
    rest = rows - len(tokens)
    temperature = [(0.0, 0.4, 1.0, 3.0)[(b + len(new)) % 4] for b in range(n)]  # neighbours' differ
    x = np.concatenate([x, np.zeros((rest, VOCAB))])
    draft = None if draft is None else np.concatenate([draft, np.ones((rest, VOCAB))])
    return start, tokens + [0] * rest, x, draft, temperature, au + [0.5] * rest, su


@pytest.mark.parametrize("n", list(PLANS))
@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("captured", [False, True])
def test_more_requests_than_the_last_plans(binding, n, with_draft, captured):
    """n up to 64 and above, eager and captured once; greedy requests beside others."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = make(binding, n_pages=4 * n, max_seqs=n, max_rows=n)
        rng = random.Random(n + with_draft)
        logits, dl = (torch.zeros(n, VOCAB, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        tok, tp, a_u, s_u = ints([0] * n), torch.zeros(n, device="cuda"), f64([0.0] * n), f64([0.0] * n)
        accepted, following = ints([9] * n), ints([9] * n)
        ws = torch.zeros(c.verify_workspace_bytes(n, VOCAB, with_draft), dtype=torch.uint8, device="cuda")

        def step():
            c.verify(tok, logits, accepted, following, tp, a_u, s_u, draft_logits=dl if with_draft else None, workspace=ws)

        c.plan(ints(list(range(n))), ints([3] * n), ints([1] * n), rows=n)
        step()
        side.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        for new in PLANS[n] + PLANS[n][::-1]:
            start, tokens, x, draft, temperature, au, su = rows_of(rng, new, n, n, with_draft)
            for dst, src in ((logits, x), (dl, draft), (tok, tokens), (tp, temperature), (a_u, au), (s_u, su)):
                if src is not None:
                    dst.copy_(torch.tensor(src))
            ws.fill_(0xff)  # statistics that the call does not write are NaN
            accepted.fill_(9), following.fill_(9)
            c.plan(ints(list(range(len(new)))), ints([3] * len(new)), ints(new), rows=n)
            graph.replay() if captured else step()
            assert c.status()[0] == sum(new)
            want = ref.verify(start, tokens, logits.double().cpu().numpy(), dl.double().cpu().numpy() if with_draft else None, temperature,
                              au, su)
            assert accepted.tolist() == want[0] and following.tolist() == want[1]
        c.plan(ints([0, 0]), ints([3, 3]), ints([1, 1]), rows=n)  # refused: nobody has rows
        graph.replay() if captured else step()
        assert accepted.tolist() == [0] * n and following.tolist() == [-1] * n
        side.synchronize()
        if captured:
            del graph


def test_a_request_of_more_rows_than_31_bits_of_threads(binding):
    """16 threads decide on a row: 2^27 rows and some, all of which stand, as the drafts' weights are above 0; the last row's token
    is drawn from the statistics that were kept for its place."""
    rows, vocab = 2 ** 27 + 70, 3
    c = make(binding)
    logits = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    logits[-1] = torch.tensor([0.0, 4.0, 2.0])
    p = ref.law([0.0, 4.0, 2.0], 1.0)
    start, tokens, zeros = ints([0, 0, rows]), ints([0]).expand(rows).contiguous(), f64([0.0]).expand(rows).contiguous()
    accepted, following = ints([9, 9]), ints([9, 9])
    for u in (0.5, 0.99):
        c.verify(tokens, logits, accepted, following, torch.ones(2, device="cuda"), zeros, f64([0.5, u]), row_start=start)
        assert accepted.tolist() == [0, rows] and following.tolist() == [-1, ref.draw(p, u)]
