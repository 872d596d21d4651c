"""The paged cache's operators run together as a decoder makes its steps: plan, append with norms and a rotary form, attention
behind a window, verification, whose accepted counts and tokens (on the device) are the next step's lengths and first
tokens. Two layers with random weights around them, in fp32; the reference is the whole sequence in float64."""
import numpy as np
import pytest

from tests import verify_ref as vref
from tests.test_gpu_paged import host, ints, make
from tests.test_gpu_paged_forms import angles, norm, turn
from tests.test_gpu_paged_window import attend

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

H, KV, HD, D, V, LAYERS = 6, 2, 32, 48, 97, 2
WINDOW, SINKS, EPS = 9, 2, 1e-5
FORM = dict(layout="interleaved", dim=20, scaling="linear", factor=2.0)


@pytest.fixture(scope="module")
def binding():
    from paper_2403_00835_amd import binding as b
    return b


class Decoder:
    """The cache, the weights and the state of its requests: tokens [request, position], contexts and pending tokens."""

    def __init__(self, binding, n, length, rows):
        self.c = make(binding, page=16, n_pages=n * (length // 16 + 2), max_seqs=n, max_ctx=length + 16, max_rows=rows, heads=H, kv=KV, hd=HD,
                      dtype="f32", rope_base=10000.0)
        self.c.rotary(**FORM)
        g = torch.Generator(device="cuda").manual_seed(11)

        def w(*s):
            return torch.randn(*s, generator=g, device="cuda") / s[0] ** 0.5

        self.emb, self.head = w(V, D) * V ** 0.5, w(D, V) * 2
        self.qkv, self.o = [w(D, (H + 2 * KV) * HD) for _ in range(LAYERS)], [w(H * HD, D) for _ in range(LAYERS)]
        self.gains = [[1 + 0.3 * torch.randn(HD, generator=g, device="cuda") for _ in range(2)] for _ in range(LAYERS)]
        self.pools = [[torch.full(self.c.pool_shape, float("nan"), device="cuda") for _ in range(2)] for _ in range(LAYERS)]

    def rows(self, tokens):
        """LM-head input rows of a planned step's tokens."""
        x = self.emb[tokens.long()]
        for qkv, o, (qg, kg), (kp, vp) in zip(self.qkv, self.o, self.gains, self.pools):
            y = x @ qkv
            q, k, v = y[:, :H * HD], y[:, H * HD:(H + KV) * HD], y[:, (H + KV) * HD:]
            self.c.append(q, k, v, q, kp, vp, q_gain=qg, k_gain=kg, eps=EPS)
            out = torch.empty(x.shape[0], H * HD, device="cuda")
            self.c.attn(q, kp, vp, out, window=WINDOW, sinks=SINKS)
            x = x + out @ o
        return x

    def plain(self, tokens):
        """Logits of a whole sequence in float64."""
        n = len(tokens)
        x = host(self.emb)[tokens]
        for qkv, o, (qg, kg) in zip(self.qkv, self.o, self.gains):
            y = (x @ host(qkv)).reshape(n, H + 2 * KV, HD)
            theta = angles(FORM["dim"], scaling="linear", factor=2.0)
            q = turn(norm(y[:, :H], host(qg), EPS), range(n), theta, "interleaved")[0]
            k = turn(norm(y[:, H:H + KV], host(kg), EPS), range(n), theta, "interleaved")[0]
            a, _, _ = attend(q, k.transpose(1, 0, 2), y[:, H + KV:].transpose(1, 0, 2), 0, HD ** -0.5, WINDOW, SINKS)
            x = x + a.reshape(n, -1) @ host(o)
        return x @ host(self.head)


def greedy(net, prompt, count):
    """The next `count` tokens in float64, and the smallest lead of one of them over the second best."""
    tokens, lead = list(prompt), np.inf
    for _ in range(count):
        z = net.plain(tokens)[-1]
        best = np.sort(z)[-2:]
        lead = min(lead, best[1] - best[0])
        tokens.append(int(z.argmax()))
    return tokens[len(prompt):], lead


@pytest.mark.parametrize("captured", [False, True], ids=["eager", "graph"])
def test_blocks_of_guesses_give_the_greedy_tokens(binding, captured):
    """Ragged prompts, then blocks of a pending token and guesses (the predictions of the block before, as Jacobi decoding has them):
    greedy verification keeps what one token at a time would have given."""
    n, m, count = 4, 6, 24
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        rng = np.random.default_rng(3)
        prompts = [[int(t) for t in rng.integers(0, V, k)] for k in (5, 17, 1, 30)]
        net = Decoder(binding, n, 30 + count + m, 64)
        c, seq = net.c, ints(list(range(n)))
        # prompts: only the last row's logits of each are formed
        lens = [len(p) for p in prompts]
        ctx, new = ints([0] * n), ints(lens)
        c.plan(seq, ctx, new, rows=64, max_new=30)
        x = net.rows(torch.cat([ints(p) for p in prompts] + [ints([0] * (64 - sum(lens)))]))
        last = torch.tensor(np.cumsum(lens) - 1, device="cuda")
        accepted, pending = ints([0] * n), ints([0] * n)
        zero, one = torch.zeros(n, device="cuda"), ints(list(range(n + 1)))
        u = torch.full((n * m,), 0.5, dtype=torch.float64, device="cuda")
        c.verify(ints([0] * n), (x[last] @ net.head), accepted, pending, zero, u, u, row_start=one)
        assert accepted.tolist() == [1] * n
        ctx.add_(new)
        new.fill_(m)
        block = torch.zeros(n, m, dtype=torch.int32, device="cuda")
        kept = torch.full((n, count + m + 1), -1, dtype=torch.int32, device="cuda")
        kept[:, 0] = pending
        at = torch.zeros(n, 1, dtype=torch.long, device="cuda")
        col = torch.arange(m, device="cuda")
        ws = torch.empty(c.verify_workspace_bytes(n * m, V, False), dtype=torch.uint8, device="cuda")

        def step():
            block[:, 0] = pending
            c.plan(seq, ctx, new, rows=n * m, max_new=m)
            logits = net.rows(block.view(-1)) @ net.head
            c.verify(block.view(-1), logits, accepted, pending, zero, u, u, workspace=ws)
            # row i's prediction is the token behind block[:, i]; what stands is committed, the rest are the next guesses
            pred = logits.view(n, m, V).argmax(-1).int()
            slot = (at + 1 + col).clamp(max=kept.shape[1] - 1)
            kept.scatter_(1, slot, torch.where(col < accepted[:, None] - 1, block.gather(1, (col + 1).clamp(max=m - 1).expand(n, m)),
                                               torch.where(col == accepted[:, None] - 1, pending[:, None], kept.gather(1, slot))))
            block.copy_(pred.gather(1, (accepted[:, None].long() - 1 + col).clamp(max=m - 1)))
            ctx.add_(accepted)
            at.add_(accepted[:, None])

        steps = 0
        if captured:
            step()
            steps = 1
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step()
        while int(at.min()) + 1 < count:
            graph.replay() if captured else step()
            steps += 1
            assert c.status()[0] == n * m
            assert int(accepted.min()) >= 1 and int(accepted.max()) <= m
            if int(at.max()) + m >= kept.shape[1] - 1:
                break
        got = kept.cpu().numpy()
        side.synchronize()
        if captured:
            del graph
    ends = at[:, 0].tolist()
    assert sum(ends) > steps * n  # guesses stood
    for b in range(n):
        want, lead = greedy(net, prompts[b], min(ends[b] + 1, count))
        # fp32 of two layers: logits off by some 1e-5; no two best are as close
        assert lead > 1e-3
        assert got[b, :len(want)].tolist() == want


def test_sampled_steps_beside_prompts(binding):
    """Requests at different temperatures, one whose prompt comes in two chunks beside the others' blocks: logits against float64, and
    each step's verification against the reference on the logits that it was given."""
    n = 3
    rng = np.random.default_rng(8)
    net = Decoder(binding, n, 120, 64)
    c, temperature = net.c, [1.0, 0.0, 0.6]
    history = [[int(t) for t in rng.integers(0, V, k)] for k in (4, 50, 9)]
    done, pending = [0, 0, 0], [None] * n
    for step in range(12):
        new, tokens = [], []
        for b in range(n):
            if pending[b] is None:
                part = history[b][done[b]:done[b] + 28]
            else:  # the pending token and random guesses
                part = [pending[b]] + [int(t) for t in rng.integers(0, V, rng.integers(0, 4))]
            new.append(len(part))
            tokens.append(part)
        R = sum(new)
        c.plan(ints([2, 0, 1]), ints([done[b] for b in (2, 0, 1)]), ints([new[b] for b in (2, 0, 1)]), rows=64)
        order = (2, 0, 1)
        flat = [t for b in order for t in tokens[b]]
        x = net.rows(ints(flat + [0] * (64 - R)))
        assert c.status()[0] == R
        # logits of the rows that decide: the last of a prompt's chunk, all of a block
        first = np.concatenate([[0], np.cumsum([new[b] for b in order])])
        pick = [list(range(first[i + 1] - 1 if pending[b] is None else first[i], first[i + 1])) for i, b in enumerate(order)]
        logits = x[torch.tensor(sum(pick, []), device="cuda")] @ net.head
        start = [0] + [int(k) for k in np.cumsum([len(p) for p in pick])]
        drafts = [flat[r] for p in pick for r in p]
        au, su = rng.random(start[-1]), rng.random(n)
        accepted, following = ints([0] * n), ints([0] * n)
        c.verify(ints(drafts), logits, accepted, following, torch.tensor([temperature[b] for b in order], device="cuda"),
                 torch.tensor(au, device="cuda"), torch.tensor(su, device="cuda"), row_start=ints(start))
        want = vref.verify(start, drafts, host(logits), None, [temperature[b] for b in order], au, su)
        assert (accepted.tolist(), following.tolist()) == tuple(want)
        z = host(logits)
        for i, b in enumerate(order):
            whole = net.plain(history[b][:done[b]] + tokens[b] if pending[b] is None else history[b] + tokens[b])
            # fp32 products of 48 and 192 terms around attention over 11 tokens, values near 1, logits of some units
            np.testing.assert_allclose(z[start[i]:start[i + 1]], whole[len(whole) - len(pick[i]):], rtol=0, atol=1e-3)
            if pending[b] is None:
                done[b] += new[b]
                if done[b] == len(history[b]):
                    pending[b] = want[1][i]
            else:
                history[b] += tokens[b][:want[0][i]]
                done[b] += want[0][i]
                pending[b] = want[1][i]
            assert done[b] <= len(history[b])
    assert all(p is not None for p in pending)
