"""Plain references of the paged KV cache's operators (test infrastructure): the pool's books as lists,
rotary positions and attention in float64 on the host."""
import numpy as np


class Books:
    """The page pool: a stack of free pages (page 0 on top at first) and each slot's pages."""

    def __init__(self, page, n_pages, max_seqs):
        self.page = page
        self.free = list(range(n_pages - 1, -1, -1))
        self.table = [[] for _ in range(max_seqs)]

    def need(self, tokens):
        return -(-tokens // self.page)

    def plan(self, seq, ctx, new):
        """Returns rows [(slot in the pool, position)] or None where the plan is refused for pages."""
        total = [c + m for c, m in zip(ctx, new)]
        back = sum(max(0, len(self.table[s]) - self.need(t)) for s, t in zip(seq, total))
        take = sum(max(0, self.need(t) - len(self.table[s])) for s, t in zip(seq, total))
        if take > len(self.free) + back:
            return None
        for s, t in reversed(list(zip(seq, total))):
            while len(self.table[s]) > self.need(t):
                self.free.append(self.table[s].pop())
        for s, t in zip(seq, total):
            while len(self.table[s]) < self.need(t):
                self.table[s].append(self.free.pop())
        rows = []
        for s, c, m in zip(seq, ctx, new):
            rows += [(self.table[s][p // self.page] * self.page + p % self.page, p) for p in range(c, c + m)]
        return rows


def rotate(x, pos, base):
    """Rotate-half of rows x [R, heads, hd] at positions pos, in float64."""
    x = np.asarray(x, np.float64)
    h2 = x.shape[-1] // 2
    ang = np.asarray(pos, np.float64)[:, None] * base ** (-2.0 * np.arange(h2) / x.shape[-1])
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., :h2], x[..., h2:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def gather(pool, pages, tokens):
    """Tokens [0, tokens) of a request: pool [pages, kv heads, page, hd] -> [kv heads, tokens, hd]."""
    x = np.asarray(pool[pages], np.float64).transpose(1, 0, 2, 3)
    return x.reshape(x.shape[0], -1, x.shape[-1])[:, :tokens]


def attend(q, k, v, ctx, scale):
    """Chunk rows q [m, H, hd] at positions ctx.. over k, v [KV, ctx + m, hd]: (out, lse, weighted |v|)
    in float64, each row over its own positions only. The third is sum p |v|, the size that rounding
    errors of the weights scale with."""
    q = np.asarray(q, np.float64)
    m, H, hd = q.shape
    group = H // k.shape[0]
    out, lse, mag = np.empty((m, H, hd)), np.empty((m, H)), np.empty((m, H, hd))
    with np.errstate(all="ignore"):
        for i in range(m):
            for h in range(H):
                kk, vv = k[h // group, :ctx + i + 1], v[h // group, :ctx + i + 1]
                s = kk @ q[i, h] * scale
                t = s.max()
                p = np.exp(s - t)
                lse[i, h] = t + np.log(p.sum())
                p = p / p.sum()
                out[i, h] = (p[:, None] * vv).sum(0)
                mag[i, h] = (p[:, None] * np.abs(vv)).sum(0)
    return out, lse, mag
