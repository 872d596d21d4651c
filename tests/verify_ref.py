"""Plain reference of the verification of drafted tokens (test infrastructure): request by request and row by row, in float64."""
import numpy as np


def law(logits, temperature):
    """The distribution of a row, or None where it has none."""
    x = np.asarray(logits, np.float64)
    t = float(temperature)
    if np.isnan(x).any() or x.max() in (np.inf, -np.inf) or not 0 <= t < np.inf:
        return None
    if t == 0:
        p = np.zeros(len(x))
        p[np.argmax(x)] = 1
        return p
    p = np.exp((x - x.max()) / t)
    return p / p.sum()


def left(p, q, x):
    """What the next token is drawn from behind the refused draft x of distribution q (None: a point mass)."""
    rest = p.copy()
    if q is not None:
        rest = np.maximum(p - q, 0)
    elif 0 <= x < len(p):
        rest[x] = 0
    return rest if rest.sum() > 0 else p


def draw(p, u):
    u = min(max(u, 0.0), np.nextafter(1, 0)) if u == u else 0.0
    cum = np.cumsum(p)
    at = int(np.searchsorted(cum, u * cum[-1], side="right"))
    return min(at, int(np.nonzero(p)[0][-1]))


def verify(start, tokens, logits, draft, temperature, accept_u, sample_u):
    """accepted [n], next token [n]."""
    accepted, following = [], []
    for b, t in enumerate(temperature):
        first, end = start[b], start[b + 1]
        if first < 0 or end > len(tokens) or first >= end:
            accepted.append(0)
            following.append(-1)
            continue
        for r in range(first, end):
            p = law(logits[r], t)
            if r + 1 == end or p is None:
                break
            x = tokens[r + 1]
            q = None if draft is None else law(draft[r], t)
            px = p[x] if 0 <= x < len(p) else 0.0
            qx = 1.0 if q is None else q[x] if 0 <= x < len(p) else 0.0
            if not (0 <= x < len(p) and accept_u[r] * qx < px):
                p = left(p, q, x)
                break
        accepted.append(r + 1 - first)
        following.append(-1 if p is None else draw(p, sample_u[b]))
    return accepted, following
