"""A bounded cache and drafted tokens in float64, element by element: the weights that
cached tokens get, which of them are kept, and the verification of drafts.

Written from the definitions in include/cqsa.h; shares no code with the GPU path.
"""
import math

import numpy as np


def weigh(q, k, lse, there, length, count, causal, scale, prior, decay):
    """One sequence: q float64 [n, Hq, d], k [tokens >= length, H, d], lse [n, Hq], there
    [tokens], prior [H, tokens] or None.  W [H, length], and for bounds per token the largest
    exponent error's sources: the sum of |q k| scale and |lse| over its pairs."""
    n, Hq, _ = q.shape
    H = k.shape[1]
    G = Hq // H
    W, big = np.zeros((H, length)), np.zeros((H, length))
    for i in range(min(count, n)):
        last = min(length, length - n + i + 1) if causal else length
        for h in range(Hq):
            if not math.isfinite(lse[i, h]):
                continue
            for t in range(max(last, 0)):
                if not there[t]:
                    continue
                s = float(k[t, h // G] @ q[i, h]) * scale
                W[h // G, t] += math.exp(s - lse[i, h])
                big[h // G, t] = max(big[h // G, t], float(np.abs(k[t, h // G]) @ np.abs(q[i, h])) * scale,
                                     abs(lse[i, h]), abs(s))
    old = max(0, length - n)
    if prior is not None:
        W[:, :old] += decay * prior[:, :old]
    return W, big


def weigh_rows(q, k, lse, there, length, count, causal, scale, prior, decay):
    """weigh() by matrix products, a key head at a time; every LSE finite."""
    n, Hq, _ = q.shape
    H = k.shape[1]
    G = Hq // H
    W, big = np.zeros((H, length)), np.zeros((H, length))
    t = np.arange(length)
    last = length - n + 1 + np.arange(n) if causal else np.full(n, length)
    seen = (t < last[:, None]) & there[:length] & (np.arange(n) < count)[:, None]
    for h in range(Hq):
        kk = k[:length, h // G]
        s = q[:, h] @ kk.T * scale
        W[h // G] += np.where(seen, np.exp(np.where(seen, s, -np.inf) - np.maximum(lse[:, h, None], -1e300)), 0.0).sum(0)
        size = np.maximum(np.abs(q[:, h]) @ np.abs(kk).T * scale, np.abs(lse[:, h, None]))
        big[h // G] = np.maximum(big[h // G], np.where(seen, size, 0.0).max(0, initial=0.0))
    old = max(0, length - n)
    if prior is not None:
        W[:, :old] += decay * prior[:, :old]
    return W, big


def keep(w, there, length, budget, first, recent):
    """The positions that a head with weights w [>= length] keeps, in order."""
    def rank(t):
        if t < first or t >= length - recent:
            return (2, 0.0)
        return (0, 0.0) if math.isnan(w[t]) else (1, float(w[t]))

    have = [t for t in range(length) if there[t]]
    best = sorted(have, key=lambda t: (rank(t), -t), reverse=True)[:budget]
    return sorted(best)


def _clean(x):
    x = np.asarray(x, np.float64)
    return np.where(np.isfinite(x) & (x > 0), x, 0.0)


def verify(p, q, tokens, count, u, length=None):
    """One sequence: p [K + 1, V], q [K, V] or None.  (out [K + 1], n_out, new length, the
    least distance of a choice from its border, relative to the sum)."""
    K, V = p.shape[0] - 1, p.shape[1]
    n = min(max(int(count), 0), K)
    u = np.where(np.isnan(u), 0.0, np.asarray(u, np.float64))
    a = 0
    while a < n:
        x = int(tokens[a])
        if not 0 <= x < V:
            break
        qx = _clean(q[a, x]) if q is not None else 1.0
        if not u[a] * qx < _clean(p[a, x]):
            break
        a += 1
    r = _clean(p[a])
    if a < n:
        if q is not None:
            rest = np.maximum(r - _clean(q[a]), 0.0)
        else:
            rest = r.copy()
            if 0 <= tokens[a] < V:
                rest[tokens[a]] = max(0.0, rest[tokens[a]] - 1.0)
        if rest.any():
            r = rest
    token, near = -1, math.inf
    if r.any():
        where = np.nonzero(r)[0]
        total = np.cumsum(r[where])
        want = u[K] * math.fsum(r)
        at = np.nonzero(total > want)[0]
        token = int(where[at[0]] if at.size else where[-1])
        near = float(np.abs(total[:-1] - want).min() / total[-1]) if len(total) > 1 else math.inf
    out = np.full(K + 1, -1, np.int64)
    out[:a] = tokens[:a]
    out[a] = token
    return out, a + 1, None if length is None else max(0, int(length) - (n - a)), near
