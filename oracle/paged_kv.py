"""fp64 attention over a cache with a sliding window and sinks, the weight its tokens receive, and eviction by it.

One sequence, one head layout at a time; keys and values are [tokens, KV heads, channels], queries [rows, heads, channels],
the rows being the last ones of the cache: row i of n sits at slot T - n + i (below 0 if there are more rows than tokens).
A row at slot t sees the slots j <= t, with a window only those with j < sinks or j > t - window, and of those only the
ones that `there` marks (tokens whose page exists).
"""
from __future__ import annotations

import numpy as np


def visible(n_rows: int, tokens: int, window: int, sinks: int, there=None) -> np.ndarray:
    """[rows, tokens] truth values."""
    t = np.arange(tokens - n_rows, tokens)[:, None]
    j = np.arange(tokens)[None]
    seen = j <= t
    if window:
        seen &= (j < sinks) | (j > t - window)
    return seen if there is None else seen & np.asarray(there, dtype=bool)[None]


def attention(q, k, v, scale, window=0, sinks=0, there=None):
    """-> out [rows, heads, channels], lse [rows, heads], weights p [rows, heads, tokens], and two sizes that error bounds
    are made of: sum_j p_j |v_j| like out, and max_j scale sum_d |q_d k_jd| like lse."""
    q, k, v = (np.asarray(x, dtype=np.float64) for x in (q, k, v))
    n, Hq, dh = q.shape
    T, Hkv = k.shape[0], k.shape[1]
    seen = visible(n, T, window, sinks, there)
    out, mag = np.zeros((n, Hq, dh)), np.zeros((n, Hq, dh))
    lse, big = np.full((n, Hq), -np.inf), np.zeros((n, Hq))
    p = np.zeros((n, Hq, T))
    for h in range(Hq):
        g = h // (Hq // Hkv)
        kk = np.where(seen.any(axis=0)[:, None], k[:, g], 0.0)      # what no row sees may hold anything
        vv = np.where(seen.any(axis=0)[:, None], v[:, g], 0.0)
        s = np.where(seen, scale * (q[:, h] @ kk.T), -np.inf)
        some = seen.any(axis=1)
        if not some.any():
            continue
        top = np.where(some, np.max(s, axis=1, initial=-np.inf), 0.0)
        e = np.exp(s - top[:, None])
        total = e.sum(axis=1)
        p[:, h] = e / np.where(some, total, 1.0)[:, None]
        lse[some, h] = (top + np.log(np.where(some, total, 1.0)))[some]
        out[:, h], mag[:, h] = p[:, h] @ vv, p[:, h] @ np.abs(vv)
        big[:, h] = np.max(np.where(seen, scale * (np.abs(q[:, h]) @ np.abs(kk).T), 0.0), axis=1, initial=0.0)
    return out, lse, p, mag, big


def score(p: np.ndarray, n_kv_heads: int) -> np.ndarray:
    """Weight that every token receives: [KV heads, tokens] from the p of attention()."""
    n, Hq, T = p.shape
    return p.reshape(n, n_kv_heads, Hq // n_kv_heads, T).sum(axis=(0, 2))


def evict(scores, budget: int, sinks: int, recent: int) -> list[int]:
    """Slots that stay of one (sequence, KV head) with these scores, in order."""
    T = len(scores)
    if T <= budget:
        return list(range(T))
    middle = list(range(sinks, T - recent))
    rank = {j: -np.inf if np.isnan(scores[j]) else float(scores[j]) for j in middle}
    # NaN ranks below every number, -infinity included
    best = sorted(middle, key=lambda j: (bool(np.isnan(scores[j])), -rank[j], j))[: budget - sinks - recent]
    return sorted(list(range(sinks)) + best + list(range(T - recent, T)))
