"""fp64 numpy statement of the calls on the decode cache: queries and keys normalised and rotated, attention of one token over
a paged cache, and eviction by sums of attention. One sequence and head after the other, in plain steps. Test infrastructure, as
chunkkv_oracle.py; pinned by tests/test_oracle_decode.py.
"""
from __future__ import annotations

import numpy as np


def rotate(x: np.ndarray, gain, eps: float, cos: np.ndarray, sin: np.ndarray) -> np.ndarray:
    """x [..., d]: divided by its root mean square and multiplied by `gain` (None: neither), then element i is rotated with
    element i + d / 2 by the angle whose cosine and sine are cos[..., i], sin[..., i]."""
    x = np.asarray(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(gain, dtype=np.float64)
    a, b = np.split(x, 2, axis=-1)
    return np.concatenate([a * cos - b * sin, b * cos + a * sin], axis=-1)


def place(table: np.ndarray, row: int, page_size: int, num_pages: int):
    """(page, slot) of a sequence's row; None where its page is outside the cache."""
    page = int(table[row // page_size])
    return (page, row % page_size) if 0 <= page < num_pages else None


def attend(q: np.ndarray, K: np.ndarray, V: np.ndarray, tables: np.ndarray, lengths: np.ndarray):
    """q [B, Hq, d], K / V [pages, page_size, Hkv, d] -> out [B, Hq, d] and the rows' attention summed over the query heads of a
    KV head [B, Hkv, rows of a table]."""
    B, Hq, d = q.shape
    pages, page_size, Hkv, _ = K.shape
    G, cap = Hq // Hkv, tables.shape[1] * page_size
    out, sums = np.zeros((B, Hq, d)), np.zeros((B, Hkv, cap))
    for b in range(B):
        for h in range(Hkv):
            n = min(max(int(lengths[b, h]), 0), cap)
            where = [place(tables[b], j, page_size, pages) for j in range(n)]
            rows = [j for j in range(n) if where[j] is not None]
            if not rows:
                continue
            at = np.array([where[j] for j in rows])
            k, v = K[at[:, 0], at[:, 1], h], V[at[:, 0], at[:, 1], h]
            for g in range(h * G, (h + 1) * G):
                with np.errstate(invalid="ignore"):
                    s = (k @ q[b, g]) / np.sqrt(d)
                    top = s.max()
                    if top == -np.inf:
                        continue
                    p = np.exp(s - top)
                    p /= p.sum()
                    out[b, g] = p @ v
                sums[b, h, rows] += p
    return out, sums


def evict_rows(weights: np.ndarray, n: int, w: int, c: int, budget: int) -> list:
    """Former rows of a head's rows after eviction, from its sums of attention (f32)."""
    if n <= budget:
        return list(range(n))
    C = (n - w) // c
    r = n - C * c
    k = (budget - r) // c
    s = [float(np.float32(np.sum(weights[i * c:(i + 1) * c].astype(np.float64)))) for i in range(C)]
    order = sorted(range(C), key=lambda i: (s[i] == s[i], -s[i] if s[i] == s[i] else 0.0, i))      # not-a-number first
    best = set(order[:k])
    coming = iter(sorted(i for i in best if i >= k))
    chunks = [i if i in best else next(coming) for i in range(k)]
    return [i * c + j for i in chunks for j in range(c)] + list(range(C * c, n))


def evict(weights, tables, lengths, K, V, w: int, c: int, budget: int):
    """New (weights, lengths, K, V, idx); rows in pages outside the cache are zero when read and not written."""
    B, Hkv, cap = weights.shape
    pages, page_size = K.shape[:2]
    weights, lengths, K, V = weights.copy(), lengths.copy(), K.copy(), V.copy()
    idx = np.full((B, Hkv, budget), -1, dtype=np.int32)
    for b in range(B):
        for h in range(Hkv):
            n = min(max(int(lengths[b, h]), 0), cap)
            rows = evict_rows(weights[b, h], n, w, c, budget)
            idx[b, h, :len(rows)] = rows
            if n <= budget:
                continue
            for cache in (K, V):
                held = {}
                for j in rows:
                    at = place(tables[b], j, page_size, pages)
                    held[j] = cache[at[0], at[1], h].copy() if at is not None else np.zeros_like(cache[0, 0, h])
                for i, j in enumerate(rows):
                    at = place(tables[b], i, page_size, pages)
                    if at is not None and i != j:
                        cache[at[0], at[1], h] = held[j]
            weights[b, h, :len(rows)] = weights[b, h, rows]
            weights[b, h, len(rows):n] = 0.0
            lengths[b, h] = len(rows)
    return weights, lengths, K, V, idx
