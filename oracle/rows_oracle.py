"""fp64 numpy statement of the calls for turns of many tokens and shared prefixes: tables of rotary angles, rotations in both layouts and of a part of
the head, rows appended to a paged cache, attention of a turn's tokens over it and of tokens that share a prefix. Plain steps, one
sequence and head after the other. Test infrastructure, as decode_oracle.py; pinned by tests/test_oracle_rows.py.
"""
from __future__ import annotations

import math

import numpy as np

from oracle.decode_oracle import place


def frequencies(rot, base, scaling="none", factor=1.0, original=0.0, low=0.0, high=0.0):
    """Radians a position of the rot / 2 pairs."""
    out = []
    for i in range(rot // 2):
        w = base ** (-2.0 * i / rot)
        if scaling == "linear":
            w = w / factor
        elif scaling == "dims":
            dim = lambda turns: rot * math.log(original / (2.0 * math.pi * turns)) / (2.0 * math.log(base))  # noqa: E731
            a, b = max(math.floor(dim(high)), 0), min(math.ceil(dim(low)), rot - 1)
            s = min(max((i - a) / max(b - a, 1e-3), 0.0), 1.0)
            w = s * w / factor + (1.0 - s) * w
        elif scaling == "waves":
            s = min(max((original * w / (2.0 * math.pi) - low) / (high - low), 0.0), 1.0)
            w = s * w + (1.0 - s) * w / factor
        out.append(w)
    return np.array(out)


def tables(n_pos, rot, base, scaling="none", factor=1.0, original=0.0, low=0.0, high=0.0, scale=1.0, first=0):
    p = first + np.arange(n_pos, dtype=np.float64)
    a = p[:, None] * frequencies(rot, base, scaling, factor, original, low, high)
    return scale * np.cos(a), scale * np.sin(a)


def rotate(x, gain, eps, cos, sin, interleaved):
    """x [..., d]; cos, sin [..., rot / 2]: norm over all dims (gain None: neither), then the pairs of the first rot dims."""
    x = np.array(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(gain, dtype=np.float64)
    h = cos.shape[-1]
    a, b = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
    y = x.copy()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def append_places(starts, T, tables_, lengths, page_size, num_pages):
    """Of every token and KV head, (page, slot) or None; tokens of no sequence: None for the whole token."""
    B, Hkv = lengths.shape
    out = [None] * T
    for b in range(B):
        n = int(starts[b + 1]) - int(starts[b])
        for i in range(n):
            row = [int(lengths[b, h]) - n + i for h in range(Hkv)]
            out[int(starts[b]) + i] = [place(tables_[b], r, page_size, num_pages) if 0 <= r < tables_.shape[1] * page_size else None for r in row]
    return out


def rows_of(K, V, table, n, h):
    """Keys and values of the first n rows of a head that are there, and their numbers."""
    pages, page_size = K.shape[:2]
    n = min(max(int(n), 0), len(table) * page_size)
    j = np.arange(n)
    page = np.asarray(table, dtype=np.int64)[j // page_size]
    j = j[(page >= 0) & (page < pages)]
    page = np.asarray(table, dtype=np.int64)[j // page_size]
    return K[page, j % page_size, h], V[page, j % page_size, h], j


def softmax_rows(q, k, v, seen):
    """q [n, d] over k, v [rows, d], of which seen [n, rows]. Zeros where nothing is seen or no logit is above -inf."""
    out = np.zeros((len(q), v.shape[1]))
    for i in range(len(q)):
        at = np.flatnonzero(seen[i])
        with np.errstate(invalid="ignore", over="ignore"):
            s = k[at] @ q[i] / math.sqrt(len(q[i]))
            if not len(at) or np.all(s == -np.inf):
                continue
            p = np.exp(s - (np.nan if np.isnan(s).any() else s.max()))
            out[i] = (p / p.sum()) @ v[at]
    return out


def attend_rows(q, starts, K, V, tables_, lengths, causal, result=None):
    """q [T, Hq, d] -> out [T, Hq, d]; tokens of no sequence keep what `result` holds."""
    T, Hq, d = q.shape
    B, Hkv = lengths.shape
    G, cap = Hq // Hkv, tables_.shape[1] * K.shape[1]
    out = np.zeros(q.shape) if result is None else result
    for b in range(B):
        t0, t1 = int(starts[b]), int(starts[b + 1])
        n = t1 - t0
        for h in range(Hkv):
            L = min(max(int(lengths[b, h]), 0), cap)
            k, v, j = rows_of(K, V, tables_[b], L, h)
            limit = L - (n - 1 - np.arange(n)) if causal else np.full(n, L)
            for g in range(h * G, (h + 1) * G):
                out[t0:t1, g] = softmax_rows(q[t0:t1, g], k, v, j < limit[:, None])
    return out


def attend_shared(q, starts, K, V, prefix_tables, prefix_lengths, tables_, lengths):
    B, Hq, d = q.shape
    Hkv = lengths.shape[1]
    G = Hq // Hkv
    group = np.full(B, -1)
    for p in range(len(prefix_lengths)):
        group[int(starts[p]):int(starts[p + 1])] = p
    out = np.zeros(q.shape)
    for b in range(B):
        for h in range(Hkv):
            k, v, _ = rows_of(K, V, tables_[b], lengths[b, h], h)
            if group[b] >= 0:
                pk, pv, _ = rows_of(K, V, prefix_tables[group[b]], prefix_lengths[group[b], h], h)
                k, v = np.concatenate([pk, k]), np.concatenate([pv, v])
            out[b, h * G:(h + 1) * G] = softmax_rows(q[b, h * G:(h + 1) * G], k, v, np.ones((G, len(k)), dtype=bool))
    return out
