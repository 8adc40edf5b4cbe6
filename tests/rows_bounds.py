"""How far the calls for turns and shared prefixes may be off.

Attention. As tests/decode_bounds.py, with S_j the sum of |q_i k_ji| of row j, n the rows that a query head sees, tiles of 128 rows:
  logit    17 d / 16 cuts of at most 2^-23 S_j in the product (none where a single term is not zero: it fits 24 bits); its factor and the difference to the reference 2^-24 of the largest logit each, counted
           four times with the reference's own.
  weight   both ends of a ratio have that error, so twice; an exponential 2^-22, as often as a reference moves (once a tile at most) and records
           are joined (148 at most); its sum n / 2 + 200 additions of 2^-24 (128 in pairs a tile, then tiles and records, counted too high).
  output   the weight's rounding to bf16, 2^-8, the sum's being taken before it; a tile's product cuts 8 * 17 terms at 2^-23 of sum p |v|, and scaling and
           joining round by 2^-24 each.
All of it times sum p |v|, then one rounding to bf16, 2^-8 of the output.

Counting. With logits that are all 0, weights are 1, exact in bf16, and values that are small whole numbers add up exactly: the output is
sum / n, off by the reciprocal, the product and the rounding: (2^-8 + 2^-22) of it. A row too many or too few moves it by 1 / n of a value.
"""
import numpy as np

from oracle import rows_oracle as ora

U, E = 2.0 ** -8, 2.0 ** -24
TILE, RECORDS = 128, 148


def factor(q, k, seen):
    """Of sum p |v|, for query rows q [n, d] over k [rows, d] of which seen [n, rows]; and p."""
    d = q.shape[1]
    s = q @ k.T / np.sqrt(d)
    S = np.abs(q) @ np.abs(k).T
    s = np.where(seen, s, -np.inf)
    top = s.max(1, keepdims=True, initial=-np.inf)
    p = np.exp(s - np.where(np.isfinite(top), top, 0.0))
    total = p.sum(1, keepdims=True)
    p = np.divide(p, total, out=np.zeros_like(p), where=total > 0)
    terms = (q != 0).astype(float) @ (k != 0).T
    cuts = np.where(seen & (terms > 1), (17 * d / 16 + 1) * 2.0 ** -23 * S, 0.0).max(1, initial=0.0) / np.sqrt(d)
    n = seen.sum(1)
    tiles = n / TILE + 2
    large = np.where(seen, np.abs(np.where(seen, s, 0.0)), 0.0).max(1, initial=0.0)
    rel = 2 * (cuts + 4 * E * large) + (tiles + RECORDS + 2) * 2.0 ** -22 + (n / 2 + 200) * E
    return U + rel + tiles * (8 * 17 * 2.0 ** -23 + E) + RECORDS * E, p


def check_rows(out, q, k, v, seen, what=""):
    """out [n, d] of query rows q over k, v [rows, d]; all as values."""
    ref = ora.softmax_rows(q, k, v, seen)
    f, p = factor(q, k, seen)
    assert f.max(initial=0.0) < 2e-2, f.max()
    tol = U * np.abs(ref) + (1 + U) * f[:, None] * (p @ np.abs(v))
    off = np.abs(out - ref)
    assert not np.isnan(off).any() and (off <= tol).all(), (what, np.argwhere(~(off <= tol))[:3].tolist(), (off - tol).max())


def check_attend(out, q, starts, K, V, tables, lengths, causal):
    T, Hq, d = q.shape
    B, Hkv = lengths.shape
    G, cap = Hq // Hkv, tables.shape[1] * K.shape[1]
    for b in range(B):
        t0, t1 = int(starts[b]), int(starts[b + 1])
        n = t1 - t0
        for h in range(Hkv):
            L = min(max(int(lengths[b, h]), 0), cap)
            k, v, j = ora.rows_of(K, V, tables[b], L, h)
            limit = L - (n - 1 - np.arange(n)) if causal else np.full(n, L)
            for g in range(h * G, (h + 1) * G):
                check_rows(out[t0:t1, g], q[t0:t1, g], k, v, j < limit[:, None], (b, g))


def check_shared(out, q, starts, K, V, prefix_tables, prefix_lengths, tables, lengths):
    B, Hq, d = q.shape
    Hkv = lengths.shape[1]
    G = Hq // Hkv
    group = np.full(B, -1)
    for p in range(len(prefix_lengths)):
        group[int(starts[p]):int(starts[p + 1])] = p
    for b in range(B):
        for h in range(Hkv):
            k, v, _ = ora.rows_of(K, V, tables[b], lengths[b, h], h)
            if group[b] >= 0:
                pk, pv, _ = ora.rows_of(K, V, prefix_tables[group[b]], prefix_lengths[group[b], h], h)
                k, v = np.concatenate([pk, k]), np.concatenate([pv, v])
            check_rows(out[b, h * G:(h + 1) * G], q[b, h * G:(h + 1) * G], k, v, np.ones((G, len(k)), dtype=bool), (b, h))


def count_rows(out, ref):
    """Outputs of attention whose logits are all 0 over whole numbers, against sums that are exact."""
    assert np.array_equal(np.isnan(ref), np.isnan(out))
    fine = ~np.isnan(ref)
    # (the reference's own n additions of up to 8 / n round by 2^-53 each: n 8 2^-53 < 2^-40 up to a thousand rows, and a row moves a mean that is 0 by 1 / n)
    off = np.abs(out - ref)[fine] > (U + 4 * E) * np.abs(ref)[fine] + 2.0 ** -40
    assert not off.any(), (int(off.sum()), np.argwhere(~(np.abs(out - ref) <= (U + 4 * E) * np.abs(ref) + 2.0 ** -40))[:4].tolist())
