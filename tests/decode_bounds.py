"""How far attention over a paged cache may be off, head by head: from the rows that a query head sees and nothing else, so that what stands in rows
that are not seen, or in another head's, widens no tolerance.

With S_j the sum of the |q_i k_ji| of row j, s_j its logit, n the rows seen, all for one query head, and steps of 16 rows and dims:
  logit    a product of the tensor core adds 16 terms to a sum and may cut each of the 17 at 2^-23 of the largest: 17 d / 16 cuts, and the sum of
           its two halves, each at most 2^-23 S_j (none where a single product is not zero: it fits 24 bits). The factor 1 / sqrt(d), its product and the
           difference to the reference round by 2^-24 of the largest logit each, the reference counted twice: 4.
  weight   both ends of a ratio have that error, so twice; a weight is a product of at most 16 exponentials (its own, moves of the reference, joins) of 2^-22 each;
           the sum of weights has n / 8 terms a lane and 200 joins, 2^-24 each.
  output   the terms of p in bf16 twice: 2^-16. A step of 16 rows cuts 2 * 17 terms at 2^-23 of sum p |v| and may scale what is there (2^-24); 200 joins.
           A warp takes at most n / 16 + 1 steps of a head. In one launch they are 18 at most (1152 rows a CTA, four warps); in two, the T tiles (of 16
           rows a warp; counted too high here, with those that stand for beginnings) are dealt evenly to 148 CTAs, so T / 148 + 1.
Everything is multiplied by sum p |v|; then one rounding to bf16.
"""
import numpy as np

from oracle import chunkkv_oracle, decode_oracle as ora
from tests.helpers import rand_bits

U, E = 2.0 ** -8, 2.0 ** -24
MOST = 1e-2                       # a factor of sum p |v| beyond this says nothing: no comparison goes by it


def wide(bits):
    return chunkkv_oracle.bf16_bits_to_f64(bits)


def new_cache(rng, B, Hkv, d, page, per, spare=3):
    pages = B * per + spare
    K, V = rand_bits(rng, (pages, page, Hkv, d)), rand_bits(rng, (pages, page, Hkv, d))
    return K, V, rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32)


def bounds(q, K, V, tables, lengths):
    """q [B, Hq, d], K, V as values. (out, its tolerance [B, Hq, d], sums of weights, their error [B, Hkv, rows], factors of sum p |v| [B, Hq]);
    not-a-number where the formula's output is not finite."""
    B, Hq, d = q.shape
    pages, page, Hkv, _ = K.shape
    G, cap = Hq // Hkv, tables.shape[1] * page
    dealt = max(18, B * -(-Hkv // 8) * -(-G // 8) * (cap // 16 + 5) // 148 + 2)
    out, sums = ora.attend(q, K, V, tables, lengths)
    tol, err, factor = np.full(out.shape, np.nan), np.zeros(sums.shape), np.zeros((B, Hq))
    for b in range(B):
        for h in range(Hkv):
            n = min(max(int(lengths[b, h]), 0), cap)
            page_of = tables[b, np.arange(n) // page]
            rows = np.flatnonzero((page_of >= 0) & (page_of < pages))
            k, v = K[page_of[rows], rows % page, h], V[page_of[rows], rows % page, h]
            for g in range(h * G, (h + 1) * G):
                with np.errstate(invalid="ignore"):
                    s = k @ q[b, g] / np.sqrt(d) if len(rows) else np.zeros(0)
                if not np.isfinite(s).any():                    # nothing seen: zeros, exactly; or nothing that is a number
                    if not len(rows) or np.all(s == -np.inf):
                        tol[b, g] = 0.0
                    continue
                if np.isnan(s).any() or np.any(s == np.inf):
                    err[b, h, rows] = np.nan
                    continue
                seen = np.isfinite(s)
                terms = np.abs(k[seen] * q[b, g])
                cuts = np.where((terms != 0).sum(1) > 1, (17 * d / 16 + 1) * 2.0 ** -23 * terms.sum(1), 0.0) / np.sqrt(d)
                rel = 2 * (cuts.max() + 4 * E * np.abs(s[seen]).max()) + 16 * 2.0 ** -22 + (len(rows) / 8 + 200) * E
                p = np.where(seen, np.exp(s - s[seen].max()), 0.0)
                p /= p.sum()
                factor[b, g] = rel + 2.0 ** -16 + min(len(rows) // 16 + 1, dealt) * (34 * 2.0 ** -23 + E) + 200 * E
                with np.errstate(invalid="ignore"):
                    tol[b, g] = U * np.abs(out[b, g]) + (1 + U) * factor[b, g] * (p @ np.abs(v))
                err[b, h, rows] += (rel + G * E) * p
    return out, tol, sums, err, factor


def check(out, weights, before, q, K, V, tables, lengths):
    """What a call gave, as values (weights and before may be None), against the formula."""
    ref, tol, sums, err, factor = bounds(q, K, V, tables, lengths)
    assert factor.max() < MOST, factor.max()
    fine = np.isfinite(ref) & np.isfinite(tol)
    assert np.array_equal(np.isnan(ref), np.isnan(out)) and np.array_equal(np.isfinite(ref), np.isfinite(out))
    off = np.abs(out - ref)[fine] > tol[fine]
    assert not off.any(), (off.sum(), (np.abs(out - ref)[fine] - tol[fine]).max())
    if weights is None:
        return
    cap = sums.shape[2]
    seen = np.arange(cap) < np.clip(lengths, 0, cap)[..., None]
    assert np.array_equal(weights[~seen], before[~seen])
    want = before + sums
    ok = np.isfinite(want) & np.isfinite(err)
    assert np.array_equal(np.isfinite(want), np.isfinite(weights))
    assert (np.abs(weights - want) <= 2 * E * np.abs(want) + err)[ok].all()


# ------------------------------------------------------------------------------------------------ caches with what must not be seen
def absent(d, room, seed=51):
    """Heads of which many rows are not there: lengths and pages out of range; the largest numbers, infinities and not-a-number in every row that nobody sees."""
    Hq, Hkv, page, per, B = 6, 2, 8, 6, 5
    rng = np.random.default_rng(seed)
    K, V, tables = new_cache(rng, B, Hkv, d, page, per)
    lengths = np.array([[6, 48], [19, 0], [48, 33], [-7, 1], [2**31 - 1, -2**31]], dtype=np.int64).astype(np.int32)
    tables[2, 2], tables[2, 4], tables[4, 1], tables[3, :] = -1, len(K), -2**31, 2**31 - 1
    used = np.zeros(K.shape[:3], dtype=bool)
    for b in range(B):
        for h in range(Hkv):
            for j in range(min(max(int(lengths[b, h]), 0), per * page)):
                at = ora.place(tables[b], j, page, len(K))
                if at is not None:
                    used[at[0], at[1], h] = True
    bad = np.array([0x7FC0, 0x7F80, 0xFF80, 0x7F7F, 0xFF7F, 0x7F00, 0xFF00], dtype=np.uint16)
    for x in (K, V):
        x[~used] = rng.choice(bad, (int((~used).sum()), d))
    tables = np.concatenate([tables, np.full((B, room), -1, dtype=np.int32)], 1)
    return rand_bits(rng, (B, Hq, d)), K, V, tables, lengths


def extreme(d, G, room, seed=52):
    """Six KV heads: 0 with logits of -inf in some rows and in whole steps, 1 in every row, 2 with one of +inf, 3 with logits of +-1e4, 4 with one that is
    not a number, 5 with ordinary ones."""
    page, per, Hkv, n = 16, 8, 6, 120
    rng = np.random.default_rng(seed)
    K, V, tables = new_cache(rng, 1, Hkv, d, page, per)
    q = rand_bits(rng, (1, Hkv * G, d))
    q[..., 0] = 0x3F80                                                       # 1.0
    row = np.arange(n)
    p, s = tables[0, row // page], row % page
    some = (row % 3 != 0) | ((row >= 16) & (row < 80))
    K[p[some], s[some], 0, 0] = 0xFF80
    K[p, s, 1, 0] = 0xFF80
    K[p[50], s[50], 2, 0] = 0x7F80
    K[p, s, 3] = 0
    K[p, s, 3, 0] = np.where(row == 77, 0x47C3, 0xC7C3)                      # +-99840
    K[p[70], s[70], 4, 3] = 0x7FC0
    tables = np.concatenate([tables, np.full((1, room), -1, dtype=np.int32)], 1)
    return q, K, V, tables, np.full((1, Hkv), n, dtype=np.int32)
