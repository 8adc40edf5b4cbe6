"""The calls on the decode cache against the fp64 statement, at the sizes, lengths and masks where they can go wrong.

Tolerances (u = 2^-8: half a step of bf16, relative; e = 2^-24: of fp32)
  rotation   the fp32 value is within 40 e (|a cos| + |b sin|) of the formula's: a sum of at most 128 squares in 16 steps and 3
             shuffles, half of it by the square root (12 e), rsqrt and three products (8 e), the rotation (2 e), rounded up; then
             one rounding, u of the value.
  attention  a logit is a sum of d exact products in d / 16 steps of the tensor core, which may cut its terms at 2^-23 of the
             largest on either side: within d / 8 * 2^-23 * sum |q k| / sqrt(d), call the largest of those `ds`. A weight is within
             a = 2 ds + 4 * 2^-22 (two exponentials, both ends) + rows / 32 * 2^-23 (the sum) of its value, relative; out then within (a + 2^-16 + the same
             sum's error) * sum p |v| for the split of p and the sums of O, plus one rounding, u. Sums of weights: a times the
             value, plus half a step of fp32 of the sum before and after.
  eviction   exact.
"""
import threading

import numpy as np
import pytest
import torch

import paper_2502_00299_b200 as ck
from oracle import chunkkv_oracle, decode_oracle as ora
from tests.helpers import Guarded, rand_bits, to_dev

pytestmark = pytest.mark.gpu
U, E = 2.0 ** -8, 2.0 ** -24


def wide(bits):
    return chunkkv_oracle.bf16_bits_to_f64(bits)


def f64(t):
    return t.double().cpu().numpy()


def i32(x):
    return torch.tensor(np.ascontiguousarray(x), dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------ rotation
def angles(n, d, seed=0):
    a = np.random.default_rng(seed).uniform(-4, 4, (n, d // 2))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def rotated(x, gain, eps, cos, sin):
    """The formula's values and the tolerance, of x [T, H, d] with cos, sin [T, d / 2]."""
    ref = ora.rotate(x, gain, eps, cos[:, None], sin[:, None])
    a, b = np.split(np.abs(x) if gain is None else np.abs(ora.rotate(x, gain, eps, np.ones_like(cos[:, None]), np.zeros_like(sin[:, None]))), 2, -1)
    c, s = np.abs(cos[:, None]), np.abs(sin[:, None])
    scale = np.concatenate([a * c + b * s, b * c + a * s], -1)
    return ref, U * np.abs(ref) + 40 * E * scale * (1 + U)


SHAPES = [(8, 2, 64), (32, 8, 128), (28, 4, 128), (5, 5, 64), (20, 1, 128), (1, 1, 128), (3, 1, 64)]


@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
@pytest.mark.parametrize("T", [1, 2, 33, 700])
@pytest.mark.parametrize("norm", [False, True])
def test_rotation(Hq, Hkv, d, T, norm):
    rng = np.random.default_rng(T + Hq)
    extra = 8 * (T % 3)
    bits = rand_bits(rng, (T, (Hq + 2 * Hkv) * d + extra))
    gq, gk = (rand_bits(rng, (d,)) if norm else None for _ in range(2))
    cos, sin = angles(50, d)
    pos = rng.integers(0, 50, T)
    if T > 2:
        pos[1], pos[2] = -1, 50                                   # outside the table: zeros
    x = wide(bits[:, :(Hq + Hkv) * d]).reshape(T, Hq + Hkv, d)
    known = (pos >= 0) & (pos < 50)
    q, k = ck.rotate_qk(to_dev(bits), Hq, Hkv, d, torch.tensor(cos).cuda(), torch.tensor(sin).cuda(), i32(pos),
                        None if gq is None else to_dev(gq), None if gk is None else to_dev(gk), 1e-5)
    at = np.where(known, pos, 0)
    for got, part, gain in ((q, x[:, :Hq], gq), (k, x[:, Hq:], gk)):
        ref, tol = rotated(part, None if gain is None else wide(gain), 1e-5, cos[at].astype(np.float64), sin[at].astype(np.float64))
        ref[~known] = 0
        assert (np.abs(f64(got) - ref) <= tol * known[:, None, None]).all()


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 64), (28, 4, 128)])
def test_rotation_into_views(Hq, Hkv, d):
    """Head-major outputs and the place in the activation: bit for bit what packed outputs hold; nothing else changes."""
    T = 37
    rng = np.random.default_rng(1)
    qkv, gain = to_dev(rand_bits(rng, (T, (Hq + 2 * Hkv) * d + 16))), to_dev(rand_bits(rng, (d,)))
    cos, sin = (torch.tensor(t).cuda() for t in angles(64, d))
    pos = i32(rng.integers(0, 64, T))
    q, k = ck.rotate_qk(qkv, Hq, Hkv, d, cos, sin, pos, gain, gain)
    hq, hk = Guarded((Hq, T, d), torch.bfloat16), Guarded((Hkv, T, d), torch.bfloat16)
    ck.rotate_qk(qkv, Hq, Hkv, d, cos, sin, pos, gain, gain, out_q=hq.t.permute(1, 0, 2), out_k=hk.t.permute(1, 0, 2))
    assert torch.equal(hq.t.permute(1, 0, 2), q) and torch.equal(hk.t.permute(1, 0, 2), k)
    hq.check(), hk.check()
    inside = qkv.clone()
    heads = inside[:, :(Hq + 2 * Hkv) * d].unflatten(1, (-1, d))
    ck.rotate_qk(inside, Hq, Hkv, d, cos, sin, pos, gain, gain, out_q=heads[:, :Hq], out_k=heads[:, Hq:Hq + Hkv])
    assert torch.equal(heads[:, :Hq], q) and torch.equal(heads[:, Hq:Hq + Hkv], k)
    assert torch.equal(inside[:, (Hq + Hkv) * d:], qkv[:, (Hq + Hkv) * d:])
    one_q, one_k = ck.rotate_qk(qkv[:1], Hq, Hkv, d, cos, sin, pos[:1], gain, gain, out_q=torch.empty_strided((1, Hq, d), (3, d, 1), dtype=torch.bfloat16, device="cuda"))
    assert torch.equal(one_q, q[:1]) and torch.equal(one_k, k[:1])
    none_q, none_k = ck.rotate_qk(qkv[:0], Hq, Hkv, d, cos, sin, pos[:0], gain, gain)
    assert none_q.shape == (0, Hq, d) and none_k.shape == (0, Hkv, d)


def test_rotation_is_the_window_queries_one_for_a_window():
    """The same pairs and angles as the call that prepares the observation window (which rounds from 64 bits)."""
    Hq, Hkv, d, T, w = 8, 2, 128, 50, 16
    rng = np.random.default_rng(2)
    qkv = to_dev(rand_bits(rng, (T, (Hq + 2 * Hkv) * d)))
    cos, sin = (torch.tensor(t).cuda() for t in angles(T, d))
    q, _ = ck.rotate_qk(qkv, Hq, Hkv, d, cos, sin, torch.arange(T, device="cuda", dtype=torch.int32))
    want = ck.window_queries(qkv, Hq, Hkv, d, w, cos[-w:].contiguous(), sin[-w:].contiguous())
    got = q[-w:].permute(1, 0, 2)
    # two roundings of values that differ by some e: the same number or its neighbour, and hardly ever the neighbour
    assert (got.double() - want.double()).abs().le(2 * U * want.double().abs() + 1e-5).all() and (got != want).float().mean() < 0.01


def new_cache(rng, B, Hkv, d, page, per, spare=3):
    pages = B * per + spare
    K, V = rand_bits(rng, (pages, page, Hkv, d)), rand_bits(rng, (pages, page, Hkv, d))
    return K, V, rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32)


@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
@pytest.mark.parametrize("page", [1, 5, 16])
def test_append(Hq, Hkv, d, page):
    B, per = 6, 4
    rng = np.random.default_rng(page)
    K, V, tables = new_cache(rng, B, Hkv, d, page, per)
    lengths = rng.integers(1, per * page + 1, (B, Hkv)).astype(np.int32)
    lengths[0] = 0                                                # a padded sequence
    lengths[1, -1] = per * page + 1                               # no row left
    lengths[2, 0] = -5
    lengths[3] = [np.iinfo(np.int32).min, *lengths[3, 1:]]
    tables[4, 1], tables[4, 2], tables[5, 0] = -1, len(K), np.iinfo(np.int32).max
    bits = rand_bits(rng, (B, (Hq + 2 * Hkv) * d))
    gain = rand_bits(rng, (d,))
    cos, sin = angles(40, d)
    pos = rng.integers(0, 40, B)
    dK, dV = Guarded(K.shape, torch.bfloat16), Guarded(V.shape, torch.bfloat16)
    dK.t.copy_(to_dev(K)), dV.t.copy_(to_dev(V))
    args = (torch.tensor(cos).cuda(), torch.tensor(sin).cuda(), i32(pos))
    q = ck.append_paged(to_dev(bits), Hq, *args, i32(tables), i32(lengths), dK.t, dV.t, None, to_dev(gain))
    want_q, want_k = ck.rotate_qk(to_dev(bits), Hq, Hkv, d, *args, None, to_dev(gain))
    assert torch.equal(q, want_q)                                 # (checked against the formula above)
    want_k, v = want_k.view(torch.int16).cpu().numpy().view(np.uint16), bits.reshape(B, -1, d)[:, Hq + Hkv:]
    for b in range(B):
        for h in range(Hkv):
            n = int(lengths[b, h])
            at = ora.place(tables[b], n - 1, page, len(K)) if 1 <= n <= per * page else None
            if at is not None:
                K[at[0], at[1], h], V[at[0], at[1], h] = want_k[b, h], v[b, h]
    assert torch.equal(dK.t, to_dev(K)) and torch.equal(dV.t, to_dev(V))
    dK.check(), dV.check()


# ------------------------------------------------------------------------------------------------ attention
def check_attention(q, K, V, tables, lengths, weights=None):
    """One call against the formula; K, V, q as bf16 bits. Returns (out, weights)."""
    page, (B, Hq, d) = K.shape[1], q.shape
    Hkv, cap = K.shape[2], tables.shape[1] * page
    wq, wK, wV = wide(q), wide(K), wide(V)
    ref, sums = ora.attend(wq, wK, wV, tables, lengths)
    out = Guarded((B, Hq, d), torch.bfloat16)
    dw = None
    if weights is not None:
        dw = Guarded((B, Hkv, cap), torch.float32)
        dw.t.copy_(torch.tensor(weights))
    ck.attend_paged(to_dev(q), i32(tables), i32(lengths), to_dev(K), to_dev(V), None if dw is None else dw.t, out.t)
    out.check()
    with np.errstate(invalid="ignore"):
        ds = d / 8 * 2.0 ** -23 * np.nanmax(np.where(np.isfinite(np.abs(wq)), np.abs(wq), 0).sum(-1)) * np.max(np.where(np.isfinite(wK), np.abs(wK), 0)) / np.sqrt(d)
        most = ora.attend(wq, wK, np.abs(wV), tables, lengths)[0]
    added = cap / 32 * 2.0 ** -23
    rel = 2 * ds + 4 * 2.0 ** -22 + added
    got = f64(out.t)
    fine = np.isfinite(ref)
    assert np.array_equal(fine, np.isfinite(got)) and np.array_equal(np.isnan(ref), np.isnan(got))
    err, tol = np.abs(got - ref)[fine], (U * np.abs(ref) + (1 + U) * (rel + 2.0 ** -16 + added) * most)[fine]
    assert (err <= tol).all(), (err / np.maximum(tol, 1e-300)).max()
    if dw is not None:
        dw.check()
        want = weights.astype(np.float64) + sums
        seen = np.arange(cap) < np.clip(lengths, 0, cap)[..., None]
        now = f64(dw.t)
        assert np.array_equal(now[~seen], weights.astype(np.float64)[~seen])            # rows behind the last stay as they are
        ok = np.isfinite(want)
        assert np.array_equal(ok, np.isfinite(now))
        assert (np.abs(now - want) <= E * 2 * np.abs(want) + 2 * rel * sums)[ok].all()
    return out.t, None if dw is None else dw.t


EDGES = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 191, 200]


@pytest.mark.parametrize("Hq,Hkv,d", SHAPES + [(9, 1, 128), (16, 1, 64), (24, 2, 128), (17, 1, 128), (40, 1, 64), (33, 1, 128)])
@pytest.mark.parametrize("page", [1, 3, 16, 100])
@pytest.mark.parametrize("room", [0, 9000])
def test_attention_at_every_edge(Hq, Hkv, d, page, room):
    """Both forms: one launch where no sequence can have many rows, two (and shares of CTAs) where the tables have room for more."""
    per = -(-200 // page)
    B = -(-len(EDGES) // Hkv)
    rng = np.random.default_rng(Hq * page)
    lengths = np.resize(rng.permutation(EDGES), (B, Hkv)).astype(np.int32)
    K, V, tables = new_cache(rng, B, Hkv, d, page, per)
    q = rand_bits(rng, (B, Hq, d), 2.0)
    tables = np.concatenate([tables, np.full((B, room // page), -1, dtype=np.int32)], 1)
    check_attention(q, K, V, tables, lengths)
    check_attention(q, K, V, tables, lengths, rng.random((B, Hkv, tables.shape[1] * page)).astype(np.float32))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("room", [0, 2000])
def test_attention_sees_no_row_that_is_not_there(d, room):
    """Not-a-number and infinities behind a head's last row, in other heads' rows and in pages of nobody; pages outside the cache; lengths out of range."""
    Hq, Hkv, page, per, B = 6, 2, 8, 6, 5
    rng = np.random.default_rng(5)
    K, V, tables = new_cache(rng, B, Hkv, d, page, per)
    lengths = np.array([[5, 48], [17, 0], [48, 31], [-3, 1], [2**31 - 1, -2**31]], dtype=np.int64).astype(np.int32)
    tables[2, 1], tables[2, 3], tables[4, 0], tables[3, :] = -1, len(K), -2**31, 2**31 - 1
    used = set()
    for b in range(B):
        for h in range(Hkv):
            for j in range(min(max(int(lengths[b, h]), 0), per * page)):
                at = ora.place(tables[b], j, page, len(K))
                if at is not None:
                    used.add((*at, h))
    for p in range(len(K)):
        for s in range(page):
            for h in range(Hkv):
                if (p, s, h) not in used:
                    K[p, s, h], V[p, s, h] = rng.choice([0x7FC0, 0x7F80, 0xFF80, 0x7F7F, 0xFF7F], 2).astype(np.uint16)
    q = rand_bits(rng, (B, Hq, d))
    tables = np.concatenate([tables, np.full((B, room), -1, dtype=np.int32)], 1)
    out, _ = check_attention(q, K, V, tables, lengths, rng.random((B, Hkv, tables.shape[1] * page)).astype(np.float32))
    assert not out[3].any() and not out[1, 3:].any() and not out[4, 3:].any()          # heads that see nothing: zeros


@pytest.mark.parametrize("d,G", [(64, 3), (128, 8), (128, 12)])
@pytest.mark.parametrize("room", [0, 2000])
def test_attention_of_infinite_and_extreme_logits(d, G, room):
    """Keys that no query attends to (logit -inf) weigh nothing, a head of nothing else gets zeros; +inf and not-a-number go the formula's way;
    logits of +-1e4 neither overflow nor lose the largest."""
    page, per, Hkv = 16, 8, 6
    rng = np.random.default_rng(6)
    K, V, tables = new_cache(rng, 1, Hkv, d, page, per)
    q = rand_bits(rng, (1, Hkv * G, d))
    q[..., 0] = 0x3F80                                                       # 1.0
    lengths = np.full((1, Hkv), 120, dtype=np.int32)
    at = [ora.place(tables[0], j, page, len(K)) for j in range(120)]
    for j, (p, s) in enumerate(at):
        if j % 3:
            K[p, s, 0, 0] = 0xFF80                                           # some rows, and a whole step of them
        if 16 <= j < 80:
            K[p, s, 0, 0] = 0xFF80
        K[p, s, 1, 0] = 0xFF80                                               # every row
        K[p, s, 3, 1:] = 0
        K[p, s, 3, 0] = 0x47C3 if j == 77 else 0xC7C3                        # +-99840: logits of 1e4
    K[at[50][0], at[50][1], 2, 0] = 0x7F80                                   # a logit of +inf
    K[at[70][0], at[70][1], 4, 3] = 0x7FC0                                   # not a number
    tables = np.concatenate([tables, np.full((1, room), -1, dtype=np.int32)], 1)
    w = np.zeros((1, Hkv, tables.shape[1] * page), dtype=np.float32)
    out, sums = check_attention(q, K, V, tables, lengths, w)
    assert not out[0, G:2 * G].any() and not sums[0, 1].any()
    assert torch.isnan(out[0, 2 * G:3 * G]).all() and torch.isnan(out[0, 4 * G:5 * G]).all() and torch.isfinite(out[0, 5 * G:]).all()
    assert torch.equal(out[0, 3 * G], to_dev(V[at[77][0], at[77][1], 3]))


@pytest.mark.parametrize("room", [0, 2000])
def test_attention_over_large_and_infinite_values(room):
    """Values of up to 2^88 are not too large (products with powers of two are exact: the same output, times as much); an infinite one reaches
    its own dim alone."""
    rng = np.random.default_rng(31)
    K, V, tables = new_cache(rng, 2, 2, 64, 16, 8)
    q, lengths = rand_bits(rng, (2, 6, 64)), np.full((2, 2), 120, dtype=np.int32)
    lengths[1, 1] = 0
    tables = np.concatenate([tables, np.full((2, room), -1, dtype=np.int32)], 1)
    v = to_dev(V).clamp(-3.9, 3.9)
    args = to_dev(q), torch.from_numpy(tables).cuda(), torch.from_numpy(lengths).cuda(), to_dev(K)
    out = ck.attend_paged(*args, v)
    assert torch.equal(ck.attend_paged(*args, v * 2.0**86), out * 2.0**86)
    p, s = ora.place(tables[0], 77, 16, len(K))
    v[p, s, 1, 5] = float("inf")
    got = ck.attend_paged(*args, v)
    rest = torch.arange(64, device=got.device) != 5
    assert not torch.isfinite(got[0, 3:, 5]).any()
    assert torch.equal(got[..., rest], out[..., rest]) and torch.equal(got[1], out[1]) and torch.equal(got[0, :3], out[0, :3])


@pytest.mark.parametrize("Hq,Hkv,d,B,n,page", [(8, 2, 64, 1, 20011, 16), (32, 8, 128, 1, 3501, 16), (12, 1, 128, 2, 9001, 64), (12, 1, 128, 2, 17001, 64), (28, 4, 128, 3, 2500, 7),
                                               (4, 4, 64, 40, 300, 32), (2, 1, 128, 300, 90, 16)])
def test_attention_over_long_and_many_caches(Hq, Hkv, d, B, n, page):
    rng = np.random.default_rng(n)
    per = -(-n // page)
    K, V, tables = new_cache(rng, B, Hkv, d, page, per)
    lengths = np.maximum(n - (rng.random((B, Hkv)) ** 2 * n).astype(np.int32), 0).astype(np.int32)
    lengths[0, 0] = n
    check_attention(rand_bits(rng, (B, Hq, d), 3.0), K, V, tables, lengths, np.zeros((B, Hkv, per * page), dtype=np.float32))


@pytest.mark.parametrize("Hkv,B,d", [(1, 1, 128), (5, 1, 64), (3, 2, 64), (3, 5, 64), (2, 8, 128), (8, 4, 64), (1, 60, 128), (6, 20, 64), (148, 1, 64), (149, 1, 64)])
def test_attention_with_every_size_of_cluster(Hkv, B, d):
    """Short caches: a head's rows go to 16, 8, 4, 2 or 1 CTAs, of four warps with 149 heads; with fewer steps of 16 rows than CTAs among them."""
    rng = np.random.default_rng(Hkv * B)
    page, per = (16, 9) if B > 1 or Hkv > 5 else (16, 110)                   # (more than 1536 rows: 16)
    K, V, tables = new_cache(rng, B, Hkv, d, page, per)
    lengths = rng.integers(0, page * per + 1, (B, Hkv)).astype(np.int32)
    lengths[0, 0] = page * per
    check_attention(rand_bits(rng, (B, 2 * Hkv, d), 2.0), K, V, tables, lengths, rng.random((B, Hkv, per * page)).astype(np.float32))


def test_attention_reads_pages_that_sequences_share():
    rng = np.random.default_rng(21)
    K, V, tables = new_cache(rng, 3, 2, 64, 16, 5)
    tables[1, :3] = tables[0, :3]                                            # a common prefix
    tables[2, 4] = tables[2, 0]                                              # a page twice
    check_attention(rand_bits(rng, (3, 4, 64)), K, V, tables, np.array([[80, 70], [66, 48], [79, 80]], dtype=np.int32), np.zeros((3, 2, 80), dtype=np.float32))


@pytest.mark.parametrize("room", [0, 2000])
def test_rows_that_are_not_seen_get_no_weight_whatever_becomes_of_the_head(room):
    rng = np.random.default_rng(22)
    K, V, tables = new_cache(rng, 1, 1, 64, 16, 4)
    tables[0, 1] = -1
    K[tables[0, 2], 3, 0, 5] = 0x7FC0                                        # not a number: so are the outputs
    tables = np.concatenate([tables, np.full((1, room), -1, dtype=np.int32)], 1)
    w = torch.full((1, 1, tables.shape[1] * 16), 0.5, device="cuda")
    out = ck.attend_paged(to_dev(rand_bits(rng, (1, 2, 64))), i32(tables), i32([[60]]), to_dev(K), to_dev(V), w)
    assert torch.isnan(out).all() and (w[0, 0, 16:32] == 0.5).all() and (w[0, 0, 60:] == 0.5).all() and torch.isnan(w[0, 0, :16]).all()


def test_native_and_general_calls_are_the_same(monkeypatch):
    """The binding's general way (other streams, given outputs, declined arguments) queues what the native one does."""
    from paper_2502_00299_b200 import binding
    rng = np.random.default_rng(23)
    Hq, Hkv, d, page, per, B = 8, 2, 64, 16, 5, 3
    K, V, tables = new_cache(rng, B, Hkv, d, page, per)
    lengths = np.array([[70, 33], [1, 80], [0, 5]], dtype=np.int32)
    qkv, gain = to_dev(rand_bits(rng, (B, (Hq + 2 * Hkv) * d))), to_dev(rand_bits(rng, (d,)))
    cos, sin = (torch.tensor(x).cuda() for x in angles(9, d))
    pos = i32([3, 8, 0])

    def all_of_them(**k):
        dK, dV, dl, w = to_dev(K), to_dev(V), i32(lengths), torch.rand(B, Hkv, per * page, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
        torch.cuda.synchronize()
        r = list(ck.rotate_qk(qkv, Hq, Hkv, d, cos, sin, pos, gain, None, 1e-6, **k))
        r.append(ck.append_paged(qkv, Hq, cos, sin, pos, i32(tables), dl, dK, dV, gain, gain, 1e-6, **k))
        r.append(ck.attend_paged(r[2], i32(tables), dl, dK, dV, **k))
        r.append(ck.attend_paged(r[2], i32(tables), dl, dK, dV, w, **k))
        r.append(ck.evict_paged(w, i32(tables), dl, dK, dV, 4, 3, 20, **k))
        torch.cuda.synchronize()
        return r + [dK, dV, dl, w]

    taken = []
    with monkeypatch.context() as m:
        for name in ("rotate_qk", "append_paged", "attend_paged", "evict_paged"):
            was = getattr(binding._native, name)
            m.setattr(binding._native, name, lambda *a, was=was: taken.append(was(*a)) or taken[-1])
        native = all_of_them()
    assert len(taken) == 5 and all(t is not None and type(t) is not int for t in taken)
    side = torch.cuda.Stream()
    with monkeypatch.context() as m:
        for name in ("rotate_qk", "append_paged", "attend_paged", "evict_paged"):
            m.setattr(binding._native, name, lambda *a: None)
        general = all_of_them()
    other = all_of_them(stream=side)
    for a, b, c in zip(native, general, other):
        assert torch.equal(a, b) and torch.equal(a, c)
    with pytest.raises(ck.ChunkKVError):
        ck.evict_paged(native[-1], i32(tables), native[-2], native[-4], native[-3], 4, 3, 5)       # budget below w + c - 1
    with pytest.raises(ck.ChunkKVError):
        ck.rotate_qk(qkv, Hq, Hkv, d, cos, sin, pos, eps=-1.0)


def test_attention_beyond_32_bit_offsets():
    """A cache of more than 2^32 elements: its last pages are read and written."""
    Hkv, d, page, Hq, B = 8, 128, 16, 8, 1
    pages = 2 ** 32 // (page * Hkv * d) + 10
    K, V = (torch.zeros(pages, page, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rng = np.random.default_rng(8)
    bits = [rand_bits(rng, (4, page, Hkv, d)) for _ in range(2)]
    K[-4:], V[-4:] = to_dev(bits[0]), to_dev(bits[1])
    tables, lengths = np.array([[pages - 1, pages - 3, pages - 4, pages - 2]]), np.full((B, Hkv), 60, dtype=np.int32)
    q = rand_bits(rng, (B, Hq, d))
    out = ck.attend_paged(to_dev(q), i32(tables), i32(lengths), K, V)
    small = ck.attend_paged(to_dev(q), i32(tables - (pages - 4)), i32(lengths), K[-4:].clone(), V[-4:].clone())
    assert torch.equal(out, small) and out.any()
    cos, sin = torch.ones(4, 64, device="cuda"), torch.zeros(4, 64, device="cuda")
    qkv = to_dev(rand_bits(rng, (1, 3 * Hkv * d)))
    ck.append_paged(qkv, Hq, cos, sin, i32([0]), i32(tables), i32(lengths), K, V)
    assert torch.equal(V[pages - 2, 59 % page].flatten(), qkv[0, 2 * Hkv * d:]) and torch.equal(K[pages - 2, 59 % page].flatten(), qkv[0, Hkv * d:2 * Hkv * d])
    w = torch.rand(B, Hkv, 64, device="cuda")
    before = V[tables[0]].view(-1, Hkv, d).clone()
    idx = ck.evict_paged(w, i32(tables), i32(lengths), K, V, 4, 1, 30)
    after = V[tables[0]].view(-1, Hkv, d)
    for h in range(Hkv):
        assert torch.equal(after[:30, h], before[idx[0, h].long(), h])


@pytest.mark.parametrize("n", [1500, 6000])
def test_attention_is_the_same_every_time_and_beside_others(n):
    """Bit for bit: again, on another stream while other calls run, and as replays of graphs captured on two streams."""
    rng = np.random.default_rng(9)
    Hq, Hkv, d, page, B = 32, 8, 128, 16, 3
    K, V, tables = new_cache(rng, B, Hkv, d, page, -(-n // page))
    sets = []
    for i in range(2):
        lengths = rng.integers(1, n, (B, Hkv)).astype(np.int32)
        sets.append((to_dev(rand_bits(rng, (B, Hq, d))), i32(tables), i32(lengths), to_dev(K), to_dev(V)))
    zeros = torch.zeros(B, Hkv, tables.shape[1] * page, device="cuda")
    want = []
    for s in sets:
        w = zeros.clone()
        want.append((ck.attend_paged(*s, w), w))
        w = zeros.clone()
        assert torch.equal(ck.attend_paged(*s, w), want[-1][0]) and torch.equal(w, want[-1][1])
        assert torch.equal(ck.attend_paged(*s), want[-1][0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for round_ in range(20):
        got = []
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                w = zeros.clone()
            got.append((ck.attend_paged(*s, w, stream=st), w))
        torch.cuda.synchronize()
        for (o, w), (o0, w0) in zip(got, want):
            assert torch.equal(o, o0) and torch.equal(w, w0)
    graphs, outs, sums = [], [], []
    for s, st in zip(sets, streams):
        g, w = torch.cuda.CUDAGraph(), zeros.clone()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=st):
            outs.append(ck.attend_paged(*s, w))
        graphs.append(g)
        sums.append(w)
    for _ in range(3):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for o, w, (o0, w0) in zip(outs, sums, want):
        assert torch.equal(o, o0) and torch.allclose(w, 3 * w0, rtol=1e-6, atol=0)
    # lengths are read when a graph runs
    sets[0][2].fill_(7)
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], ck.attend_paged(*sets[0]))


def test_calls_of_several_threads():
    """Four host threads, a stream each, at the same time: what one call alone gives (short and long form, whose scratch is each call's own)."""
    rng = np.random.default_rng(12)
    jobs = []
    for i, (Hq, Hkv, d, B, n) in enumerate([(32, 8, 128, 3, 1500), (8, 2, 64, 2, 200), (12, 1, 128, 5, 2500), (8, 8, 64, 40, 700)]):
        K, V, tables = new_cache(rng, B, Hkv, d, 16, -(-n // 16))
        jobs.append((to_dev(rand_bits(rng, (B, Hq, d))), i32(tables), i32(rng.integers(1, n, (B, Hkv))), to_dev(K), to_dev(V)))
    want = [ck.attend_paged(*j) for j in jobs]
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    got = [[] for _ in jobs]

    def work(i):
        with torch.cuda.stream(streams[i]):
            for k in range(50):
                got[i].append(ck.attend_paged(*jobs[i], stream=streams[i] if k % 2 else None))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(jobs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert len(g) == 50 and all(torch.equal(x, w) for x in g)


# ------------------------------------------------------------------------------------------------ eviction
def check_eviction(rng, B, Hkv, d, page, per, lengths, w, c, budget, weights, holes=()):
    K, V, tables = new_cache(rng, B, Hkv, d, page, per)
    for b, p, v in holes:
        tables[b, p] = v
    cap = per * page
    weights = np.where(np.arange(cap) < np.clip(lengths, 0, cap)[..., None], weights, 0).astype(np.float32)
    dK, dV = Guarded(K.shape, torch.bfloat16), Guarded(V.shape, torch.bfloat16)
    dK.t.copy_(to_dev(K)), dV.t.copy_(to_dev(V))
    dw, dl, di = Guarded(weights.shape, torch.float32), Guarded(lengths.shape, torch.int32), Guarded((B, Hkv, budget), torch.int32)
    dw.t.copy_(torch.tensor(weights)), dl.t.copy_(i32(lengths))
    idx = ck.evict_paged(dw.t, i32(tables), dl.t, dK.t, dV.t, w, c, budget, out_idx=di.t)
    ww, ll, kk, vv, ii = ora.evict(weights, tables, lengths, K, V, w, c, budget)
    assert np.array_equal(idx.cpu().numpy(), ii)
    assert np.array_equal(dl.t.cpu().numpy(), ll) and np.array_equal(dw.t.cpu().numpy(), ww, equal_nan=True)
    assert torch.equal(dK.t.view(torch.int16), to_dev(kk).view(torch.int16)) and torch.equal(dV.t.view(torch.int16), to_dev(vv).view(torch.int16))
    for g in (dK, dV, dw, dl, di):
        g.check()


def some_weights(rng, shape, kind):
    if kind == "spread":
        return np.exp(rng.standard_normal(shape) * 3)
    if kind == "ties":
        return rng.integers(0, 3, shape)
    if kind == "equal":
        return np.full(shape, 0.25)
    x = rng.standard_normal(shape)
    x[rng.random(shape) < 0.02] = np.nan
    x[rng.random(shape) < 0.02] = np.inf
    x[rng.random(shape) < 0.02] = -np.inf
    x[rng.random(shape) < 0.2] = -0.0
    return x


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("w,c,budget", [(4, 1, 60), (0, 1, 1), (32, 10, 100), (16, 16, 64), (5, 3, 7), (1, 7, 133), (50, 20, 69), (100, 1, 101)])
def test_eviction(kind, w, c, budget):
    rng = np.random.default_rng(budget + c)
    B, Hkv, d, page, per = 3, 4, 64, 16, 12
    lengths = rng.integers(0, per * page + 1, (B, Hkv)).astype(np.int32)
    lengths[0] = [budget, budget + 1, per * page, 0]
    lengths[1, :2] = [-4, per * page + 100]
    check_eviction(rng, B, Hkv, d, page, per, lengths, w, c, budget, some_weights(rng, (B, Hkv, per * page), kind))


@pytest.mark.parametrize("B,Hkv,d,page,per,w,c,frac", [(1, 8, 128, 16, 230, 32, 10, 0.9), (40, 8, 64, 8, 20, 8, 4, 0.5), (1, 1, 128, 100, 90, 64, 1, 0.97),
                                                       (2, 3, 128, 1, 700, 300, 2, 0.6), (1, 2, 64, 64, 1000, 16, 1, 0.5), (80, 4, 128, 16, 9, 16, 1, 0.9)])
def test_eviction_of_short_and_long_heads(B, Hkv, d, page, per, w, c, frac):
    """One CTA a head up to eight; keys in shared memory and, for the longest, read again from the sums."""
    rng = np.random.default_rng(per)
    cap = per * page
    lengths = (cap - rng.integers(0, 9, (B, Hkv))).astype(np.int32)
    weights = np.exp(rng.standard_normal((B, Hkv, cap)) * 2)
    weights[rng.random(weights.shape) < 0.1] = 0
    check_eviction(rng, B, Hkv, d, page, per, lengths, w, c, int(cap * frac), weights)


def test_eviction_with_pages_outside_the_cache():
    rng = np.random.default_rng(3)
    lengths = np.full((2, 2), 96, dtype=np.int32)
    check_eviction(rng, 2, 2, 64, 8, 12, lengths, 6, 2, 50, rng.random((2, 2, 96)), holes=[(0, 2, -1), (0, 9, 1000), (1, 11, -2**31), (1, 0, 2**31 - 1)])


def test_eviction_again_changes_nothing():
    rng = np.random.default_rng(4)
    K, V, tables = new_cache(rng, 2, 2, 64, 16, 8)
    w = torch.rand(2, 2, 128, device="cuda")
    dl, t, dK, dV = i32(np.full((2, 2), 128)), i32(tables), to_dev(K), to_dev(V)
    ck.evict_paged(w, t, dl, dK, dV, 16, 4, 80)
    kept = [x.clone() for x in (w, dl, dK, dV)]
    idx = ck.evict_paged(w, t, dl, dK, dV, 16, 4, 80)
    assert all(torch.equal(a, b) for a, b in zip(kept, (w, dl, dK, dV)))
    assert torch.equal(idx, torch.arange(80, device="cuda", dtype=torch.int32).expand(2, 2, 80))


def test_calls_with_nothing_to_do():
    """No sequence at all, and a batch of padding: nothing is written but zeros and what stays."""
    Hq, Hkv, d = 4, 2, 64
    K, V = (torch.full((3, 16, Hkv, d), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cos, sin = (torch.tensor(x).cuda() for x in angles(4, d))
    for B in (0, 2):
        table, lengths = torch.zeros(B, 2, device="cuda", dtype=torch.int32), torch.zeros(B, Hkv, device="cuda", dtype=torch.int32)
        w = torch.zeros(B, Hkv, 32, device="cuda")
        q = ck.append_paged(torch.ones(B, (Hq + 2 * Hkv) * d, device="cuda", dtype=torch.bfloat16), Hq, cos, sin, torch.zeros(B, device="cuda", dtype=torch.int32),
                            table, lengths, K, V)
        out = ck.attend_paged(q, table, lengths, K, V, w)
        idx = ck.evict_paged(w, table, lengths, K, V, 2, 1, 4)
        assert q.shape == out.shape == (B, Hq, d) and not out.any() and not w.any() and not lengths.any()
        assert idx.shape == (B, Hkv, 4) and (idx == -1).all() and (K == 7).all() and (V == 7).all()


@pytest.mark.parametrize("B,Hq,Hkv", [(1, 65535, 1), (1, 4099, 4099), (9001, 1, 1), (2, 65534, 32767)])
def test_very_many_heads_and_sequences(B, Hq, Hkv):
    """As many query heads as there may be, of one KV head and of many; more sequences than any launch has CTAs at once."""
    rng = np.random.default_rng(B + Hkv)
    d, page, per = 64, 4, 2
    K, V, tables = new_cache(rng, B, Hkv, d, page, per, spare=1)
    lengths = rng.integers(0, page * per + 1, (B, Hkv)).astype(np.int32)
    check_attention(rand_bits(rng, (B, Hq, d)), K, V, tables, lengths, rng.random((B, Hkv, page * per)).astype(np.float32))
    # appended: every head's last row is the token's, and nothing else changed
    dK, dV, cos, sin = to_dev(K), to_dev(V), torch.ones(1, d // 2, device="cuda"), torch.zeros(1, d // 2, device="cuda")
    qkv, zeros = to_dev(rand_bits(rng, (B, (Hq + 2 * Hkv) * d))), torch.zeros(B, device="cuda", dtype=torch.int32)
    q = ck.append_paged(qkv, Hq, cos, sin, zeros, i32(tables), i32(lengths), dK, dV)
    assert torch.equal(q.flatten(1), qkv[:, :Hq * d])
    b, h = np.nonzero(lengths)
    at = lengths[b, h] - 1
    p, s = tables[b, at // page], at % page
    want_K, want_V = to_dev(K), to_dev(V)
    heads = qkv.view(B, -1, d)
    want_K[p, s, h], want_V[p, s, h] = heads[b, Hq + h], heads[b, Hq + Hkv + h]
    assert torch.equal(dK, want_K) and torch.equal(dV, want_V)
    check_eviction(rng, B, Hkv, d, page, per, lengths, 1, 1, 5, rng.random((B, Hkv, page * per)))


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("captured", [False, True])
def test_decoding_on_a_compressed_cache(captured):
    """Two prompts are compressed into a paged cache (their clipped last chunk kept by some heads), then ten tokens are appended and attended to; after
    the fifth the cache goes back to its budget. Everything against the formulas on the cache that they leave."""
    Hq, Hkv, d, w, c, budget, page, per, B, steps = 8, 2, 64, 8, 10, 68, 16, 6, 2, 10
    rng = np.random.default_rng(11)
    row = (Hq + 2 * Hkv) * d
    cos, sin = angles(600, d, 3)
    dcos, dsin = torch.tensor(cos).cuda(), torch.tensor(sin).cuda()
    gain = rand_bits(rng, (d,), 0.3)
    dgain = to_dev(gain)
    pages = B * per + 2
    cK, cV = torch.zeros(pages, page, Hkv, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(pages, page, Hkv, d, dtype=torch.bfloat16, device="cuda")
    tables = rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32)
    dtab = i32(tables)
    lengths = []
    prompts = [313, 405]
    for b, L in enumerate(prompts):
        qkv = to_dev(rand_bits(rng, (L, row)))
        qkv[L - 12:, Hq * d:(Hq + Hkv) * d - d] *= 3                        # the first head's last rows draw attention: it keeps the clipped chunk
        K = torch.empty(Hkv, L, d, dtype=torch.bfloat16, device="cuda")
        q, _ = ck.rotate_qk(qkv, Hq, Hkv, d, dcos, dsin, torch.arange(L, device="cuda", dtype=torch.int32), dgain, dgain, out_k=K.permute(1, 0, 2))
        V = qkv[:, (Hq + Hkv) * d:].view(L, Hkv, d).permute(1, 0, 2).contiguous()
        idx = ck.compress_layer_paged(q[-w:].permute(1, 0, 2).contiguous(), K, V, Hq, w, c, budget, dtab[b], cK, cV)
        lengths.append((idx >= 0).sum(1, dtype=torch.int32))
    dl = torch.stack(lengths)
    weights = torch.zeros(B, Hkv, per * page, device="cuda")
    pos = i32(prompts)
    x = torch.empty(B, row, dtype=torch.bfloat16, device="cuda")

    def step():
        dl.add_(1)
        q = ck.append_paged(x, Hq, dcos, dsin, pos, dtab, dl, cK, cV, dgain, dgain)
        out = ck.attend_paged(q, dtab, dl, cK, cV, weights)
        pos.add_(1)
        return q, out

    replay = None
    if captured:
        state = [t.clone() for t in (dl, pos, cK, cV, weights)]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            x.zero_()
            step()
        torch.cuda.current_stream().wait_stream(s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held = step()
        for t, v in zip((dl, pos, cK, cV, weights), state):
            t.copy_(v)
        replay = lambda: (g.replay(), held)[1]
    sums = np.zeros(weights.shape)
    for i in range(steps):
        bits = rand_bits(rng, (B, row))
        x.copy_(to_dev(bits))
        n0 = dl.cpu().numpy().copy()
        before = cK.clone()
        q, out = replay() if replay else step()
        torch.cuda.synchronize()
        heads = wide(bits).reshape(B, -1, d)
        at = np.array([p + i for p in prompts])
        ref, tol = rotated(heads[:, :Hq], wide(gain), 1e-6, cos[at].astype(np.float64), sin[at].astype(np.float64))
        assert (np.abs(f64(q) - ref) <= tol).all()
        kref, ktol = rotated(heads[:, Hq:Hq + Hkv], wide(gain), 1e-6, cos[at].astype(np.float64), sin[at].astype(np.float64))
        K, V = f64(cK), f64(cV)
        for b in range(B):
            for h in range(Hkv):
                p, s = ora.place(tables[b], int(n0[b, h]), page, pages)
                assert (np.abs(K[p, s, h] - kref[b, h]) <= ktol[b, h]).all() and np.array_equal(V[p, s, h], heads[b, Hq + Hkv + h])
                before[p, s, h] = cK[p, s, h]
        assert torch.equal(before, cK)
        want, got = ora.attend(f64(q), K, V, tables, n0 + 1)
        sums += got
        most = ora.attend(f64(q), K, np.abs(V), tables, n0 + 1)[0]
        assert (np.abs(f64(out) - want) <= U * np.abs(want) + 1e-4 * most).all()
        assert np.allclose(f64(weights), sums, rtol=1e-4, atol=1e-7)
        if i == 4:
            before = [f64(t) for t in (cK, cV)]
            W, n1 = weights.cpu().numpy(), dl.cpu().numpy()
            idx = ck.evict_paged(weights, dtab, dl, cK, cV, w, c, budget).cpu().numpy()
            ww, ll, kk, vv, ii = ora.evict(W, tables, n1, *before, w, c, budget)
            assert np.array_equal(ii, idx) and np.array_equal(ll, dl.cpu().numpy()) and (ll <= budget).all() and (n1 > budget).any()
            assert np.array_equal(kk, f64(cK)) and np.array_equal(vv, f64(cV)) and np.array_equal(ww, weights.cpu().numpy())
            sums = f64(weights)
    assert ck.device_status() == 0
