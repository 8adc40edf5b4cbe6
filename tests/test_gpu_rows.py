"""Rotary tables and layouts, turns of many tokens and shared prefixes, against oracle/rows_oracle.py in 64 bits. Tolerances: tests/rows_bounds.py."""
import numpy as np
import pytest
import torch

import paper_2502_00299_b200 as ck
from oracle import rows_oracle as ora
from tests import rows_bounds
from tests.decode_bounds import wide
from tests.helpers import Guarded, bits_of, rand_bits, to_dev

pytestmark = pytest.mark.gpu
U, E = 2.0 ** -8, 2.0 ** -24


def i32(x):
    return torch.tensor(np.ascontiguousarray(x).astype(np.int32), device="cuda")


def values(t):
    return wide(bits_of(t))


@pytest.fixture(autouse=True)
def no_abandoned_wait():
    yield
    assert ck.device_status() == 0


# ------------------------------------------------------------------------------------------------ tables
# A pair's angle is good to 2^-31 of a turn, 3e-9; the 32-bit fraction of an eighth of a turn, its product with 2 pi and two series of at most five products and
# sums round by 2^-24 each: 2^-22 of the scale bounds them.
@pytest.mark.parametrize("n,rot,first", [(1, 16, 0), (7, 128, 0), (1000, 48, 12345), (3, 96, -5), (4097, 32, 1 << 20), (300, 64, (1 << 31) - 10)])
@pytest.mark.parametrize("kind,factor,low,high", [("none", 1.0, 0.0, 0.0), ("linear", 3.0, 0.0, 0.0), ("dims", 8.0, 1.0, 32.0), ("waves", 4.0, 1.0, 4.0)])
def test_tables(n, rot, first, kind, factor, low, high):
    want = ora.tables(n, rot, 10000.0, kind, factor, 4096.0, low, high, 1.25, first)
    got = ck.rope_tables(n, rot, 10000.0, kind, factor, 4096.0, low, high, 1.25, first)
    # (the reference's own angles are products in 64 bits: 2^-53 of up to 2^31 rad)
    for g, w in zip(got, want):
        assert g.shape == (n, rot // 2) and np.abs(g.cpu().numpy() - w).max() <= 1.25 * (2.0 ** -22 + 2.0 ** -52 * abs(first))


def test_tables_into_given_outputs():
    c, s = Guarded((33, 8), torch.float32), Guarded((33, 8), torch.float32)
    r = ck.rope_tables(33, 16, 500000.0, out_cos=c.t, out_sin=s.t)
    assert r[0] is c.t and r[1] is s.t
    c.check(); s.check()
    w = ora.tables(33, 16, 500000.0)
    assert np.abs(c.t.cpu().numpy() - w[0]).max() <= 2.0 ** -22 and np.abs(s.t.cpu().numpy() - w[1]).max() <= 2.0 ** -22
    assert ck.rope_tables(0, 16, 10.0)[0].shape == (0, 8)


# ------------------------------------------------------------------------------------------------ rotations
def angles(rng, n_pos, rot):
    a = rng.uniform(-3, 3, (n_pos, rot // 2))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def rotated(x, gain, eps, cos, sin, inter):
    """(values, tolerance): products and sums in 32 bits - the norm's sum of at most 128 squares, its root, two products, then two products and a
    sum, 2^-24 each, 100 of them - and one rounding."""
    y = ora.rotate(x, gain, eps, cos, sin, inter)
    size = ora.rotate(np.abs(x), None if gain is None else np.abs(gain), eps, np.abs(cos), -np.abs(sin), inter)
    size = np.maximum(size, ora.rotate(np.abs(x), None if gain is None else np.abs(gain), eps, np.abs(cos), np.abs(sin), inter))
    return y, U * np.abs(y) + (1 + U) * 100 * E * np.abs(size)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,norm", [(1, 1, 1, 64, 16, False), (5, 8, 2, 64, 32, True), (37, 7, 1, 128, 128, True), (130, 12, 4, 128, 48, False),
                                                (2000, 32, 8, 128, 64, True), (3, 6, 3, 64, 64, False), (9, 5, 5, 128, 112, True)])
def test_rotate(T, Hq, Hkv, d, rot, norm, inter):
    rng = np.random.default_rng(T + rot)
    row = (Hq + 2 * Hkv) * d + 8
    x = rand_bits(rng, (T, row))
    gq, gk = (rand_bits(rng, d), rand_bits(rng, d)) if norm else (None, None)
    cos, sin = angles(rng, 50, rot)
    pos = rng.integers(0, 50, T)
    pos[T // 2] = -1 if T > 2 else pos[T // 2]
    q, k = ck.rotate_rows(to_dev(x), Hq, Hkv, d, torch.tensor(cos).cuda(), torch.tensor(sin).cuda(), i32(pos), inter,
                          to_dev(gq) if norm else None, to_dev(gk) if norm else None, 1e-5)
    heads = wide(x[:, :(Hq + Hkv) * d]).reshape(T, Hq + Hkv, d)
    at = np.maximum(pos, 0)
    for got, part, gain in ((q, heads[:, :Hq], gq), (k, heads[:, Hq:], gk)):
        want, tol = rotated(part, wide(gain) if norm else None, 1e-5, cos[at].astype(np.float64)[:, None], sin[at].astype(np.float64)[:, None], inter)
        want[pos < 0] = 0.0
        assert (np.abs(values(got) - want) <= tol).all()
    if not norm:
        assert np.array_equal(bits_of(q)[pos >= 0][..., rot:], x[:, :Hq * d].reshape(T, Hq, d)[pos >= 0][..., rot:])


@pytest.mark.parametrize("inter", [False, True])
def test_rotate_in_place_and_head_major(inter):
    T, Hq, Hkv, d, rot = 19, 6, 2, 128, 64
    rng = np.random.default_rng(8)
    x = rand_bits(rng, (T, (Hq + 2 * Hkv) * d))
    cos, sin = (torch.tensor(t).cuda() for t in angles(rng, 40, rot))
    pos = i32(rng.integers(0, 40, T))
    qkv = to_dev(x)
    q, k = ck.rotate_rows(qkv, Hq, Hkv, d, cos, sin, pos, inter)
    K = torch.zeros(Hkv, T, d, dtype=torch.bfloat16, device="cuda")
    view = qkv.view(T, Hq + 2 * Hkv, d)
    ck.rotate_rows(qkv, Hq, Hkv, d, cos, sin, pos, inter, out_q=view[:, :Hq], out_k=K.permute(1, 0, 2))
    assert torch.equal(view[:, :Hq], q) and torch.equal(K.permute(1, 0, 2), k)
    assert np.array_equal(bits_of(qkv)[:, Hq * d:], x[:, Hq * d:])


def test_whole_heads_in_halves_are_rotate_qk():
    T, Hq, Hkv, d = 300, 8, 2, 128
    rng = np.random.default_rng(9)
    x, g = to_dev(rand_bits(rng, (T, (Hq + 2 * Hkv) * d))), to_dev(rand_bits(rng, d))
    cos, sin = (torch.tensor(t).cuda() for t in angles(rng, 40, d))
    pos = i32(rng.integers(0, 40, T))
    for a, b in zip(ck.rotate_rows(x, Hq, Hkv, d, cos, sin, pos, False, g, g), ck.rotate_qk(x, Hq, Hkv, d, cos, sin, pos, g, g)):
        assert torch.equal(a, b)


def test_dims_that_stay_and_rows_that_turn_may_be_infinite():
    x = np.full((2, 3 * 64), 0x3F80, dtype=np.uint16)
    x[0, 40], x[0, 64 + 3] = 0x7F80, 0x7FC0
    one, none = torch.ones(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda")
    for inter in (False, True):
        q, k = ck.rotate_rows(to_dev(x), 1, 1, 64, one, none, i32([0, 1]), inter)
        q, k = values(q), values(k)
        assert q[0, 0, 40] == np.inf and np.isfinite(np.delete(q[0, 0], 40)).all() and np.isnan(k[0, 0, 3])
        assert np.isnan(k[0, 0]).sum() == 2 and (q[1] == 1).all() and (k[1] == 1).all()         # (it and the one that it turns with)


# ------------------------------------------------------------------------------------------------ appended rows
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rot,B,norm,page", [(64, 32, 1, False, 16), (128, 128, 3, True, 5), (128, 48, 40, False, 16), (64, 64, 1100, True, 3)])
def test_append(d, rot, B, norm, page, inter):
    Hq, Hkv, per = 6, 2, 6
    rng = np.random.default_rng(B)
    n = rng.integers(0, 9, B) if B > 1 else np.array([13])
    if B > 2:
        n[1] = 0
    starts = 2 + np.r_[0, np.cumsum(n)]                                      # (tokens in front of all sequences and behind them)
    T = int(starts[-1]) + 3
    pages = B * per + 3
    K0, V0 = rand_bits(rng, (pages, page, Hkv, d)), rand_bits(rng, (pages, page, Hkv, d))
    table = rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32)
    lengths = np.clip(n[:, None] + rng.integers(-3, per * page - 9, (B, Hkv)), 0, None)      # some have fewer rows than new tokens
    if B > 1:
        table[0, 0], lengths[B - 1, 1] = -1, per * page + 2                  # a page that is not there; rows beyond the table
    x = rand_bits(rng, (T, (Hq + 2 * Hkv) * d))
    g = rand_bits(rng, d) if norm else None
    cos, sin = angles(rng, 50, rot)
    pos = rng.integers(0, 50, T)
    K, V, oq = Guarded(K0.shape, torch.bfloat16), Guarded(V0.shape, torch.bfloat16), Guarded((T, Hq, d), torch.bfloat16)
    K.t.copy_(to_dev(K0)); V.t.copy_(to_dev(V0)); oq.t.fill_(7.0)
    gain = to_dev(g) if norm else None
    r = ck.append_rows_paged(to_dev(x), Hq, i32(starts), torch.tensor(cos).cuda(), torch.tensor(sin).cuda(), i32(pos), i32(table), i32(lengths), K.t, V.t,
                             inter, gain, gain, 1e-5, oq.t)
    assert r is oq.t
    K.check("K"); V.check("V"); oq.check("q")
    heads = wide(x).reshape(T, Hq + 2 * Hkv, d)
    c, s = cos[pos].astype(np.float64)[:, None], sin[pos].astype(np.float64)[:, None]
    q, q_tol = rotated(heads[:, :Hq], wide(g) if norm else None, 1e-5, c, s, inter)
    k, k_tol = rotated(heads[:, Hq:Hq + Hkv], wide(g) if norm else None, 1e-5, c, s, inter)
    got_q, got_K, got_V = values(oq.t), bits_of(K.t), bits_of(V.t)
    at = ora.append_places(starts, T, table, lengths, page, pages)
    same = np.ones(K0.shape[:3], dtype=bool)
    for t in range(T):
        if at[t] is None:
            assert (got_q[t] == 7.0).all()
            continue
        assert (np.abs(got_q[t] - q[t]) <= q_tol[t]).all()
        for h in range(Hkv):
            if at[t][h] is not None:
                p, slot = at[t][h]
                same[p, slot, h] = False
                assert (np.abs(wide(got_K[p, slot, h]) - k[t, h]) <= k_tol[t, h]).all()
                assert np.array_equal(got_V[p, slot, h], x[t].reshape(-1, d)[Hq + Hkv + h])
    assert np.array_equal(got_K[same], K0[same]) and np.array_equal(got_V[same], V0[same])


def test_one_token_each_is_append_paged():
    B, Hq, Hkv, d, page, per = 9, 8, 2, 128, 16, 3
    rng = np.random.default_rng(11)
    x = to_dev(rand_bits(rng, (B, (Hq + 2 * Hkv) * d)))
    cos, sin = (torch.tensor(t).cuda() for t in angles(rng, 40, d))
    pos, table, lengths = i32(rng.integers(0, 40, B)), i32(rng.permutation(B * per).reshape(B, per)), i32(rng.integers(0, 49, (B, Hkv)))
    caches = [[torch.zeros(B * per, page, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2)]
    a = ck.append_paged(x, Hq, cos, sin, pos, table, lengths, *caches[0])
    b = ck.append_rows_paged(x, Hq, i32(np.arange(B + 1)), cos, sin, pos, table, lengths, *caches[1])
    assert torch.equal(a, b) and torch.equal(caches[0][0], caches[1][0]) and torch.equal(caches[0][1], caches[1][1])


# ------------------------------------------------------------------------------------------------ attention of turns
def paged(rng, B, Hkv, d, page, per, spare=3, counting=False):
    pages = B * per + spare
    if counting:                                                             # keys of zeros, values of small whole numbers
        from workloads import f32_to_bf16_bits
        K = np.zeros((pages, page, Hkv, d), dtype=np.uint16)
        V = f32_to_bf16_bits(rng.integers(-8, 9, K.shape).astype(np.float32))
    else:
        K, V = rand_bits(rng, (pages, page, Hkv, d)), rand_bits(rng, (pages, page, Hkv, d))
    return K, V, rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32)


def attend(q, starts, K, V, table, lengths, causal):
    out = Guarded(q.shape, torch.bfloat16)
    out.t.fill_(7.0)
    args = to_dev(q), i32(starts), i32(table), i32(lengths), to_dev(K), to_dev(V), causal
    r = ck.attend_rows_paged(*args, out.t)
    assert r is out.t
    out.check("out")
    assert torch.equal(bits(ck.attend_rows_paged(*args, out=torch.full_like(out.t, 7.0))), bits(out.t))      # same result every time
    return values(out.t)


def bits(t):
    return t.view(torch.int16)


COUNT = [   # Hq, Hkv, d, page, tokens, rows before them (a list: of each head)
    (1, 1, 64, 16, [1], [0]),
    (1, 1, 128, 16, [1], [1]),
    (4, 1, 128, 16, [1, 1], [127, 128]),
    (8, 2, 64, 8, [3, 0, 5], [0, 7, 300]),
    (8, 2, 128, 100, [130, 1, 77], [5, 1000, 129]),
    (7, 1, 128, 5, [64, 40], [33, 500]),
    (12, 4, 64, 64, [300], [1200]),
    (6, 6, 64, 16, [257, 255, 256], [0, 1, 640]),
    (40, 2, 128, 1, [9, 30], [200, 11]),
    (200, 1, 128, 16, [3, 0, 1], [300, 4, 77]),
    (130, 1, 64, 32, [2], [129]),
    (300, 1, 64, 16, [3, 2], [200, 50]),                                     # more query heads than a block holds
    (16, 2, 128, 32, [1] * 40, list(range(0, 800, 20))),
    (4, 2, 128, 16, [700], [2500]),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("Hq,Hkv,d,page,n,before", COUNT)
def test_every_row_counts_once(Hq, Hkv, d, page, n, before, causal):
    """Logits of 0: means of what is seen."""
    rng = np.random.default_rng(sum(n) + d)
    B = len(n)
    starts = 1 + np.r_[0, np.cumsum(n)]
    T = int(starts[-1]) + 2
    lengths = np.array([[max(0, n[b] + before[b] - 3 * (h % 2)) for h in range(Hkv)] for b in range(B)])
    per = -(-int(lengths.max()) // page) + 1
    K, V, table = paged(rng, B, Hkv, d, page, per, counting=True)
    q = rand_bits(rng, (T, Hq, d))
    out = attend(q, starts, K, V, table, lengths, causal)
    ref = np.full(q.shape, 7.0)
    G, v = Hq // Hkv, wide(V)
    for b in range(B):
        for h in range(Hkv):
            L = lengths[b, h]
            rows = v[table[b, np.arange(L) // page], np.arange(L) % page, h]
            sums = np.concatenate([np.zeros((1, d)), np.cumsum(rows, 0)])
            for i in range(n[b]):
                m = max(L - (n[b] - 1 - i), 0) if causal else L
                ref[starts[b] + i, h * G:(h + 1) * G] = sums[m] / max(m, 1)
    rows_bounds.count_rows(out, ref)


RANDOM = [
    (1, 1, 64, 16, [1], [0]),
    (8, 2, 128, 16, [5, 1, 9], [300, 0, 77]),
    (7, 1, 64, 100, [64, 3], [260, 900]),
    (8, 8, 128, 16, [130], [400]),
    (32, 4, 128, 64, [33, 0, 17], [1000, 5, 2000]),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("scale", [1.0, 6.0])
@pytest.mark.parametrize("Hq,Hkv,d,page,n,before", RANDOM)
def test_attention_of_a_turn(Hq, Hkv, d, page, n, before, scale, causal):
    rng = np.random.default_rng(sum(n) + d + Hq)
    B = len(n)
    starts = np.r_[0, np.cumsum(n)]
    lengths = np.array([[max(0, n[b] + before[b] - 3 * (h % 2)) for h in range(Hkv)] for b in range(B)])
    per = -(-int(lengths.max()) // page)
    K, V, table = paged(rng, B, Hkv, d, page, per)
    if page == 16:                                                           # rows in no page
        table[0, per // 2] = -1
    q = rand_bits(rng, (int(starts[-1]), Hq, d), scale)
    out = attend(q, starts, K, V, table, lengths, causal)
    rows_bounds.check_attend(out, wide(q), starts, wide(K), wide(V), table, lengths, causal)


def put(K, table, b, row, h, dims, what):
    page = K.shape[1]
    K[table[b, row // page], row % page, h, dims] = what


@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_are_not_seen_do_not_matter(d):
    """Infinities, not-a-number and the largest numbers behind lengths, in nobody's pages, and in the turn's own rows behind a token."""
    Hq, Hkv, page, B, n = 8, 2, 16, 3, [150, 5, 40]
    rng = np.random.default_rng(21)
    starts = np.r_[0, np.cumsum(n)]
    lengths = np.array([[400, 391], [5, 3], [300, 260]])
    per = 26
    K, V, table = paged(rng, B, Hkv, d, page, per)
    table[2, 3] = -1
    used = np.zeros(K.shape[:3], dtype=bool)
    for b in range(B):
        for h in range(Hkv):
            j = np.arange(lengths[b, h])
            p = table[b, j // page]
            used[p[p >= 0], (j % page)[p >= 0], h] = True
    bad = np.array([0x7FC0, 0x7F80, 0xFF80, 0x7F7F, 0xFF7F], dtype=np.uint16)
    for x in (K, V):
        x[~used] = rng.choice(bad, (int((~used).sum()), d))
    q = rand_bits(rng, (int(starts[-1]), Hq, d))
    for causal in (False, True):
        out = attend(q, starts, K, V, table, lengths, causal)
        rows_bounds.check_attend(out, wide(q), starts, wide(K), wide(V), table, lengths, causal)
    # values of the turn that later tokens only see: those dims are no numbers from there on, and nothing else changes
    bad_rows = [(0, 300, 0, [1, d - 1], 0x7F80), (0, 393, 0, [5], 0x7FC0), (0, 250, 1, [0, 33], 0xFF80), (1, 4, 0, [7], 0x7FC0), (2, 259, 1, [2], 0x7F80)]
    clean = attend(q, starts, K, V, table, lengths, True)
    for b, row, h, dims, what in bad_rows:
        put(V, table, b, row, h, dims, what)
    out = attend(q, starts, K, V, table, lengths, True)
    want = np.zeros(out.shape, dtype=bool)
    for b, row, h, dims, _ in bad_rows:
        for i in range(n[b]):
            if row < lengths[b, h] - (n[b] - 1 - i):
                want[starts[b] + i, h * 4:(h + 1) * 4, dims] = True
    assert want.any() and np.array_equal(~np.isfinite(out), want) and np.array_equal(out[~want], clean[~want])


@pytest.mark.parametrize("d", [64, 128])
def test_logits_that_are_not_finite(d):
    """-inf in some rows and in whole tiles, in every row, one of +inf, one that is no number, logits of +-1e4, and ordinary ones beside them."""
    page, Hkv, G, rows = 16, 6, 3, 500
    rng = np.random.default_rng(22)
    K, V, table = paged(rng, 1, Hkv, d, page, 32)
    q = rand_bits(rng, (20, Hkv * G, d))
    q[..., 0] = 0x3F80                                                       # 1.0
    j = np.arange(rows)
    p, s = table[0, j // page], j % page
    some = (j % 3 != 0) | ((j >= 128) & (j < 300))
    K[p[some], s[some], 0, 0] = 0xFF80
    K[p, s, 1, 0] = 0xFF80
    K[p[50], s[50], 2, 0] = 0x7F80
    K[p, s, 3] = 0
    K[p, s, 3, 0] = np.where(j == 333, 0x47C3, 0xC7C3)                       # +-99840
    K[p[70], s[70], 4, 3] = 0x7FC0
    lengths = np.full((1, Hkv), rows)
    out = attend(q, [0, 20], K, V, table, lengths, False)
    with np.errstate(all="ignore"):
        ref = ora.attend_rows(wide(q), [0, 20], wide(K), wide(V), table, lengths, False)
    assert np.array_equal(np.isnan(ref), np.isnan(out)) and not out[:, G:2 * G].any()
    for h in (0, 3, 5):
        k, v, at = ora.rows_of(wide(K), wide(V), table[0], rows, h)
        keep = np.isfinite(k).all(1)
        for g in range(h * G, (h + 1) * G):
            rows_bounds.check_rows(out[:, g], wide(q)[:, g], k[keep], v[keep], np.ones((20, int(keep.sum())), dtype=bool), (h, g))


def test_large_values_are_added_up_before_they_are_divided():
    rng = np.random.default_rng(23)
    K, V, table = paged(rng, 1, 1, 128, 16, 40)
    V[...] = 0x6B80                                                          # 2^88
    out = attend(rand_bits(rng, (9, 4, 128)), [0, 9], K, V, table, np.array([[600]]), True)
    assert (np.abs(out / 2.0 ** 88 - 1) <= 2 * U).all()


# ------------------------------------------------------------------------------------------------ shared prefixes
def shared(q, starts, K, V, pt, pl, table, lengths):
    out = Guarded(q.shape, torch.bfloat16)
    out.t.fill_(7.0)
    args = to_dev(q), i32(starts), i32(pt), i32(pl), i32(table), i32(lengths), to_dev(K), to_dev(V)
    assert ck.attend_shared_paged(*args, out.t) is out.t
    out.check("out")
    assert torch.equal(bits(ck.attend_shared_paged(*args)), bits(out.t))     # same result every time
    return values(out.t)


SHARED = [  # Hq, Hkv, d, page, sequences of each group, prefix rows, own rows (most), sequences of no group in front and behind
    (1, 1, 64, 16, [1], [0], 0, 0, 0),
    (4, 1, 128, 16, [1], [1], 1, 0, 0),
    (8, 2, 128, 8, [3, 0, 5], [300, 7, 128], 40, 2, 1),
    (7, 1, 64, 100, [40], [1000], 200, 0, 0),
    (32, 8, 128, 16, [64], [700], 30, 0, 0),
    (28, 4, 64, 5, [30, 7, 50], [257, 1500, 0], 129, 0, 3),
    (200, 1, 64, 16, [3], [300], 60, 1, 1),
    (300, 1, 128, 16, [2, 1], [400, 100], 60, 1, 0),                         # more query heads than a block holds
    (6, 6, 64, 64, [300], [900], 3, 0, 0),
    (16, 2, 64, 16, [], [], 90, 5, 0),                                       # no prefix at all
]


@pytest.mark.parametrize("counting", [True, False])
@pytest.mark.parametrize("Hq,Hkv,d,page,sizes,prefix,own,front,back", SHARED)
def test_shared_prefixes(Hq, Hkv, d, page, sizes, prefix, own, front, back, counting):
    rng = np.random.default_rng(Hq + d + own)
    B, P = front + sum(sizes) + back, len(sizes)
    starts = front + np.r_[0, np.cumsum(sizes)].astype(int)
    lengths = rng.integers(0, own + 1, (B, Hkv))
    lengths[rng.random((B, Hkv)) < 0.2] = 0
    pl = np.array([[max(0, x - 3 * (h % 2)) for h in range(Hkv)] for x in prefix]).reshape(P, Hkv)
    per, per_pre = max(1, -(-own // page)), max(1, -(-max(prefix, default=0) // page))
    K, V, all_ = paged(rng, 1, Hkv, d, page, B * per + P * per_pre, counting=counting)
    table, pt = all_[0, :B * per].reshape(B, per), all_[0, B * per:].reshape(P, per_pre)
    q = rand_bits(rng, (B, Hq, d), 2.0)
    if page == 8:                                                            # pages that are not there
        pt[0, 2], table[3, 0] = -1, len(K)
    out = shared(q, starts, K, V, pt, pl, table, lengths)
    if not counting:
        rows_bounds.check_shared(out, wide(q), starts, wide(K), wide(V), pt, pl, table, lengths)
        return
    rows_bounds.count_rows(out, ora.attend_shared(np.zeros(q.shape), starts, np.zeros(K.shape), wide(V), pt, pl, table, lengths))


def test_a_prefix_of_infinite_logits_leaves_the_own_rows():
    rng = np.random.default_rng(31)
    K, V, all_ = paged(rng, 1, 1, 64, 16, 30)
    pt, table = all_[:, :20], all_[0, 20:30].reshape(2, 5)
    q = rand_bits(rng, (2, 4, 64))
    q[..., 0] = 0x3F80
    for p in pt[0]:
        K[p, :, 0, 0] = 0xFF80
    out = shared(q, [0, 2], K, V, pt, np.array([[320]]), table, np.array([[70], [0]]))
    assert not out[1].any()
    k, v, _ = ora.rows_of(wide(K), wide(V), table[0], 70, 0)
    rows_bounds.check_rows(out[0], wide(q)[0], k, v, np.ones((4, 70), dtype=bool))


# ------------------------------------------------------------------------------------------------ as they are used
def turn_inputs(rng, Hq=8, Hkv=2, d=128, page=16, sizes=(40, 3, 130), before=(300, 7, 0), per=32):
    """A batch of conversations in one cache, a turn's activations, and tables of angles."""
    B = len(sizes)
    starts = np.r_[0, np.cumsum(sizes)]
    T = int(starts[-1])
    K, V, table = paged(rng, B, Hkv, d, page, per)
    lengths = np.array([[b + n for _ in range(Hkv)] for b, n in zip(before, sizes)])
    x = rand_bits(rng, (T, (Hq + 2 * Hkv) * d))
    pos = np.concatenate([b + np.arange(n) for b, n in zip(before, sizes)])
    return starts, K, V, table, lengths, x, pos


@pytest.mark.parametrize("inter", [False, True])
def test_a_turn_then_single_tokens_on_what_was_compressed(inter):
    """Tables, rotated prompts, compressed into pages; a turn appended and attended to; then a token each, over a shared prefix as over one table."""
    Hq, Hkv, d, page, L, w, c, budget = 8, 2, 128, 16, 1024, 16, 10, 256
    rng = np.random.default_rng(41)
    cos, sin = ck.rope_tables(2048, 64, 10000.0, "dims", 4.0, 512.0, 1.0, 32.0)
    x = to_dev(rand_bits(rng, (L, (Hq + 2 * Hkv) * d)))
    q, k = ck.rotate_rows(x, Hq, Hkv, d, cos, sin, i32(np.arange(L)), inter)
    K, V = k.permute(1, 0, 2).contiguous(), x.view(L, Hq + 2 * Hkv, d)[:, Hq + Hkv:].permute(1, 0, 2).contiguous()
    per, n = 24, 100
    cK, cV = (torch.zeros(2 * per, page, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = i32(rng.permutation(2 * per).reshape(2, per))
    idx = ck.compress_layer_paged(q[L - w:].permute(1, 0, 2).contiguous(), K, V, Hq, w, c, budget, table[0], cK, cV)
    kept = (idx >= 0).sum(1, dtype=torch.int32)
    # a turn of n tokens
    y = to_dev(rand_bits(rng, (n, (Hq + 2 * Hkv) * d)))
    pos = i32(L + np.arange(n))
    lengths = (kept + n)[None].contiguous()
    starts = i32([0, n])
    qt = ck.append_rows_paged(y, Hq, starts, cos, sin, pos, table[:1].contiguous(), lengths, cK, cV, inter)
    out = ck.attend_rows_paged(qt, starts, table[:1].contiguous(), lengths, cK, cV)
    args = values(qt), [0, n], values(cK), values(cV), table[:1].cpu().numpy(), lengths.cpu().numpy()
    rows_bounds.check_attend(values(out), *args, True)
    want, _ = ck.rotate_rows(y, Hq, Hkv, d, cos, sin, pos, inter)
    assert torch.equal(want, qt)
    # two sequences that share it, each with a token of its own, as rows of a second table
    own = torch.stack([table[1, :8], table[1, 8:16]]).contiguous()
    z = to_dev(rand_bits(rng, (2, (Hq + 2 * Hkv) * d)))
    one = torch.ones(2, Hkv, dtype=torch.int32, device="cuda")
    q1 = ck.append_rows_paged(z, Hq, i32([0, 1, 2]), cos, sin, i32([L + n] * 2), own, one, cK, cV, inter)
    got = ck.attend_shared_paged(q1, i32([0, 2]), table[:1].contiguous(), lengths, own, one, cK, cV)
    rows_bounds.check_shared(values(got), values(q1), [0, 2], values(cK), values(cV), table[:1].cpu().numpy(), lengths.cpu().numpy(), own.cpu().numpy(), np.ones((2, Hkv), int))


def test_streams_graphs_and_calls_side_by_side():
    """Two captured graphs and eager calls on other streams: nothing in common but the tensors given."""
    rng = np.random.default_rng(42)
    starts, K, V, table, lengths, x, pos = turn_inputs(rng)
    Hq = 8
    dK, dV, dt, dl, ds = to_dev(K), to_dev(V), i32(table), i32(lengths), i32(starts)
    q = to_dev(rand_bits(rng, (int(starts[-1]), Hq, 128)))
    qs = to_dev(rand_bits(rng, (3, Hq, 128)))
    one = i32([0, 3])
    want = ck.attend_rows_paged(q, ds, dt, dl, dK, dV)
    want_s = ck.attend_shared_paged(qs, one, dt[:1].contiguous(), dl[:1].contiguous(), dt, dl, dK, dV)
    graphs, outs = [], []
    for kind in (0, 1):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                o = ck.attend_rows_paged(q, ds, dt, dl, dK, dV) if kind == 0 else ck.attend_shared_paged(qs, one, dt[:1].contiguous(), dl[:1].contiguous(), dt, dl, dK, dV)
        graphs.append((g, s))
        outs.append(o)
    torch.cuda.synchronize()
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, s in graphs:
            with torch.cuda.stream(s):
                g.replay()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        a = ck.attend_rows_paged(q, ds, dt, dl, dK, dV, stream=side)
        b = ck.attend_shared_paged(qs, one, dt[:1].contiguous(), dl[:1].contiguous(), dt, dl, dK, dV)
        torch.cuda.synchronize()
        assert torch.equal(bits(outs[0]), bits(want)) and torch.equal(bits(outs[1]), bits(want_s)) and torch.equal(bits(a), bits(want)) and torch.equal(bits(b), bits(want_s))


def test_calls_directly_behind_one_another():
    """Appended rows, lengths and queries that the call ahead still writes, time after time, against calls one by one."""
    rng = np.random.default_rng(43)
    starts, K, V, table, lengths, x, pos = turn_inputs(rng)
    cos, sin = (torch.tensor(t).cuda() for t in angles(rng, 512, 128))
    dx, dp, dt, dl, ds = to_dev(x), i32(pos), i32(table), i32(lengths), i32(starts)
    q0 = i32([0, 1, 2, 3])

    def run(wait):
        cK, cV = to_dev(K), to_dev(V)
        res = []
        for _ in range(6):
            q = ck.append_rows_paged(dx, 8, ds, cos, sin, dp, dt, dl, cK, cV)
            if wait:
                torch.cuda.synchronize()
            o = ck.attend_rows_paged(q, ds, dt, dl, cK, cV)
            if wait:
                torch.cuda.synchronize()
            res += [ck.attend_shared_paged(o[:3].contiguous(), q0, dt, dl, dt, dl, cK, cV), ck.attend_paged(q[:3].contiguous(), dt, dl, cK, cV)]
            if wait:
                torch.cuda.synchronize()
            dx.copy_(dx.roll(1, 0))
        for _ in range(6):
            dx.copy_(dx.roll(-1, 0))
        torch.cuda.synchronize()
        return res

    for a, b in zip(run(True), run(False)):
        assert torch.equal(bits(a), bits(b))


def test_native_and_general_calls_agree(monkeypatch):
    from paper_2502_00299_b200 import binding
    rng = np.random.default_rng(44)
    starts, K, V, table, lengths, x, pos = turn_inputs(rng)
    cos, sin = (torch.tensor(t).cuda() for t in angles(rng, 512, 64))
    q = to_dev(rand_bits(rng, (int(starts[-1]), 8, 128)))

    def run():
        cK, cV = to_dev(K), to_dev(V)
        return [*ck.rope_tables(100, 64, 10000.0, "waves", 8.0, 512.0, 1.0, 4.0, first=7), *ck.rotate_rows(to_dev(x), 8, 2, 128, cos, sin, i32(pos), True),
                ck.append_rows_paged(to_dev(x), 8, i32(starts), cos, sin, i32(pos), i32(table), i32(lengths), cK, cV), cK, cV,
                ck.attend_rows_paged(q, i32(starts), i32(table), i32(lengths), cK, cV, False),
                ck.attend_shared_paged(q[:3].contiguous(), i32([0, 1, 3]), i32(table[:2]), i32(lengths[:2]), i32(table), i32(lengths), cK, cV)]

    native = run()

    class General:
        def __getattr__(self, name):
            return lambda *a: None

    monkeypatch.setattr(binding, "_native", General())
    for a, b in zip(native, run()):
        assert torch.equal(a, b)


@pytest.mark.parametrize("page", [16, 1000])
def test_rows_beyond_32_bits_of_a_long_cache(page):
    """Pages at the end of a cache of more than 2^32 bytes."""
    Hkv, d, per = 8, 128, max(1, 640 // page)
    pages = (1 << 33) // (page * Hkv * d * 2) // 2 + 8
    rng = np.random.default_rng(45)
    table = (pages - 1 - np.arange(per)).reshape(1, per)
    K = torch.zeros(pages, page, Hkv, d, dtype=torch.bfloat16, device="cuda")
    V = torch.zeros_like(K)
    rows = rand_bits(rng, (2, per, page, Hkv, d))
    K[pages - per:], V[pages - per:] = to_dev(rows[0]), to_dev(rows[1])
    n = 600
    q = rand_bits(rng, (20, 16, d))
    lengths = np.full((1, Hkv), n)
    out = values(ck.attend_rows_paged(to_dev(q), i32([0, 20]), i32(table), i32(lengths), K, V))
    local = per - 1 - np.arange(per)
    rows_bounds.check_attend(out, wide(q), [0, 20], wide(rows[0]), wide(rows[1]), local.reshape(1, per), lengths, True)
    got = values(ck.attend_shared_paged(to_dev(q), i32([0, 20]), i32(table), i32(lengths), i32(np.full((20, 1), -1)), i32(np.zeros((20, Hkv))), K, V))
    rows_bounds.check_shared(got, wide(q), [0, 20], wide(rows[0]), wide(rows[1]), local.reshape(1, per), lengths, np.full((20, 1), -1), np.zeros((20, Hkv), int))
    x = to_dev(rand_bits(rng, (1, 32 * d)))
    one = torch.ones(4, 64, device="cuda")
    ck.append_rows_paged(x, 16, i32([0, 1]), one, torch.zeros_like(one), i32([0]), i32(table), i32(lengths), K, V)
    assert torch.equal(V[pages - 1 - (n - 1) // page, (n - 1) % page], x.view(32, d)[24:])


def test_starts_that_make_no_sense_read_and_write_nothing_out_of_range():
    """Descending, negative and too large: whatever comes out, it is written inside of out, and the call ends."""
    rng = np.random.default_rng(46)
    starts, K, V, table, lengths, x, pos = turn_inputs(rng)
    T = int(starts[-1])
    q = to_dev(rand_bits(rng, (T, 8, 128)))
    cos, sin = (torch.tensor(t).cuda() for t in angles(rng, 512, 128))
    for bad in ([5, 3, 100, 20], [-7, 2, T + 500, 4], [T, T, T, T], [2**31 - 1, -2**31, 0, 9]):
        out, oq = Guarded((T, 8, 128), torch.bfloat16), Guarded((T, 8, 128), torch.bfloat16)
        cK, cV = Guarded(K.shape, torch.bfloat16), Guarded(V.shape, torch.bfloat16)
        cK.t.copy_(to_dev(K)); cV.t.copy_(to_dev(V))
        ck.attend_rows_paged(q, i32(bad), i32(table), i32(lengths), cK.t, cV.t, True, out.t)
        ck.attend_shared_paged(q[:3].contiguous(), i32(bad), i32(table), i32(lengths), i32(table), i32(lengths), cK.t, cV.t)
        ck.append_rows_paged(to_dev(x), 8, i32(bad), cos, sin, i32(pos), i32(table), i32(lengths), cK.t, cV.t, out_q=oq.t)
        torch.cuda.synchronize()
        for t in (out, oq, cK, cV):
            t.check()
