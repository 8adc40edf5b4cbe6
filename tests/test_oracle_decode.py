"""What pins the fp64 statement of the calls on the decode cache: closed forms, other formulations and enumeration."""
import itertools

import numpy as np
import pytest

from oracle import decode_oracle as ora


def test_rotation_is_complex_multiplication_of_normalised_halves():
    rng = np.random.default_rng(0)
    x, gain, a = rng.standard_normal((5, 64)), rng.standard_normal(64), rng.uniform(-3, 3, 32)
    y = ora.rotate(x, None, 0.0, np.cos(a), np.sin(a))
    z = (x[:, :32] + 1j * x[:, 32:]) * np.exp(1j * a)
    assert np.allclose(y, np.concatenate([z.real, z.imag], 1), atol=1e-14)
    assert np.allclose(np.linalg.norm(y, axis=1), np.linalg.norm(x, axis=1))
    assert np.array_equal(ora.rotate(x, None, 0.0, np.ones(32), np.zeros(32)), x)
    n = ora.rotate(x, gain, 1e-3, np.ones(32), np.zeros(32))
    assert np.allclose(n, x * gain / np.sqrt((x ** 2).sum(1, keepdims=True) / 64 + 1e-3), atol=1e-14)
    assert np.allclose(ora.rotate(7 * x, gain, 0.0, np.cos(a), np.sin(a)), ora.rotate(x, gain, 0.0, np.cos(a), np.sin(a)))


def _cache(rng, B, Hkv, d, page, per):
    pages = B * per + 2
    return (rng.standard_normal((pages, page, Hkv, d)), rng.standard_normal((pages, page, Hkv, d)),
            rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32))


def test_attention_against_a_dense_softmax_and_its_closed_forms():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(1)
    B, Hq, Hkv, d, page, per = 2, 6, 2, 64, 4, 3
    K, V, tables = _cache(rng, B, Hkv, d, page, per)
    lengths = np.array([[12, 5], [1, 0]], dtype=np.int32)
    q = rng.standard_normal((B, Hq, d))
    out, sums = ora.attend(q, K, V, tables, lengths)
    for b in range(B):
        dense_K, dense_V = K[tables[b]].reshape(-1, Hkv, d), V[tables[b]].reshape(-1, Hkv, d)
        for g in range(Hq):
            n = lengths[b, g // 3]
            if n == 0:
                assert not out[b, g].any()
                continue
            p = torch.softmax(torch.tensor(dense_K[:n, g // 3] @ q[b, g] / 8.0), 0).numpy()
            assert np.allclose(out[b, g], p @ dense_V[:n, g // 3], atol=1e-13)
    assert np.allclose(sums.sum(-1), np.where(lengths > 0, 3, 0)) and not sums[0, 1, 5:].any()
    assert np.allclose(out[1, :3], V[tables[1, 0], 0, 0])                       # one row: its value
    uniform, _ = ora.attend(np.zeros_like(q), K, V, tables, lengths)
    assert np.allclose(uniform[0, 0], V[tables[0]].reshape(-1, Hkv, d)[:12, 0].mean(0))
    # rows in pages outside the cache are not there
    holes = tables.copy()
    holes[0, 1] = -1
    part, s = ora.attend(q, K, V, holes, lengths)
    short = np.concatenate([K[tables[0, 0]], K[tables[0, 2]]])[:, 0]
    p = np.exp(short @ q[0, 0] / 8.0)
    assert np.allclose(part[0, 0], (p / p.sum()) @ np.concatenate([V[tables[0, 0]], V[tables[0, 2]]])[:, 0]) and not s[0, 0, 4:8].any()


@pytest.mark.parametrize("n,w,c,budget", [(9, 2, 1, 5), (13, 2, 2, 8), (14, 3, 3, 8), (11, 0, 2, 4), (12, 4, 3, 6), (8, 3, 2, 8), (7, 1, 4, 4)])
def test_eviction_keeps_the_largest_chunks_with_the_fewest_moves(n, w, c, budget):
    rng = np.random.default_rng(n)
    for _ in range(20):
        x = rng.integers(0, 4, n).astype(np.float32)                            # many ties
        rows = ora.evict_rows(x, n, w, c, budget)
        assert len(rows) <= budget and len(set(rows)) == len(rows)
        if n <= budget:
            assert rows == list(range(n))
            continue
        C = (n - w) // c
        r = n - C * c
        k = (budget - r) // c
        assert w <= r < w + c and len(rows) == k * c + r and rows[k * c:] == list(range(n - r, n))
        chunks = [rows[i * c] // c for i in range(k)]
        assert all(rows[i * c:(i + 1) * c] == list(range(ch * c, ch * c + c)) for i, ch in enumerate(chunks))
        s = [float(x[i * c:(i + 1) * c].sum()) for i in range(C)]
        assert sum(s[i] for i in chunks) == max(sum(s[i] for i in ids) for ids in itertools.combinations(range(C), k))
        assert sorted(chunks) == sorted(sorted(range(C), key=lambda i: (-s[i], i))[:k])     # ties to the lower chunk
        assert all(chunks[i] == i for i in chunks if i < k)                                # those below k stay
        moved = [ch for i, ch in enumerate(chunks) if ch != i]
        assert moved == sorted(moved) and all(ch >= k for ch in moved)


def test_eviction_moves_rows_with_their_sums():
    rng = np.random.default_rng(3)
    B, Hkv, d, page, per = 2, 2, 4, 4, 5
    K, V, tables = _cache(rng, B, Hkv, d, page, per)
    lengths = np.array([[20, 11], [6, 17]], dtype=np.int32)
    x = rng.random((B, Hkv, 20)).astype(np.float32) * (np.arange(20) < lengths[..., None])
    y, new, K2, V2, idx = ora.evict(x, tables, lengths, K, V, 3, 2, 10)
    # 20 rows: 8 chunks and 4 behind, 3 of the chunks; 11: 4 and 3, 3 of them; 17: 7 and 3, 3 of them
    assert new.tolist() == [[10, 9], [6, 9]]
    for b in range(B):
        dense, before = (t[tables[b]].reshape(-1, Hkv, d) for t in (K2, K))
        for h in range(Hkv):
            m = new[b, h]
            assert np.array_equal(dense[:m, h], before[idx[b, h, :m], h]) and np.array_equal(y[b, h, :m], x[b, h, idx[b, h, :m]])
            assert not y[b, h, m:].any() and (idx[b, h, m:] == -1).all()
    assert ora.evict_rows(np.array([1, np.nan, 3, 2, 0, 0], dtype=np.float32), 6, 1, 1, 3) == [2, 1, 5]
