"""Pins of oracle/rows_oracle.py: against decode_oracle where both state the same, and against values worked out otherwise."""
import math

import numpy as np
import pytest

from oracle import decode_oracle, rows_oracle as ora


def test_frequencies():
    w = ora.frequencies(64, 10000.0)
    assert w[0] == 1.0 and np.allclose(w[16], 10000.0 ** -0.5) and len(w) == 32
    assert np.allclose(ora.frequencies(64, 10000.0, "linear", 4.0), w / 4)
    for kind, low, high in (("dims", 1.0, 32.0), ("waves", 1.0, 4.0)):
        s = ora.frequencies(64, 10000.0, kind, 8.0, 8192.0, low, high)
        r = w / s
        assert np.all(r >= 1 - 1e-12) and np.all(r <= 8 + 1e-12) and np.all(np.diff(r) >= -1e-12)
        assert r[0] == 1.0 and np.isclose(r[-1], 8.0) and ((r > 1.001) & (r < 7.999)).any()
    turns = 8192.0 * w / (2 * math.pi)
    s = ora.frequencies(64, 10000.0, "waves", 8.0, 8192.0, 1.0, 4.0)
    assert np.allclose(s[turns >= 4], w[turns >= 4]) and np.allclose(s[turns <= 1], w[turns <= 1] / 8)


def test_tables():
    c, s = ora.tables(5, 16, 10000.0, scale=1.5, first=-2)
    assert c.shape == (5, 8) and np.allclose(c[2], 1.5) and np.allclose(s[2], 0) and np.allclose(s[0], -s[4]) and np.allclose(c * c + s * s, 2.25)
    assert np.isclose(s[3, 0], 1.5 * math.sin(1.0))


@pytest.mark.parametrize("gain", [False, True])
def test_whole_heads_in_halves_are_those_of_the_decode_oracle(gain):
    rng = np.random.default_rng(1)
    x, g = rng.standard_normal((3, 2, 64)), rng.standard_normal(64) if gain else None
    cos, sin = rng.standard_normal((3, 1, 32)), rng.standard_normal((3, 1, 32))
    assert np.allclose(ora.rotate(x, g, 1e-5, cos, sin, False), decode_oracle.rotate(x, g, 1e-5, cos, sin))


def test_pairs_are_halves_in_another_order_and_the_rest_stays():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((4, 64))
    a = rng.standard_normal((4, 16))
    y = ora.rotate(x, None, 0.0, np.cos(a), np.sin(a), True)
    order = np.r_[np.arange(0, 32, 2), np.arange(1, 32, 2), np.arange(32, 64)]
    assert np.allclose(y[:, order], ora.rotate(x[:, order], None, 0.0, np.cos(a), np.sin(a), False))
    assert np.array_equal(y[:, 32:], x[:, 32:]) and np.allclose((y * y).sum(1), (x * x).sum(1))


def _cache(rng, B, Hkv, d, page, per):
    pages = B * per + 2
    K, V = rng.standard_normal((2, pages, page, Hkv, d))
    return K, V, rng.permutation(pages)[:B * per].reshape(B, per).astype(np.int32)


def test_one_token_a_sequence_is_the_decode_oracle():
    rng = np.random.default_rng(3)
    K, V, t = _cache(rng, 3, 2, 16, 4, 5)
    t[1, 1] = -1
    lengths = np.array([[7, 20], [11, 0], [99, -3]], dtype=np.int32)
    q = rng.standard_normal((3, 4, 16))
    want, _ = decode_oracle.attend(q, K, V, t, lengths)
    for causal in (False, True):
        assert np.allclose(ora.attend_rows(q, [0, 1, 2, 3], K, V, t, lengths, causal), want)
    none = np.zeros((0, 2), dtype=np.int32)
    assert np.allclose(ora.attend_shared(q, [0], K, V, np.zeros((0, 1), dtype=np.int32), none, t, lengths), want)


def test_causal_tokens_see_what_single_steps_would():
    rng = np.random.default_rng(4)
    K, V, t = _cache(rng, 2, 2, 16, 4, 5)
    lengths = np.array([[12, 9], [3, 2]], dtype=np.int32)                    # (the second has fewer rows than new tokens)
    starts = np.array([1, 4, 8])
    q = rng.standard_normal((9, 4, 16))
    out = ora.attend_rows(q, starts, K, V, t, lengths, True)
    for b in range(2):
        n = starts[b + 1] - starts[b]
        for i in range(n):
            want, _ = decode_oracle.attend(q[starts[b] + i][None], K, V, t[b:b + 1], lengths[b:b + 1] - (n - 1 - i))
            assert np.allclose(out[starts[b] + i], want[0])
    assert not out[0].any() and not out[8].any() and not out[4].any()


def test_a_prefix_is_rows_in_front():
    rng = np.random.default_rng(5)
    K, V, t = _cache(rng, 5, 2, 16, 4, 6)
    q = rng.standard_normal((3, 4, 16))
    prefix, own = t[:2, :3], np.concatenate([t[2:, :3]])
    pl, ol = np.full((2, 2), 8), np.array([[5, 4], [0, 1], [12, 7]])
    out = ora.attend_shared(q, [0, 2, 3], K, V, prefix, pl, own, ol)
    joined = np.stack([np.concatenate([prefix[g][:2], own[b]]) for b, g in enumerate((0, 0, 1))])
    want, _ = decode_oracle.attend(q, K, V, joined, ol + 8)
    assert np.allclose(out, want)


def test_places_of_appended_rows():
    t = np.array([[3, 1], [0, 9]], dtype=np.int32)
    at = ora.append_places([1, 3, 6], 7, t, np.array([[5, 1], [8, 2]], dtype=np.int32), 4, 5)
    assert at[0] is None and at[6] is None
    assert at[1] == [(3, 3), None] and at[2] == [(1, 0), (3, 0)]             # rows 3, 4 and -1, 0
    assert at[3] == [None, None] and at[5] == [None, (0, 1)]                 # rows 5 .. 7 lie in a page that is not there; -1, 0, 1
