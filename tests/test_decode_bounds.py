"""The tolerances of attention would see a mistake: what attention with a row too few, a row too many or weights that are a few per cent off gives lies
outside them, in every head, also where rows that nobody sees hold the largest numbers. No GPU."""
import numpy as np
import pytest

from oracle import decode_oracle as ora
from tests.decode_bounds import MOST, absent, bounds, check, extreme, wide


def _values(case):
    q, K, V, tables, lengths = case
    return wide(q), wide(K), wide(V), tables, lengths


def _round(x):
    """To bf16, half to even."""
    b = x.astype(np.float32).view(np.uint32)
    return ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).view(np.float32).astype(np.float64)


CASES = [("absent", 64), ("absent", 128), ("extreme", 64), ("extreme", 128)]


def _case(name, d):
    return _values(absent(d, 0) if name == "absent" else extreme(d, 3, 0))


@pytest.mark.parametrize("name,d", CASES)
def test_the_formula_rounded_is_within(name, d):
    q, K, V, tables, lengths = _case(name, d)
    out, sums = ora.attend(q, K, V, tables, lengths)
    before = np.random.default_rng(0).random(sums.shape)
    ok = np.isfinite(out)
    out[ok] = _round(out[ok])
    check(out, before + sums, before, q, K, V, tables, lengths)
    assert 0 < bounds(q, K, V, tables, lengths)[4].max() < MOST


def _with(q, K, V, tables, n, b, h, g, drop=None, scale=1.0):
    """Query head g's output without row `drop`, with logits `scale` times as large."""
    page = K.shape[1]
    rows = [j for j in range(n) if j != drop and ora.place(tables[b], j, page, len(K)) is not None]
    at = np.array([ora.place(tables[b], j, page, len(K)) for j in rows])
    s = K[at[:, 0], at[:, 1], h] @ q[b, g] * scale / np.sqrt(q.shape[2])
    p = np.exp(s - s.max())
    return p / p.sum() @ V[at[:, 0], at[:, 1], h]


@pytest.mark.parametrize("name,d", CASES)
def test_mistakes_are_outside(name, d):
    q, K, V, tables, lengths = _case(name, d)
    ref, tol, sums, err, _ = bounds(q, K, V, tables, lengths)
    G, n = q.shape[1] // K.shape[2], np.clip(lengths, 0, tables.shape[1] * K.shape[1])
    # query heads whose output is a number and whose rows share the weight (where one has it all, nothing else matters)
    heads = [(b, h, g) for b in range(len(q)) for h in range(K.shape[2]) for g in range(h * G, (h + 1) * G)
             if np.isfinite(tol[b, g]).all() and (sums[b, h] > 0.01).sum() >= 4]
    assert len({(b, h) for b, h, _ in heads}) >= (5 if name == "absent" else 2)
    for b, h, g in heads:
        def outside(wrong):
            return (np.abs(wrong - ref[b, g]) > tol[b, g]).any()

        args = q, K, V, tables, int(n[b, h]), b, h, g
        assert not outside(_with(*args)) and outside(_with(*args, scale=1.05)) and outside(ref[b, g] * 0.98)
        for row in np.flatnonzero(sums[b, h] > 0.02 * G):
            assert outside(_with(*args, drop=row)), (b, h, g, row)
        # sums of weights that are one per cent off
        assert (sums[b, h] * 1e-2 > 2.0 ** -23 * sums[b, h] + err[b, h])[sums[b, h] > 0].all()
