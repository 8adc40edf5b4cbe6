"""Angles of far positions. The other tests' reference is in 64 bits, whose own angles are no better than 2^-21 there; here frequencies have 60 digits and a
position's angle is a fraction of a turn in whole numbers."""
import decimal
import math

import numpy as np
import pytest

import paper_2502_00299_b200 as ck

pytestmark = pytest.mark.gpu
D = decimal.Decimal
PI = D("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899")
N = 1 << 16


def turns(rot, base, kind, factor, original, low, high):
    """Turns a position of each pair."""
    with decimal.localcontext(decimal.Context(prec=60)):
        out = []
        for i in range(rot // 2):
            w = (-(D(2) * i / rot) * D(base).ln()).exp()
            f = D(factor)
            if kind == "linear":
                w /= f
            elif kind == "dims":
                dim = lambda n: rot * (D(original) / (2 * PI * D(n))).ln() / (2 * D(base).ln())  # noqa: E731
                a, b = max(math.floor(dim(high)), 0), min(math.ceil(dim(low)), rot - 1)
                s = min(max(D(i - a) / max(D(b - a), D("0.001")), D(0)), D(1))
                w = s * w / f + (1 - s) * w
            elif kind == "waves":
                s = min(max((D(original) * w / (2 * PI) - D(low)) / (D(high) - D(low)), D(0)), D(1))
                w = s * w + (1 - s) * w / f
            out.append(w / (2 * PI))
        return out


def angles(first, turn):
    """Radians of N positions from `first` on: the first one's fraction of a turn, then N steps in 64 bits (2^-48 of a turn off at the end)."""
    with decimal.localcontext(decimal.Context(prec=60)):
        begin, step = (int((x % 1 + 1) % 1 * 2 ** 64) for x in (first * turn, turn))
    at = np.uint64(begin) + np.arange(N, dtype=np.uint64) * np.uint64(step)
    return at.astype(np.float64) * (2 * math.pi / 2.0 ** 64)


SCALINGS = [("none", 1.0, 0.0, 0.0, 0.0), ("linear", 8.0, 0.0, 0.0, 0.0), ("dims", 8.0, 128.0, 1.0, 32.0), ("dims", 8.0, 512.0, 1.0, 32.0), ("dims", 3.0, 8192.0, 1.0, 32.0),
            ("waves", 8.0, 8192.0, 1.0, 4.0), ("linear", 0.5, 0.0, 0.0, 0.0)]


@pytest.mark.parametrize("first", [1 << 31, (1 << 31) - 12345, -(1 << 31), 1000])
@pytest.mark.parametrize("rot", [64, 128, 48])
@pytest.mark.parametrize("kind,factor,original,low,high", SCALINGS)
def test_angles_at_any_position(kind, factor, original, low, high, rot, first):
    base, scale = 10000.0, 1.25
    got = [t.cpu().numpy().astype(np.float64) for t in ck.rope_tables(N, rot, base, kind, factor, original, low, high, scale, first)]
    turned = 0
    for i, w in enumerate(turns(rot, base, kind, factor, original, low, high)):
        a = angles(first, w)
        c, s = np.cos(a), np.sin(a)
        assert np.abs(got[0][:, i] - scale * c).max() <= 2.0 ** -22 * scale and np.abs(got[1][:, i] - scale * s).max() <= 2.0 ** -22 * scale
        # An angle that is off turns all values the same way, a rounding this way and that: the mean over four turns and more has what is left of N independent
        # roundings of at most 2^-22, five standard deviations of it here, and 2^-31 of a turn (more where a factor below 1 makes more of an error)
        if float(w) * N >= 4:
            turned += 1
            off = ((got[1][:, i] * c - got[0][:, i] * s) / scale).mean()
            assert abs(off) <= 2 * math.pi * 2.0 ** -31 / min(factor, 1.0) + 5 * 2.0 ** -22 / math.sqrt(N), (i, off)
    assert turned >= 4
