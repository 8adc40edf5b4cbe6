"""Sizes and numbers at the border of what the calls for tables, turns and shared prefixes take. No GPU."""
import pytest

from tests.test_rows_args import ALIGN, NOWS, SHAPE, P, _attend, _shared, _tables


def test_scales_that_no_float_holds():
    for bad in (3.5e38, -3.5e38, 1e300):
        assert _tables(scale=bad) == SHAPE, bad
    assert _tables(scale=3.4e38, co=P + 4) == ALIGN                          # (sizes and numbers are taken)


def units(T, sets, own, Hq, Hkv):
    """As the header has it: of T tokens in so many sets, and of so many sequences with rows of their own."""
    G = Hq // Hkv
    t, s = max(1, 256 // G), -(-G // 256)
    return ((T // t + sets if sets else 0) + own) * s * Hkv


# (query heads a KV head of 1, 7, 200, 256, 257, 300 and 1000)
@pytest.mark.parametrize("Hq,Hkv", [(8, 8), (28, 4), (200, 1), (512, 2), (257, 1), (300, 1), (2000, 2)])
@pytest.mark.parametrize("n,sets", [(40000, 3000), (9, 7000), (255, 1)])
def test_blocks_times_tiles(Hq, Hkv, n, sets):
    """The number of pages from which on the calls refuse, and one below: then they get as far as the missing scratch."""
    for page in (1, 16, 128):
        checks = [(lambda per: _attend(T=n, B=sets, Hq=Hq, Hkv=Hkv, per=per, page=page), units(n, sets, 0, Hq, Hkv))]
        checks += [(lambda per: _shared(B=n, P_=sets, Hq=Hq, Hkv=Hkv, per=per, pper=1, page=page), units(n, sets, n, Hq, Hkv)),
                   (lambda per: _shared(B=n, P_=sets, Hq=Hq, Hkv=Hkv, per=1, pper=per, page=page), units(n, sets, n, Hq, Hkv)),
                   (lambda per: _shared(B=n, P_=0, Hq=Hq, Hkv=Hkv, per=per, page=page), units(n, 0, n, Hq, Hkv))]
        for call, u in checks:
            tiles = -(-2 ** 31 // u) - 4                                     # the first number of whole tiles that is too many
            first = -(-tiles * 128 // page)
            if first * page >= 1 << 30 or first < 2:                         # (a table's own limit)
                continue
            assert call(first) == SHAPE and call(first - 1) == NOWS, (page, first, u)
