"""Which sizes attention takes: the call, its scratch and the header say the same, without a GPU."""
import itertools

import pytest

import paper_2502_00299_b200 as ck
from tests.test_decode_args import NOWS, OK, SHAPE, _attend

size = ck.lib.chunkkv_attend_scratch_bytes


def _allowed(B, Hq, Hkv, rows):
    """The header's limits for well-formed heads."""
    return B * Hq < 2 ** 30 and rows < 2 ** 30 and B * Hkv * -(-(Hq // Hkv) // 8) * (rows // 16 + 8) < 2 ** 31


CASES = [(B, G * Hkv, Hkv, rows, sums) for B, Hkv, G, rows, sums in itertools.product(
    (1, 8, 256, 4099, 1 << 22), (1, 8, 128), (1, 8, 9, 16, 17), (1 << 10, 1 << 20, 1 << 24, (1 << 29) + 1, (1 << 30) - 1), (0, 1)) if G * Hkv <= 65535]


def test_a_size_has_scratch_where_the_call_takes_it():
    both = set()
    for B, Hq, Hkv, rows, sums in CASES:
        need = size(B, Hq, Hkv, 64, rows, 1, sums)
        got = _attend(B=B, Hq=Hq, Hkv=Hkv, d=64, per=rows, page=1, weights=256 if sums else None, size=0, scratch=None)
        assert (need > 0) == _allowed(B, Hq, Hkv, rows), (B, Hq, Hkv, rows)
        # (nothing here is short enough to need no scratch: a call that is allowed stops at the missing scratch, before any CUDA call)
        if need != 256:
            assert got == (NOWS if need else SHAPE), (B, Hq, Hkv, rows, got)
        both.add(need > 0)
    assert both == {True, False}


@pytest.mark.parametrize("Hkv", [8, 16])
def test_many_query_heads_over_a_million_rows_are_within_the_limits(Hkv):
    """256 sequences of 128 query heads in tables for 2^20 rows: every documented limit holds."""
    assert size(256, 128, Hkv, 128, 1 << 16, 16, 0) > 256
    assert _attend(B=256, Hq=128, Hkv=Hkv, d=128, per=1 << 16, page=16, scratch=None) == NOWS


def test_refused_sizes_have_no_scratch():
    assert size(8, 8, 8, 64, 1 << 29, 1, 0) == 0 and _attend(B=8, Hq=8, Hkv=8, per=1 << 29, page=1) == SHAPE
    assert _attend(B=0, per=1 << 29, page=1) == OK
