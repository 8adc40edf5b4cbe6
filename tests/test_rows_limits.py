"""Sizes and numbers at the border of what the calls for tables, turns and shared prefixes take. No GPU."""
import paper_2502_00299_b200 as ck
from tests.test_rows_args import ALIGN, SHAPE, P, _tables


def test_scales_that_no_float_holds():
    for bad in (3.5e38, -3.5e38, 1e300):
        assert _tables(scale=bad) == SHAPE, bad
    assert _tables(scale=3.4e38, co=P + 4) == ALIGN                          # (sizes and numbers are taken)
