"""Rows that several blocks of a launch share: what the calls promise does not depend on where the cuts lie."""
import numpy as np
import pytest

import paper_2502_00299_b200 as ck
from oracle import rows_oracle as ora
from tests.decode_bounds import wide
from tests.helpers import rand_bits, to_dev
from tests.test_gpu_rows import i32, paged, values

pytestmark = pytest.mark.gpu
NEG, INF, NAN = 0xFF80, 0x7F80, 0x7FC0


@pytest.mark.parametrize("what", [INF, NAN])
@pytest.mark.parametrize("B,rows", [(1, 4000), (200, 300)])                  # a tile a block; units that are whole and units that are cut, at any place
@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_infinite_values_in_rows_of_no_weight(d, shared, B, rows, what):
    """Logits of -inf in a whole tile, and in it a value that is not finite: 0 times it is no number, in a block of its own as beside other rows."""
    page, n, Hq = 16, 5, 4
    rng = np.random.default_rng(rows + d)
    K, V, table = paged(rng, 1, 1, d, page, -(-rows // page))
    q = rand_bits(rng, (n, Hq, d))
    q[..., 0] = 0x3F80
    at = lambda j: (table[0, j // page], j % page, 0)  # noqa: E731
    for j in range(128, 256):
        K[at(j)][0] = NEG
    V[at(130)][7] = V[at(255)][d - 1] = what
    args = to_dev(np.tile(q, (B, 1, 1))), i32(n * np.arange(B + 1)), i32(np.tile(table, (B, 1))), i32(np.full((B, 1), rows))
    if shared:
        none = i32(np.zeros((B * n, 1)))
        out = values(ck.attend_shared_paged(*args, none - 1, none, to_dev(K), to_dev(V)))
    else:
        out = values(ck.attend_rows_paged(*args, to_dev(K), to_dev(V)))
    with np.errstate(all="ignore"):
        ref = ora.attend_rows(wide(q), [0, n], wide(K), wide(V), table, np.array([[rows]]), not shared)
    want = np.zeros(ref.shape, dtype=bool)
    want[..., [7, d - 1]] = True
    assert np.array_equal(~np.isfinite(ref), want) and np.array_equal(~np.isfinite(out), np.tile(want, (B, 1, 1)))
    assert ck.device_status() == 0


@pytest.mark.parametrize("d", [64, 128])
def test_nothing_but_infinite_logits_over_a_cut(d):
    """Every logit is -inf, values are not finite: zeros, as from a single block."""
    page, rows = 16, 4000
    rng = np.random.default_rng(d)
    K, V, table = paged(rng, 1, 1, d, page, rows // page)
    q = rand_bits(rng, (3, 2, d))
    q[..., 0] = 0x3F80
    K[..., 0], V[..., 3] = NEG, INF
    args = to_dev(q), i32([0, 3]), i32(table)
    assert not ck.attend_rows_paged(*args, i32([[rows]]), to_dev(K), to_dev(V), False).any()
    assert not ck.attend_shared_paged(*args, i32([[rows]]), i32(np.full((3, 1), -1)), i32(np.zeros((3, 1))), to_dev(K), to_dev(V)).any()


@pytest.mark.parametrize("d", [64, 128])
def test_values_behind_a_token_in_a_block_of_their_own(d):
    """Tokens that see none of a block's rows take nothing from them, whatever they hold."""
    page, n, rows = 16, 200, 4000
    rng = np.random.default_rng(d + 1)
    K, V, table = paged(rng, 1, 1, d, page, rows // page)
    q = to_dev(rand_bits(rng, (n, 1, d)))
    lengths = i32([[rows]])
    clean = ck.attend_rows_paged(q, i32([0, n]), i32(table), lengths, to_dev(K), to_dev(V))
    for j in (rows - 1, rows - 40, rows - 128):
        V[table[0, j // page], j % page, 0, 5] = INF
    out = ck.attend_rows_paged(q, i32([0, n]), i32(table), lengths, to_dev(K), to_dev(V))
    got, was = values(out), values(clean)
    assert (~np.isfinite(got[n - 128:, 0, 5])).all() and np.isfinite(got[:n - 128]).all()
    assert np.array_equal(got[:n - 128], was[:n - 128]) and np.array_equal(np.delete(got, 5, 2), np.delete(was, 5, 2))
