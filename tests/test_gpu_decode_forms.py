"""Forms of the kernels on the decode cache that take large sizes to reach: selections of an eviction with several keys a thread, the joining of attention's
sums with eight rows a thread, and short caches of more heads than SMs with more than eight query heads each."""
import numpy as np
import pytest
import torch

import paper_2502_00299_b200 as ck
from tests.decode_bounds import check, new_cache, wide
from tests.helpers import rand_bits, to_dev
from tests.test_gpu_decode import check_eviction, f64, i32, some_weights
from tests.test_gpu_decode_bounds import run

pytestmark = pytest.mark.gpu


# A thread of 512 has ceil(C / 512) keys of C chunks: up to 4, 6, 8, 10, 12 and 24 of them in registers, near the first and the last C of each
CHUNKS = [1025, 2048, 2049, 3060, 3080, 4096, 4097, 5120, 5121, 6144, 6145, 9000, 12288, 12289]


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("C", CHUNKS)
def test_selections_of_many_chunks(C, kind):
    """Row by row and in chunks of three; the second head has fewer chunks, the third stays as it is."""
    rng = np.random.default_rng(C)
    for c, w, keep in ((1, 20, 0.6), (3, 7, 0.3), (1, 0, 0.02)):
        n = C * c + w
        page = 64
        per = -(-n // page)
        budget = min(int(C * keep), 8192) * c + w + c - 1
        lengths = np.array([[n, n - 5 * c, budget]], dtype=np.int32)
        check_eviction(rng, 1, 3, 64, page, per, lengths, w, c, budget, some_weights(rng, (1, 3, per * page), kind))


@pytest.mark.parametrize("C,k", [(9000, 8191), (9000, 8192), (9000, 8193), (12288, 8192), (12289, 8192), (12289, 1)])
def test_selections_at_the_limits_of_their_lists(C, k):
    rng = np.random.default_rng(C + k)
    per = -(-(C + 16) // 64)
    check_eviction(rng, 1, 2, 64, 64, per, np.full((1, 2), C + 16, dtype=np.int32), 16, 1, k + 16, some_weights(rng, (1, 2, per * 64), "ties"))


# More than 303104 rows in the tables take eight rows a thread; records of a unit are joined by a warp (76 sequences of eight heads), a CTA (9) or several (3, 1)
@pytest.mark.parametrize("Hq,Hkv,d,B,n,page", [(8, 8, 64, 76, 550, 16), (8, 8, 128, 76, 513, 16), (16, 8, 128, 9, 4300, 100), (8, 4, 64, 3, 26000, 64),
                                               (12, 1, 128, 3, 110000, 64), (10, 1, 64, 80, 4000, 16)])
def test_sums_over_more_rows_than_threads(Hq, Hkv, d, B, n, page):
    assert B * Hkv * -(-n // page) * page > 303104
    rng = np.random.default_rng(n)
    per = -(-n // page)
    K, V, tables = new_cache(rng, min(B, 8), Hkv, d, page, per)
    tables = np.concatenate([np.roll(tables, b, 1) for b in range(-(-B // len(tables)))])[:B]      # (sequences share pages: they are only read)
    lengths = np.maximum(n - (rng.random((B, Hkv)) ** 2 * n).astype(np.int32), 0).astype(np.int32)
    lengths[0] = n
    run(rand_bits(rng, (B, Hq, d), 2.0), K, V, np.ascontiguousarray(tables), lengths, True)


@pytest.mark.parametrize("G", [9, 12, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,Hkv,rows", [(149, 1, 80), (40, 5, 96), (74, 4, 90), (149, 1, 700), (20, 8, 1150), (300, 2, 150)])
def test_short_caches_of_many_heads_with_wide_groups(B, Hkv, rows, d, G):
    """CTAs of four warps for up to 16 query heads each, with sums where their logits have room (a hundred rows), else in two launches."""
    rng = np.random.default_rng(B + rows)
    page = 16
    per = -(-rows // page)
    K, V, tables = new_cache(rng, min(B, 20), Hkv, d, page, per)
    tables = np.ascontiguousarray(np.resize(tables, (B, per)))
    lengths = rng.integers(0, rows + 1, (B, Hkv)).astype(np.int32)
    lengths[0, 0], lengths[-1, -1] = rows, 0
    q = rand_bits(rng, (B, G * Hkv, d), 2.0)
    for sums in (False, True):
        run(q, K, V, tables, lengths, sums)


def test_short_sequences_in_tables_for_a_million_rows():
    """256 sequences of 128 query heads: the scratch goes by the heads, not by the tables' room, and outputs are those of small tables."""
    rng = np.random.default_rng(77)
    B, Hq, Hkv, d, page, per = 256, 128, 8, 64, 16, 4
    K, V, tables = new_cache(rng, 8, Hkv, d, page, per)
    tables = np.ascontiguousarray(np.resize(tables, (B, per)))
    lengths = rng.integers(0, per * page + 1, (B, Hkv)).astype(np.int32)
    q = rand_bits(rng, (B, Hq, d))
    roomy = torch.full((B, (1 << 20) // page), -1, device="cuda", dtype=torch.int32)
    roomy[:, :per] = i32(tables)
    assert ck.lib.chunkkv_attend_scratch_bytes(B, Hq, Hkv, d, roomy.shape[1], page, 0) < 1 << 26
    out = ck.attend_paged(to_dev(q), roomy, i32(lengths), to_dev(K), to_dev(V))
    check(f64(out), None, None, wide(q), wide(K), wide(V), tables, lengths)
