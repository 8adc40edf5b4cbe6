"""Attention against the formula with tolerances of each head's own (decode_bounds.py): heads that see nothing of the largest numbers, infinities and
not-a-number around them, and heads of extreme logits beside ordinary ones."""
import numpy as np
import pytest
import torch

import paper_2502_00299_b200 as ck
from tests.decode_bounds import absent, check, extreme, wide
from tests.helpers import Guarded, to_dev
from tests.test_gpu_decode import f64, i32

pytestmark = pytest.mark.gpu


def run(q, K, V, tables, lengths, sums, seed=0):
    """One call, checked. Returns (out, weights)."""
    out = Guarded(q.shape, torch.bfloat16)
    w = before = None
    if sums:
        w = Guarded((*lengths.shape, tables.shape[1] * K.shape[1]), torch.float32)
        before = np.random.default_rng(seed).random(w.t.shape).astype(np.float32)
        w.t.copy_(torch.from_numpy(before))
    ck.attend_paged(to_dev(q), i32(tables), i32(lengths), to_dev(K), to_dev(V), None if w is None else w.t, out.t)
    out.check()
    if w is not None:
        w.check()
    check(f64(out.t), None if w is None else f64(w.t), None if w is None else before.astype(np.float64), wide(q), wide(K), wide(V), tables, lengths)
    return out.t, None if w is None else w.t


ROOMS = [0, 300, 2000]          # pages of nobody behind a sequence's: the smallest clusters, clusters of eight and 16, two launches


@pytest.mark.parametrize("sums", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("room", ROOMS)
def test_rows_that_are_not_there(d, room, sums):
    out, _ = run(*absent(d, room), sums)
    assert not out[3].any() and not out[1, 3:].any() and not out[4, 3:].any()


@pytest.mark.parametrize("sums", [False, True])
@pytest.mark.parametrize("d,G", [(64, 3), (128, 8), (128, 12), (64, 20)])
@pytest.mark.parametrize("room", ROOMS)
def test_extreme_logits_beside_ordinary_ones(d, G, room, sums):
    case = extreme(d, G, room)
    out, _ = run(*case, sums)
    assert not out[0, G:2 * G].any() and torch.isnan(out[0, 2 * G:3 * G]).all() and torch.isnan(out[0, 4 * G:5 * G]).all()
    assert torch.isfinite(out[0, :2 * G]).all() and torch.isfinite(out[0, 5 * G:]).all()
    V, tables = case[2], case[3]
    assert torch.equal(out[0, 3 * G:4 * G], to_dev(V[tables[0, 77 // 16], 77 % 16, 3]).expand(G, d))
