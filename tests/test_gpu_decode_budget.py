"""Eviction to budgets beyond every cache: nothing is evicted, and the list of rows is written to its end and no further."""
import numpy as np
import pytest
import torch

import paper_2502_00299_b200 as ck
from tests.helpers import rand_bits, to_dev
from tests.test_gpu_decode import i32, new_cache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("budget", [2 ** 31 - 1, 2 ** 31 - 4096, 2 ** 30 + 5])
def test_the_largest_budgets(budget):
    rng = np.random.default_rng(1)
    K, V, tables = new_cache(rng, 1, 1, 64, 16, 3)
    state = torch.rand(1, 1, 48, device="cuda"), i32([[41]]), to_dev(K), to_dev(V)
    w, dl, dK, dV = [t.clone() for t in state]
    room = 1 << 14                                        # more than a step of all threads of a cluster, on both sides
    buf = torch.full((budget + 2 * room,), 77, device="cuda", dtype=torch.int32)
    idx = ck.evict_paged(w, i32(tables), dl, dK, dV, 4, 3, budget, out_idx=buf[room:room + budget])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(state, (w, dl, dK, dV)))
    assert idx.data_ptr() == buf[room:].data_ptr() and torch.equal(idx[:41], torch.arange(41, device="cuda", dtype=torch.int32))
    assert int(idx[41:].max()) == int(idx[41:].min()) == -1
    assert (buf[:room] == 77).all() and (buf[room + budget:] == 77).all()
