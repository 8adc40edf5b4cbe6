"""The same inputs give the same bits, whatever the SMs did before."""
import numpy as np
import pytest
import torch

import paper_2502_00299_b200 as ck
from tests.helpers import rand_bits, to_dev
from tests.test_gpu_rows import bits, i32

pytestmark = pytest.mark.gpu


def bf16(x):
    return torch.tensor(x, dtype=torch.float32, device="cuda").bfloat16()


@pytest.mark.parametrize("G,n", [(7, 18), (40, 3), (12, 21), (5, 2)])        # rows of queries that end inside of a warp
@pytest.mark.parametrize("d", [64, 128])
def test_what_shared_memory_held_before_does_not_matter(d, G, n):
    """Lanes behind a block's last row work on what an earlier launch left there. Here that would have every tile's second half move the references."""
    page, rows = 16, 1024
    rng = np.random.default_rng(G + d)
    u = rng.standard_normal(d)
    u /= np.linalg.norm(u)
    k = rng.standard_normal((rows, d)) + np.where(np.arange(rows) % 128 < 64, -1.0, 1.0)[:, None] * np.sqrt(d) * u
    K, V = bf16(k).view(rows // page, page, 1, d), to_dev(rand_bits(rng, (rows // page, page, 1, d)))
    q = bf16(rng.standard_normal((n, G, d)) + u)                             # (logits of the second halves lie a few powers of two above)
    args = q, i32([0, n]), i32(np.arange(rows // page)[None]), i32([[rows]]), K, V, False
    many = 256 * 300
    outs = []
    for left in (0.0, 30.0, -30.0, 0.0):                                     # wide blocks on every SM leave their queries
        x = bf16(left * u).expand(many, 1, d).contiguous()
        ck.attend_rows_paged(x, i32([0, many]), args[2], i32([[128]]), K, V, False)
        outs.append(ck.attend_rows_paged(*args))
        outs.append(ck.attend_shared_paged(q, i32([0, n]), args[2], args[3], i32(np.full((n, 1), -1)), i32(np.zeros((n, 1))), K, V))
    for i in (0, 1):
        assert all(torch.equal(bits(o), bits(outs[i])) for o in outs[i::2])
