"""A process whose very first call is captured: what the library asks of the device and sets for its kernels does not end the capture."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import torch
import paper_2502_00299_b200 as ck
d, Hq, Hkv, page, per = 128, 4, 2, 16, {per}
g = torch.Generator("cuda").manual_seed(0)
K, V = (torch.randn(per, page, Hkv, d, device="cuda", generator=g).bfloat16() for _ in range(2))
q = torch.randn(1, Hq, d, device="cuda", generator=g).bfloat16()
table = torch.arange(per, device="cuda", dtype=torch.int32)[None]
lengths = torch.full((1, Hkv), per * page - 3, device="cuda", dtype=torch.int32)
w, w1 = (torch.zeros(1, Hkv, per * page, device="cuda") for _ in range(2))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    plain = ck.attend_paged(q, table, lengths, K, V)
    out = ck.attend_paged(q, table, lengths, K, V, w)
graph.replay()
torch.cuda.synchronize()
assert out.any() and torch.equal(out, plain) and torch.equal(out, ck.attend_paged(q, table, lengths, K, V, w1)) and torch.equal(w, w1)
graph2 = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph2):
    ck.evict_paged(w, table, lengths, K, V, 16, 1, per * page // 2)
graph2.replay()
torch.cuda.synchronize()
assert (lengths == per * page // 2).all()
"""


@pytest.mark.parametrize("per", [250, 2000])          # clusters of 16; two launches and keys beyond 48 KB
def test_the_first_call_of_a_process_is_captured(per):
    r = subprocess.run([sys.executable, "-c", CODE.replace("{per}", str(per))], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-800:]
