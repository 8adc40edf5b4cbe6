"""A process whose very first calls on turns and shared prefixes are captured: what the library asks of the device and sets for its kernels does not end the capture."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import torch
import paper_2502_00299_b200 as ck
d, Hq, Hkv, page, per, n = {d}, 4, 2, 16, 40, 30
g = torch.Generator("cuda").manual_seed(0)
K, V = (torch.randn(per, page, Hkv, d, device="cuda", generator=g).bfloat16() for _ in range(2))
qkv = torch.randn(n, (Hq + 2 * Hkv) * d, device="cuda", generator=g).bfloat16()
i32 = lambda x: torch.tensor(x, device="cuda", dtype=torch.int32)
table, lengths, starts, pos = torch.arange(per, device="cuda", dtype=torch.int32)[None], i32([[600, 590]]), i32([0, n]), torch.arange(n, device="cuda", dtype=torch.int32)
all_, none = i32([0, n]), torch.zeros(n, Hkv, device="cuda", dtype=torch.int32)
own = torch.zeros(n, 1, device="cuda", dtype=torch.int32)
torch.cuda.synchronize()

def calls():
    cos, sin = ck.rope_tables(64, d, 10000.0)
    q, _ = ck.rotate_rows(qkv, Hq, Hkv, d, cos, sin, pos, True)
    q2 = ck.append_rows_paged(qkv, Hq, starts, cos, sin, pos, table, lengths, K, V, True)
    return q, q2, ck.attend_rows_paged(q, starts, table, lengths, K, V, False), ck.attend_shared_paged(q, all_, table, lengths, own, none, K, V)

graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    got = calls()
graph.replay()
torch.cuda.synchronize()
assert ck.device_status() == 0 and torch.equal(got[0], got[1]) and got[2].any()
for a, b in zip(got, calls()):
    assert torch.equal(a, b)
# (both round weights and outputs on their own: 2 * 2^-8 (sum p |v| + |out|), of values whose mean size is 0.8 and outputs below one)
assert (got[2].float() - got[3].float()).abs().max() < 0.02
"""


@pytest.mark.parametrize("d", [64, 128])
def test_the_first_calls_of_a_process_are_captured(d):
    r = subprocess.run([sys.executable, "-c", CODE.replace("{d}", str(d))], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-800:]
