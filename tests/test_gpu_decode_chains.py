"""The calls on the decode cache queued directly behind one another, so that each is on the SMs while the one ahead writes what it reads: what they
give with the GPU idle between them, bit for bit."""
import numpy as np
import pytest
import torch

import paper_2502_00299_b200 as ck
from tests.helpers import rand_bits, to_dev
from tests.test_gpu_decode import angles, i32, new_cache

pytestmark = pytest.mark.gpu


def _chain(Hq, Hkv, d, B, n, page, room, seed):
    """A batch over its budget, and a function that queues eviction, attention, a new row and attention again on it, with `between` called in between."""
    rng = np.random.default_rng(seed)
    per = -(-n // page)
    K, V, tables = new_cache(rng, B, Hkv, d, page, per)
    tables = np.concatenate([tables, np.full((B, room // page), -1, dtype=np.int32)], 1)
    lengths = n - rng.integers(0, n // 4, (B, Hkv))
    weights = np.where(np.arange(tables.shape[1] * page) < lengths[..., None], rng.random((B, Hkv, tables.shape[1] * page)), 0).astype(np.float32)
    state = [i32(lengths), to_dev(K), to_dev(V), torch.tensor(weights).cuda()]
    dl, dK, dV, w = work = [t.clone() for t in state]
    table, qkv = i32(tables), to_dev(rand_bits(rng, (B, (Hq + 2 * Hkv) * d)))
    q0, gain = to_dev(rand_bits(rng, (B, Hq, d))), to_dev(rand_bits(rng, (d,)))
    cos, sin = (torch.tensor(x).cuda() for x in angles(20, d))
    pos = i32(rng.integers(0, 20, B))

    def restore():
        for t, s in zip(work, state):
            t.copy_(s)

    def run(between=lambda: None):
        idx = ck.evict_paged(w, table, dl, dK, dV, 8, 4, n // 2)
        between()
        first = ck.attend_paged(q0, table, dl, dK, dV, w)
        between()
        idx2 = ck.evict_paged(w, table, dl, dK, dV, 8, 4, n // 3)
        between()
        q = ck.append_paged(qkv, Hq, cos, sin, pos, table, dl, dK, dV, gain, gain)      # (over the last row that is left)
        between()
        second = ck.attend_paged(q, table, dl, dK, dV, w)
        between()
        plain = ck.attend_paged(q, table, dl, dK, dV)
        return [idx, first, idx2, q, second, plain]

    return work, restore, run


SIZES = [(8, 2, 64, 2, 160, 16, 0), (8, 2, 64, 2, 160, 16, 4000), (32, 8, 128, 4, 400, 16, 0), (32, 8, 128, 4, 400, 16, 20000), (28, 4, 128, 40, 300, 7, 0)]


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("sizes", SIZES)
def test_calls_directly_behind_one_another(sizes, captured):
    work, restore, run = _chain(*sizes, seed=sum(sizes))
    restore()
    torch.cuda.synchronize()
    want = [t.clone() for t in run(torch.cuda.synchronize) + work]
    torch.cuda.synchronize()
    assert (want[6] < sizes[4] // 2).all() and want[1].any() and want[4].any()
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        restore()
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = run()
    for _ in range(25):
        restore()
        if captured:
            graph.replay()
            got = held + work
        else:
            got = run() + work
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------------ a prompt: rotation, then compression
PROMPTS = [(32, 8, 128, 2500, 32, 10, 300), (8, 2, 64, 700, 16, 5, 90), (28, 4, 128, 9001, 32, 16, 1000)]


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,L,w,c,budget", PROMPTS)
def test_compression_directly_behind_the_rotation(Hq, Hkv, d, L, w, c, budget, captured):
    """Keys that are rotated into head-major outputs and in their place in the activation, read by the calls that compress them as soon as they are queued."""
    rng = np.random.default_rng(L)
    row = (Hq + 2 * Hkv) * d
    raw, gain = to_dev(rand_bits(rng, (L, row))), to_dev(rand_bits(rng, (d,)))
    cos, sin = (torch.tensor(x).cuda() for x in angles(L, d))
    pos, qkv = torch.arange(L, device="cuda", dtype=torch.int32), raw.clone()
    K, V = (torch.empty(Hkv, L, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    V.copy_(raw[:, (Hq + Hkv) * d:].view(L, Hkv, d).permute(1, 0, 2))
    Q, q_obs = (torch.empty(Hq, n, d, device="cuda", dtype=torch.bfloat16) for n in (L, w))
    reuse = torch.sort(i32(rng.permutation(L)[:budget]))[0].expand(Hkv, budget).contiguous()
    heads = qkv.unflatten(1, (-1, d))
    tokens = lambda t: t.permute(1, 0, 2)
    n_max = ck.out_len(L, w, c, budget)
    page = 16
    table = i32(rng.permutation(-(-n_max // page)))
    cache = [torch.zeros(len(table), page, Hkv, d, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    # (made once, so that no call allocates or fills anything between two of them)
    q_obs.copy_(tokens(ck.rotate_qk(raw, Hq, Hkv, d, cos, sin, pos, gain, gain)[0][-w:]))

    def restore():
        qkv.copy_(raw)
        K.zero_()
        Q.zero_()

    def run(between=lambda: None):
        ck.rotate_qk(raw, Hq, Hkv, d, cos, sin, pos, gain, gain, out_q=tokens(Q), out_k=tokens(K))
        between()
        got = list(ck.compress_layer(q_obs, K, V, Hq, w, c, budget))
        between()
        ck.rotate_qk(raw, Hq, Hkv, d, cos, sin, pos, None, None, out_q=tokens(Q), out_k=tokens(K))
        between()
        got += ck.gather(K, V, reuse)[:2]
        between()
        ck.rotate_qk(raw, Hq, Hkv, d, cos, sin, pos, gain, gain, out_q=tokens(Q), out_k=tokens(K))
        between()
        got.append(ck.compress_layer_paged(q_obs, K, V, Hq, w, c, budget, table, *cache))
        between()
        ck.rotate_qk(qkv, Hq, Hkv, d, cos, sin, pos, gain, gain, out_q=heads[:, :Hq], out_k=heads[:, Hq:Hq + Hkv])
        between()
        got += ck.compress_layer_strided(q_obs, tokens(heads[:, Hq:Hq + Hkv]), tokens(heads[:, Hq + Hkv:]), Hq, w, c, budget)
        between()
        return got + cache

    restore()
    torch.cuda.synchronize()
    want = [t.clone() for t in run(torch.cuda.synchronize)]
    assert all(t.any() for t in want)
    if captured:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        restore()
        with torch.cuda.stream(side):
            run()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = run()
    for _ in range(15):
        restore()
        if captured:
            graph.replay()
        got = held if captured else run()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    assert ck.device_status() == 0
