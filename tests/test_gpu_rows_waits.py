"""The waits of attend_rows_paged and attend_shared_paged: many launches with several pieces a CTA, warm and cold, and waits that run out."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2502_00299_b200 as ck
from tests.helpers import rand_bits, to_dev
from tests.test_gpu_rows import i32

pytestmark = pytest.mark.gpu
EDEVICE = -6


def turn(d, T, rows, Hq=32, Hkv=8, page=16):
    rng = np.random.default_rng(rows + d)
    per = -(-rows // page)
    K, V = (to_dev(rand_bits(rng, (per, page, Hkv, d))) for _ in range(2))
    q = to_dev(rand_bits(rng, (T, Hq, d)))
    return q, i32([0, T]), i32(rng.permutation(per)[None]), i32(np.full((1, Hkv), rows)), K, V


def wait_clocks(n):
    assert ck.lib.chunkkv_test_rows_wait_clocks(ctypes.c_longlong(n)) == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [64, 130, 960, 1024, 1088])                 # one, three, 15, 16 and 17 times 64 keys
def test_several_pieces_a_block_time_after_time(d, rows):
    """Several wide pieces one after the other on every SM, two to four times as many as there are SMs, and thin ones among them."""
    args = turn(d, 4096 + 17, rows)
    want = ck.attend_rows_paged(*args, False)
    flush = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")           # (the kernel's code leaves the caches too)
    off = torch.zeros((), dtype=torch.int64, device="cuda")
    for n in range(60):
        if n % 3 == 0:
            flush.zero_()
        off += (ck.attend_rows_paged(*args, False).view(torch.int16) != want.view(torch.int16)).sum()
    assert off.item() == 0 and ck.device_status() == 0 and want.any()


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_a_wait_that_runs_out_is_reported_once_and_the_next_call_is_right(d, shared):
    """With a limit of a single clock the warps that stand about while others work give up: the call ends, says so, and leaves nothing behind."""
    if shared:
        _, _, table, lengths, K, V = turn(d, 1, 32768)
        q = turn(d, 256, 32)[0]
        own = i32(np.full((256, 1), -1))
        call = lambda: ck.attend_shared_paged(q, i32([0, 256]), table, lengths, own, torch.zeros(256, 8, dtype=torch.int32, device="cuda"), K, V)  # noqa: E731
    else:
        args = turn(d, 4096, 16384)
        call = lambda: ck.attend_rows_paged(*args, False)  # noqa: E731
    want = call()
    assert ck.device_status() == 0
    wait_clocks(1)
    try:
        call()
        assert ck.device_status() == EDEVICE and ck.device_status() == 0
    finally:
        wait_clocks(0)
    for _ in range(3):
        assert torch.equal(call(), want)
    assert ck.device_status() == 0


def test_a_wait_for_long_work_does_not_run_out():
    """Warps that have nothing to do wait while others go through all rows of a long cache: beyond the limit's fixed part, here 2^28 clocks."""
    d, page, pages, per, T = 64, 128, 40, 160000, 256 * 148
    rng = np.random.default_rng(3)
    K = torch.zeros(pages, page, 1, d, dtype=torch.bfloat16, device="cuda")
    V = torch.tensor(rng.integers(-8, 9, K.shape), device="cuda").bfloat16()
    q = to_dev(rand_bits(rng, (T, 1, d)))
    table, lengths = i32(np.arange(per)[None] % pages), i32([[per * page]])  # (every page 4000 times: the mean of them once)
    wait_clocks(1 << 28)
    try:
        e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        e[0].record()
        out = ck.attend_rows_paged(q, i32([0, T]), table, lengths, K, V, False)
        e[1].record()
        assert ck.device_status() == 0
    finally:
        wait_clocks(0)
    assert e[0].elapsed_time(e[1]) > (1 << 28) / 1.965e6                     # ms, at the fastest clock
    # logits of 0 give weights of 1, added up 64 at a time, and sums of whole numbers below 2^24 are exact: a reciprocal, a product and a rounding are left
    ref = V.double().mean((0, 1, 2))
    sums = V.double().view(-1, d).cumsum(0).abs().max().item() + (ref.abs().max() * per * page).item()
    assert sums < 2 ** 24
    assert ((out.double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -22) * ref.abs()).all()
