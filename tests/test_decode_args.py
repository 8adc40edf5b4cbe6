"""What the calls on the decode cache refuse, through the C ABI and through the binding, without a GPU."""
import pytest
import torch

import paper_2502_00299_b200 as ck
from paper_2502_00299_b200 import binding
from tests.test_native_binding import Fake, _refused

OK, NULL, SHAPE, ALIGN, NOWS, LARGE = 0, -1, -2, -3, -4, -7
P = 256                                             # an address that is aligned and never read


def _rotate(T=4, row=1536, Hq=8, Hkv=2, d=128, x=P, gq=None, gk=None, eps=1e-6, co=P, si=P, n_pos=10, pos=P, st=(1024, 128, 256, 128), oq=P, ok=P):
    return ck.lib.chunkkv_rotate_qk(x, row, T, Hq, Hkv, d, gq, gk, eps, co, si, n_pos, pos, *st, oq, ok, None)


def _append(B=4, row=1536, Hq=8, Hkv=2, d=128, x=P, gq=None, gk=None, eps=1e-6, co=P, si=P, n_pos=10, pos=P, table=P, per=3, ln=P, page=16, pages=12,
            K=P, V=P, oq=P):
    return ck.lib.chunkkv_append_paged(x, row, B, Hq, Hkv, d, gq, gk, eps, co, si, n_pos, pos, table, per, ln, page, pages, K, V, oq, None)


def _attend(B=4, Hq=8, Hkv=2, d=128, q=P, table=P, per=3, ln=P, page=16, pages=12, K=P, V=P, weights=None, out=P, scratch=P, size=0):
    return ck.lib.chunkkv_attend_paged(q, table, per, ln, page, pages, K, V, B, Hq, Hkv, d, weights, out, scratch, size, None)


def _evict(B=4, Hkv=2, d=128, weights=P, table=P, per=3, ln=P, page=16, pages=12, K=P, V=P, w=4, c=2, budget=20, idx=P):
    return ck.lib.chunkkv_evict_paged(weights, table, per, ln, page, pages, K, V, B, Hkv, d, w, c, budget, idx, None)


HEADS = [dict(Hq=9), dict(Hkv=0), dict(Hq=0), dict(Hq=1), dict(d=96), dict(d=256), dict(Hq=65536, Hkv=1)]
CACHE = [dict(page=0), dict(pages=0), dict(per=0), dict(per=-1), dict(per=1 << 26), dict(pages=1 << 27)]


def test_sizes_are_refused():
    for call, n in ((_rotate, "T"), (_append, "B"), (_attend, "B")):
        for bad in HEADS + [{n: -1}, {n: 1 << 28}]:
            assert call(**bad) == SHAPE, bad
        assert call(**{n: 0}) == OK                             # nothing to do
    for call in (_append, _attend, _evict):
        for bad in CACHE:
            assert call(**bad) == SHAPE, bad
    for bad in (dict(Hkv=0), dict(d=96), dict(B=-1), dict(w=-1), dict(c=0), dict(budget=4, w=4, c=2), dict(budget=0, w=0, c=1), dict(w=2**31 - 1, c=2**31 - 1)):
        assert _evict(**bad) == SHAPE, bad
    assert _evict(B=0) == OK and _evict(B=0, w=0, c=1, budget=1) == OK and _evict(B=0, budget=5, w=4, c=2) == OK
    assert _evict(per=4096, page=16, c=1) == LARGE and _evict(B=0, per=4095, page=16, c=1) == OK      # 65536 chunks are one too many
    assert _evict(B=0, per=4096, page=16, c=2) == OK
    for bad in (dict(row=1279), dict(n_pos=0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(st=(1024, 64, 256, 128)),
                dict(st=(1024, 128, 252, 128)), dict(st=(-1024, 128, 256, 128))):
        assert _rotate(**bad) == SHAPE, bad
    for bad in (dict(row=1535), dict(n_pos=0), dict(eps=-1.0), dict(eps=float("nan"))):
        assert _append(**bad) == SHAPE, bad
    assert _attend(B=1, Hkv=8, Hq=8, per=1 << 29, page=1) == NOWS
    assert _attend(B=8, Hkv=8, Hq=8, per=1 << 29, page=1) == SHAPE      # 2^31 steps of 16 rows and heads


def test_missing_and_unaligned_pointers_are_refused():
    for name in ("x", "co", "si", "pos", "oq", "ok"):
        assert _rotate(**{name: None}) == NULL and _rotate(**{name: P + 2}) == ALIGN, name
    for name in ("x", "co", "si", "pos", "table", "ln", "K", "V", "oq"):
        assert _append(**{name: None}) == NULL and _append(**{name: P + 2}) == ALIGN, name
    for name in ("gq", "gk"):
        assert _rotate(**{name: P + 8}) == ALIGN and _append(**{name: P + 8}) == ALIGN
    assert _rotate(row=1540) == ALIGN and _append(row=1540) == ALIGN
    for name in ("q", "table", "ln", "K", "V", "out"):
        assert _attend(**{name: None}) == NULL and _attend(**{name: P + 2}) == ALIGN, name
    assert _attend(weights=P + 2) == ALIGN
    for name in ("weights", "table", "ln", "K", "V", "idx"):
        assert _evict(**{name: None}) == NULL and _evict(**{name: P + 2}) == ALIGN, name


def test_scratch_of_attention():
    size = ck.lib.chunkkv_attend_scratch_bytes
    need = size(4, 8, 2, 128, 3, 16, 0)                       # short caches take one launch and hardly any scratch
    assert need == 256
    need = size(4, 8, 2, 128, 600, 16, 0)
    assert need > 256 and _attend(per=600, size=need - 1) == NOWS and size(4, 8, 2, 128, 600, 16, 1) >= need + 4 * 8 * 9600 * 4
    assert _attend(per=600, size=need, weights=P) == NOWS and _attend(per=600, scratch=None, size=need) == NOWS and _attend(per=600, scratch=P + 16, size=need) == ALIGN
    for bad in ((0, 8, 2, 128, 3, 16, 0), (4, 9, 2, 128, 3, 16, 0), (4, 8, 2, 96, 3, 16, 0), (4, 8, 2, 128, 0, 16, 0), (4, 8, 2, 128, 3, 0, 0)):
        assert size(*bad) == 0
    # never less for more rows or sequences
    last = 0
    for per in (1, 2, 5, 40, 300, 8192):
        now = size(3, 32, 8, 128, per, 16, 0)
        assert now >= last and size(4, 32, 8, 128, per, 16, 0) >= now
        last = now


def _kinds(*shape, dtype=torch.bfloat16):
    other = torch.float16 if dtype != torch.float16 else torch.float32
    return [Fake(*shape, dtype=dtype, cuda=False), Fake(*shape, dtype=other), Fake(*shape, dtype=dtype, contiguous=False)]


def _elsewhere(*shape, dtype=torch.bfloat16):
    t = Fake(*shape, dtype=dtype)
    t.device = torch.device("cuda", 1)
    return t


F32, I32 = torch.float32, torch.int32
B, Hq, Hkv, d, page, pages, per = 3, 8, 2, 64, 16, 9, 2
CACHE_GOOD = dict(block_tables=Fake(B, per, dtype=I32), lengths=Fake(B, Hkv, dtype=I32), cache_K=Fake(pages, page, Hkv, d), cache_V=Fake(pages, page, Hkv, d))
CACHE_BAD = {"block_tables": [Fake(B + 1, per, dtype=I32), Fake(B * per, dtype=I32), Fake(B, per, dtype=torch.int64), _elsewhere(B, per, dtype=I32)],
             "lengths": [Fake(B, Hkv + 1, dtype=I32), Fake(B * Hkv, dtype=I32), Fake(B, Hkv, dtype=torch.int64), _elsewhere(B, Hkv, dtype=I32)],
             "cache_K": _kinds(pages, page, Hkv, d) + [Fake(pages, page, Hkv * d), _elsewhere(pages, page, Hkv, d)],
             "cache_V": _kinds(pages, page, Hkv, d) + [Fake(pages - 1, page, Hkv, d), _elsewhere(pages, page, Hkv, d)]}
ANGLES_GOOD = dict(cos=Fake(50, d // 2, dtype=F32), sin=Fake(50, d // 2, dtype=F32), positions=Fake(B, dtype=I32))
ANGLES_BAD = {"cos": _kinds(50, d // 2, dtype=F32) + [Fake(50, d, dtype=F32), Fake(50 * d // 2, dtype=F32)],
              "sin": _kinds(50, d // 2, dtype=F32) + [Fake(49, d // 2, dtype=F32), _elsewhere(50, d // 2, dtype=F32)],
              "positions": [Fake(B - 1, dtype=I32), Fake(B, dtype=torch.int64), _elsewhere(B, dtype=I32)]}
GAINS_BAD = {"q_gain": _kinds(d) + [Fake(d - 1), _elsewhere(d)], "k_gain": _kinds(d) + [Fake(d - 1)]}


def test_the_binding_refuses_tensors():
    row = (Hq + 2 * Hkv) * d
    call = lambda **k: ck.rotate_qk(k.pop("qkv"), Hq, Hkv, d, **k)
    outs = {"out_q": [Fake(B, Hq, d, cuda=False), Fake(B, Hq, d, dtype=F32), Fake(B + 1, Hq, d), Fake(B, Hkv, d), _elsewhere(B, Hq, d)], "out_k": [Fake(B, Hq, d)]}
    _refused(call, dict(qkv=Fake(B, row), **ANGLES_GOOD), {"qkv": _kinds(B, row) + [Fake(B, (Hq + Hkv) * d - 1), Fake(B * row)], **ANGLES_BAD, **GAINS_BAD, **outs})
    call = lambda **k: ck.append_paged(k.pop("qkv"), Hq, **k)
    _refused(call, dict(qkv=Fake(B, row), **ANGLES_GOOD, **CACHE_GOOD),
             {"qkv": _kinds(B, row) + [Fake(B, row - 1)], **ANGLES_BAD, **CACHE_BAD, **GAINS_BAD, "out_q": _kinds(B, Hq, d) + [Fake(B, Hq - 1, d), _elsewhere(B, Hq, d)]})
    sums = [Fake(B, Hkv, per * page - 1, dtype=F32), Fake(B, Hkv, per * page), Fake(B, Hkv, per * page, dtype=F32, contiguous=False), Fake(B * Hkv, per * page, dtype=F32)]
    _refused(ck.attend_paged, dict(q=Fake(B, Hq, d), **CACHE_GOOD),
             {"q": _kinds(B, Hq, d) + [Fake(B, Hq * d), Fake(B, Hq, 128)], **CACHE_BAD, "weights": sums, "out": _kinds(B, Hq, d) + [Fake(B, Hq, d - 1), _elsewhere(B, Hq, d)]})
    call = lambda **k: ck.evict_paged(**k, w=4, c=2, budget=20)
    bad = {k: v for k, v in CACHE_BAD.items() if k not in ("lengths", "block_tables")}
    _refused(call, dict(weights=Fake(B, Hkv, per * page, dtype=F32), **CACHE_GOOD),
             {**bad, "weights": sums, "lengths": [Fake(B, Hkv + 1, dtype=I32), Fake(B, Hkv, dtype=torch.int64)], "block_tables": [Fake(B + 1, per, dtype=I32)],
              "out_idx": [Fake(B, Hkv, 19, dtype=I32), Fake(B, Hkv, 20, dtype=torch.int64), _elsewhere(B, Hkv, 20, dtype=I32)]})


def test_tensors_on_the_host_are_refused():
    x = torch.zeros(2, 64, 64, dtype=torch.bfloat16)
    for call in (lambda: ck.rotate_qk(x[0], 1, 1, 64, x[0], x[0], x[0]), lambda: ck.append_paged(x[0], 1, x[0], x[0], x[0], x, x, x[None], x[None]),
                 lambda: ck.attend_paged(x, x, x, x[None], x[None]), lambda: ck.evict_paged(x, x, x, x[None], x[None], 1, 1, 1)):
        with pytest.raises(ValueError):
            call()
    for name in ("rotate_qk", "append_paged", "attend_paged", "evict_paged"):
        with pytest.raises(TypeError):
            getattr(binding._native, name)(1, 2, 3)


def test_a_stream_of_another_device_is_refused():
    class Stream:
        device = torch.device("cuda", 1)

    with pytest.raises(ValueError, match="stream must be one of cuda:0"):
        with binding._on(torch.device("cuda", 0), Stream()):
            pass
