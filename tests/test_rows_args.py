"""What the calls for tables, turns and shared prefixes refuse, through the C ABI and through the binding, without a GPU; how their kernels read memory
and what they were compiled to."""
import os
import re

import pytest
import torch

import paper_2502_00299_b200 as ck
from paper_2502_00299_b200 import binding, build
from tests.test_decode_args import ANGLES_BAD, ANGLES_GOOD, CACHE_BAD, CACHE_GOOD, GAINS_BAD, I32, F32, P, _elsewhere, _kinds, B, Hkv, Hq, d, page, pages, per
from tests.test_decode_loads import READ_ONLY, WAIT, _code
from tests.test_native_binding import Fake, _refused

OK, NULL, SHAPE, ALIGN, NOWS = 0, -1, -2, -3, -4


def _tables(n=4, first=0, rot=64, base=10000.0, kind=0, factor=2.0, original=4096.0, low=1.0, high=32.0, scale=1.0, co=P, si=P):
    return ck.lib.chunkkv_rope_tables(n, first, rot, base, kind, factor, original, low, high, scale, co, si, None)


def _rotate(T=4, row=1536, Hq=8, Hkv=2, d=128, rot=128, inter=0, x=P, gq=None, gk=None, eps=1e-6, co=P, si=P, n_pos=10, pos=P, st=(1024, 128, 256, 128), oq=P,
            ok=P):
    return ck.lib.chunkkv_rotate_rows(x, row, T, Hq, Hkv, d, rot, inter, gq, gk, eps, co, si, n_pos, pos, *st, oq, ok, None)


def _append(T=4, B=2, starts=P, row=1536, Hq=8, Hkv=2, d=128, rot=128, inter=0, x=P, gq=None, gk=None, eps=1e-6, co=P, si=P, n_pos=10, pos=P, table=P, per=3,
            ln=P, page=16, pages=12, K=P, V=P, oq=P):
    return ck.lib.chunkkv_append_rows_paged(x, row, T, starts, B, Hq, Hkv, d, rot, inter, gq, gk, eps, co, si, n_pos, pos, table, per, ln, page, pages, K, V, oq,
                                            None)


def _attend(T=4, B=2, starts=P, Hq=8, Hkv=2, d=128, q=P, table=P, per=3, ln=P, page=16, pages=12, K=P, V=P, causal=1, out=P, scratch=P, size=0):
    return ck.lib.chunkkv_attend_rows_paged(q, T, starts, table, per, ln, page, pages, K, V, B, Hq, Hkv, d, causal, out, scratch, size, None)


def _shared(B=4, P_=2, starts=P, Hq=8, Hkv=2, d=128, q=P, pt=P, pper=5, pl=P, table=P, per=3, ln=P, page=16, pages=12, K=P, V=P, out=P, scratch=P, size=0):
    return ck.lib.chunkkv_attend_shared_paged(q, starts, P_, pt, pper, pl, table, per, ln, page, pages, K, V, B, Hq, Hkv, d, out, scratch, size, None)


HEADS = [dict(Hq=9), dict(Hkv=0), dict(Hq=0), dict(Hq=1), dict(d=96), dict(d=256), dict(Hq=65536, Hkv=1)]
CACHE = [dict(page=0), dict(pages=0), dict(per=0), dict(per=-1), dict(per=1 << 26), dict(pages=1 << 27)]


def test_sizes_are_refused():
    inf, nan = float("inf"), float("nan")
    for bad in (dict(n=-1), dict(rot=8), dict(rot=40), dict(rot=144), dict(base=1.0), dict(base=nan), dict(base=inf), dict(kind=-1), dict(kind=4), dict(scale=nan),
                dict(first=2**31 + 1), dict(first=-2**31 - 1), dict(kind=1, factor=0.0), dict(kind=2, factor=nan), dict(kind=2, original=0.0),
                dict(kind=2, low=0.0), dict(kind=3, low=4.0, high=4.0), dict(kind=3, high=inf), dict(kind=3, high=nan)):
        assert _tables(**bad) == SHAPE, bad
    assert _tables(n=0) == OK and _tables(n=0, factor=0.0, original=-1.0, low=9.0) == OK and _tables(n=0, kind=1, original=0.0) == OK
    for call in (_rotate, _append, _attend):
        for bad in HEADS + [dict(T=-1), dict(T=1 << 28)]:
            assert call(**bad) == SHAPE, bad
        assert call(T=0) == OK                                              # nothing to do
    for bad in HEADS + [dict(B=-1), dict(B=1 << 28), dict(P_=-1), dict(P_=1 << 28), dict(pper=0)]:
        assert _shared(**bad) == SHAPE, bad
    assert _shared(B=0) == OK and _append(B=0) == OK and _attend(B=0) == OK
    for call in (_append, _attend, _shared):
        for bad in CACHE:
            assert call(**bad) == SHAPE, bad
    for call in (_append, _attend):
        for bad in (dict(B=-1), dict(B=1 << 28)):
            assert call(**bad) == SHAPE, bad
    for call in (_rotate, _append):
        for bad in (dict(rot=0), dict(rot=24), dict(rot=144), dict(d=64, rot=80), dict(inter=2), dict(inter=-1), dict(n_pos=0), dict(eps=-1.0), dict(eps=nan), dict(eps=inf)):
            assert call(**bad) == SHAPE, bad
    for bad in (dict(row=1279), dict(st=(1024, 64, 256, 128)), dict(st=(1024, 128, 252, 128)), dict(st=(-1024, 128, 256, 128))):
        assert _rotate(**bad) == SHAPE, bad
    assert _append(row=1535) == SHAPE and _attend(causal=2) == SHAPE
    # blocks times tiles of 128 rows: 8 heads of (T / 256 + B) blocks, 2^22 tiles
    assert _attend(T=4, B=16, Hq=8, Hkv=8, per=1 << 29, page=1) == NOWS and _attend(T=4, B=64, Hq=8, Hkv=8, per=1 << 29, page=1) == SHAPE
    assert _shared(P_=0, pper=0, starts=None, pt=None, pl=None) == NOWS


def test_missing_and_unaligned_pointers_are_refused():
    for name in ("co", "si"):
        assert _tables(**{name: None}) == NULL and _tables(**{name: P + 4}) == ALIGN, name
    for name in ("x", "co", "si", "pos", "oq", "ok"):
        assert _rotate(**{name: None}) == NULL and _rotate(**{name: P + 2}) == ALIGN, name
    for name in ("x", "starts", "co", "si", "pos", "table", "ln", "K", "V", "oq"):
        assert _append(**{name: None}) == NULL and _append(**{name: P + 2}) == ALIGN, name
    for name in ("gq", "gk"):
        assert _rotate(**{name: P + 8}) == ALIGN and _append(**{name: P + 8}) == ALIGN
    assert _rotate(row=1540) == ALIGN and _append(row=1540) == ALIGN
    for name in ("q", "starts", "table", "ln", "K", "V", "out"):
        assert _attend(**{name: None}) == NULL and _attend(**{name: P + 2}) == ALIGN, name
    for name in ("q", "starts", "pt", "pl", "table", "ln", "K", "V", "out"):
        assert _shared(**{name: None}) == NULL and _shared(**{name: P + 2}) == ALIGN, name


def test_scratch():
    rows, shared = ck.lib.chunkkv_attend_rows_scratch_bytes, ck.lib.chunkkv_attend_shared_scratch_bytes
    need = rows(4, 2, 8, 2, 128)
    assert need > 0 and _attend(size=need - 1) == NOWS and _attend(size=need, scratch=None) == NOWS and _attend(size=need, scratch=P + 16) == ALIGN
    need = shared(4, 2, 8, 2, 128)
    assert need > 0 and _shared(size=need - 1) == NOWS and _shared(size=need, scratch=None) == NOWS and _shared(size=need, scratch=P + 16) == ALIGN
    for bad in ((0, 2, 8, 2, 128), (4, 0, 8, 2, 128), (4, 2, 9, 2, 128), (4, 2, 8, 2, 96), (-1, 2, 8, 2, 128)):
        assert rows(*bad) == 0
    for bad in ((0, 2, 8, 2, 128), (4, -1, 8, 2, 128), (4, 2, 9, 2, 128), (4, 2, 8, 2, 96)):
        assert shared(*bad) == 0
    assert shared(4, 0, 8, 2, 128) > 0
    last = 0
    for T in (1, 2, 5, 40, 300, 8192):                                      # never less for more tokens or sequences
        now = rows(T, 3, 32, 8, 128)
        assert now >= last and rows(T, 4, 32, 8, 128) >= now and shared(T, 3, 32, 8, 128) >= shared(T, 2, 32, 8, 128)
        last = now


T = 7
STARTS = [Fake(B, dtype=I32), Fake(B + 1, 1, dtype=I32), Fake(B + 1, dtype=torch.int64), _elsewhere(B + 1, dtype=I32)]


def test_the_binding_refuses_tensors():
    row = (Hq + 2 * Hkv) * d
    good = dict(ANGLES_GOOD, positions=Fake(T, dtype=I32))
    bad = dict(ANGLES_BAD, positions=[Fake(T - 1, dtype=I32), Fake(T, dtype=torch.int64), _elsewhere(T, dtype=I32)],
               cos=_kinds(50, d // 2, dtype=F32) + [Fake(50 * d // 2, dtype=F32)],
               sin=_kinds(50, d // 2, dtype=F32) + [Fake(49, d // 2, dtype=F32), Fake(50, d // 4, dtype=F32), _elsewhere(50, d // 2, dtype=F32)])
    # (the number of sequences is that of lengths)
    cache = dict(CACHE_BAD, lengths=[Fake(B, Hkv + 1, dtype=I32), Fake(B, Hkv, dtype=torch.int64), _elsewhere(B, Hkv, dtype=I32)])
    call = lambda **k: ck.rotate_rows(k.pop("qkv"), Hq, Hkv, d, **k)
    outs = {"out_q": [Fake(T, Hq, d, cuda=False), Fake(T, Hq, d, dtype=F32), Fake(T + 1, Hq, d), _elsewhere(T, Hq, d)], "out_k": [Fake(T, Hq, d)]}
    _refused(call, dict(qkv=Fake(T, row), **good), {"qkv": _kinds(T, row) + [Fake(T, (Hq + Hkv) * d - 1), Fake(T * row)], **bad, **GAINS_BAD, **outs})
    call = lambda **k: ck.append_rows_paged(k.pop("qkv"), Hq, **k)
    _refused(call, dict(qkv=Fake(T, row), starts=Fake(B + 1, dtype=I32), **good, **CACHE_GOOD),
             {"qkv": _kinds(T, row) + [Fake(T, row - 1)], "starts": STARTS, **bad, **cache, **GAINS_BAD, "out_q": _kinds(T, Hq, d) + [Fake(T, Hq - 1, d), _elsewhere(T, Hq, d)]})
    out = _kinds(T, Hq, d) + [Fake(T, Hq, d - 1), _elsewhere(T, Hq, d)]
    _refused(ck.attend_rows_paged, dict(q=Fake(T, Hq, d), starts=Fake(B + 1, dtype=I32), **CACHE_GOOD),
             {"q": _kinds(T, Hq, d) + [Fake(T, Hq * d), Fake(T, Hq, 128)], "starts": STARTS, **cache, "out": out})
    out = _kinds(B, Hq, d) + [Fake(B, Hq, d - 1), _elsewhere(B, Hq, d)]
    _refused(ck.attend_shared_paged,
             dict(q=Fake(B, Hq, d), starts=Fake(3, dtype=I32), prefix_tables=Fake(2, 4, dtype=I32), prefix_lengths=Fake(2, Hkv, dtype=I32), **CACHE_GOOD),
             {"q": _kinds(B, Hq, d) + [Fake(B, Hq * d), Fake(B, Hq, 128), Fake(B + 1, Hq, d)], "starts": [Fake(2, dtype=I32), Fake(3, dtype=torch.int64), _elsewhere(3, dtype=I32)],
              "prefix_tables": [Fake(3, 4, dtype=I32), Fake(8, dtype=I32), Fake(2, 4, dtype=torch.int64), _elsewhere(2, 4, dtype=I32)],
              "prefix_lengths": [Fake(2, Hkv + 1, dtype=I32), Fake(2, Hkv, dtype=torch.int64), _elsewhere(2, Hkv, dtype=I32)], **CACHE_BAD, "out": out})


def test_names_and_numbers_of_tables():
    with pytest.raises(ValueError, match="scaling must be one of"):
        ck.rope_tables(4, 64, 10000.0, "yes")
    for bad in (torch.zeros(4, 32), torch.zeros(4, 16, dtype=torch.float64)):
        with pytest.raises(ValueError):
            ck.rope_tables(4, 64, 10000.0, out_cos=bad)
    with pytest.raises(ValueError):
        ck.rope_tables(4, 64, 10000.0, device="cpu")


def test_tensors_on_the_host_are_refused():
    x = torch.zeros(2, 64, 64, dtype=torch.bfloat16)
    for call in (lambda: ck.rotate_rows(x[0], 1, 1, 64, x[0], x[0], x[0]), lambda: ck.append_rows_paged(x[0], 1, x[0], x[0], x[0], x[0], x, x, x[None], x[None]),
                 lambda: ck.attend_rows_paged(x, x, x, x, x[None], x[None]), lambda: ck.attend_shared_paged(x, x, x, x, x, x, x[None], x[None])):
        with pytest.raises(ValueError):
            call()
    for name in ("rope_tables", "rotate_rows", "append_rows_paged", "attend_rows_paged", "attend_shared_paged"):
        with pytest.raises(TypeError):
            getattr(binding._native, name)(1, 2, 3)


@pytest.mark.parametrize("name", ["rotate_rows.cu", "attend_rows.cu"])
def test_dependent_kernels_read_behind_their_wait(name):
    code = _code(name)
    assert not READ_ONLY.findall(code)
    kernels = re.split(r"__global__", code)[1:]
    assert kernels and code.count("cudaLaunchAttributeProgrammaticStreamSerialization") >= 1
    for k in kernels:
        assert any(w in k for w in WAIT)


def test_registers_that_warps_hand_to_one_another():
    """Warps that raise their number of registers wait for it: what all take has to be there, of 384 threads."""
    build.build()
    path = build.report_path("attend_rows.cu")
    if not os.path.exists(path):
        pytest.skip("the library came built without its reports")
    found, name = [], None
    for line in open(path):
        m = re.search(r"Compiling entry function '(\S+)'", line)
        name = m.group(1) if m else name
        m = re.search(r"Used (\d+) registers", line)
        if m and "attend_rows_kernel" in name:
            found.append(int(m.group(1)))
    code = _code("attend_rows.cu")
    up, down = int(re.search(r"setmaxnreg_inc<(\d+)>", code).group(1)), int(re.search(r"setmaxnreg_dec<(\d+)>", code).group(1))
    assert len(found) == 2 and all(384 * n >= 256 * up + 128 * down for n in found)
