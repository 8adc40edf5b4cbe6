"""How kernels that are launched as programmatic dependents read memory, from their sources: they are resident while the kernel ahead of them still writes
queries, keys, lengths, rows and sums, and the read-only path is only for data that nothing writes in a kernel's lifetime, so they do not take it."""
import os
import re

import pytest

from paper_2502_00299_b200 import build

# (a const pointer that promises to be the only one lets the compiler take that path by itself)
READ_ONLY = re.compile(r"__ldg\w*\s*\([^;]*;|ld\.global[\w.:]*\.nc[\w.:]*|const[^;,()]*\*\s*__restrict__\s*\w+")
WAIT = ("begin_dependent();", "griddepcontrol.wait;")


def _code(name):
    text = open(os.path.join(build.CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


@pytest.mark.parametrize("name", ["rotate.cu", "attend.cu", "evict.cu", "decode.cuh", "gather.cuh", "select.cuh", "resident.cuh", "panels.cuh", "ptx.cuh"])
def test_nothing_is_read_through_the_read_only_path(name):
    assert not READ_ONLY.findall(_code(name))


@pytest.mark.parametrize("name", [f for f in build.SOURCES if f not in ("api.cu", "diagnostics.cu", "score_noalloc.cu", "select.cu")])
def test_dependent_kernels_do_not_take_the_read_only_path(name):
    """Those that may be launched as dependents are those that wait."""
    dependent = [k for k in re.split(r"__global__", _code(name))[1:] if any(w in k for w in WAIT)]
    assert dependent
    for k in dependent:
        assert not READ_ONLY.findall(k), k[:200]


@pytest.mark.parametrize("name", ["rotate.cu", "attend.cu", "evict.cu"])
def test_every_kernel_waits_for_the_one_ahead(name):
    """Each of them is launched as a programmatic dependent, so each has the wait on every way through it that reads."""
    code = _code(name)
    kernels = re.split(r"__global__", code)[1:]
    assert kernels and code.count("cudaLaunchAttributeProgrammaticStreamSerialization") >= 1
    for k in kernels:
        assert any(w in k for w in WAIT)
