"""How the kernels on the decode cache read memory, from their sources: they are resident while the kernel ahead of them still writes queries, lengths,
rows and sums, and the read-only path is only for data that nothing writes in a kernel's lifetime, so they do not take it."""
import os
import re

import pytest

from paper_2502_00299_b200 import build


def _code(name):
    text = open(os.path.join(build.CSRC, name)).read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


@pytest.mark.parametrize("name", ["rotate.cu", "attend.cu", "evict.cu", "decode.cuh"])
def test_nothing_is_read_through_the_read_only_path(name):
    code = _code(name)
    # (a const pointer that promises to be the only one lets the compiler take that path by itself)
    assert not re.findall(r"__ldg\w*\s*\([^;]*;|ld\.global[\w.:]*\.nc[\w.:]*|const[^;,()]*\*\s*__restrict__\s*\w+", code)


@pytest.mark.parametrize("name", ["rotate.cu", "attend.cu", "evict.cu"])
def test_every_kernel_waits_for_the_one_ahead(name):
    """Each of them is launched as a programmatic dependent, so each has the wait on every way through it that reads."""
    code = _code(name)
    kernels = re.split(r"__global__", code)[1:]
    assert kernels and code.count("cudaLaunchAttributeProgrammaticStreamSerialization") >= 1
    for k in kernels:
        assert "begin_dependent();" in k or "griddepcontrol.wait;" in k
