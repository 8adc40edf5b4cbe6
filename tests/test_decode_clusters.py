"""Attention over short caches on a device where clusters of 16 CTAs have no room, without a GPU: the library's host code runs on a stand-in for the
CUDA calls, which notes what is launched and refuses clusters that the device does not take."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEVICE = r"""
#include <cuda_runtime_api.h>
#include <stdlib.h>
static int launched[64], n_launched, asked;
static int cluster_of(const cudaLaunchConfig_t* c) {
    for (unsigned i = 0; i < c->numAttrs; ++i)
        if (c->attrs[i].id == cudaLaunchAttributeClusterDimension) return c->attrs[i].val.clusterDim.x;
    return 1;
}
extern "C" {
int launches(int* out) { for (int i = 0; i < n_launched; ++i) out[i] = launched[i]; const int n = n_launched; n_launched = 0; return n; }
int times_asked() { return asked; }
cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int* v, cudaDeviceAttr a, int) { *v = a == cudaDevAttrMultiProcessorCount ? 148 : a == cudaDevAttrMaxSharedMemoryPerBlockOptin ? 232448 : 0; return cudaSuccess; }
cudaError_t cudaGetDriverEntryPoint(const char*, void** f, unsigned long long, cudaDriverEntryPointQueryResult* st) { *f = (void*)1; *st = cudaDriverEntryPointSuccess; return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaOccupancyMaxActiveClusters(int* n, const void*, const cudaLaunchConfig_t* c) {
    ++asked;
    *n = cluster_of(c) <= atoi(getenv("WIDEST")) ? 5 : 0;
    return atoi(getenv("WIDEST")) < 0 ? cudaErrorInvalidValue : cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void*, void**) {
    if (cluster_of(c) > 8 && cluster_of(c) > atoi(getenv("WIDEST"))) return cudaErrorInvalidClusterSize;
    launched[n_launched++] = cluster_of(c);
    return cudaSuccess;
}
}
"""
CALLS = """
import ctypes, sys
lib, device = ctypes.CDLL(sys.argv[1]), ctypes.CDLL(sys.argv[2])
lib.chunkkv_attend_scratch_bytes.restype = ctypes.c_size_t
P, seen = ctypes.c_void_p(256), []
def call(B, Hq, Hkv, d, rows, sums):
    need = lib.chunkkv_attend_scratch_bytes(B, Hq, Hkv, d, rows, 1, sums)
    args = (P, P, rows, P, 1, 10, P, P, B, Hq, Hkv, d, P if sums else None, P)
    if need > 256: assert lib.chunkkv_attend_paged(*args, P, ctypes.c_size_t(need - 1), None) == -4
    st = lib.chunkkv_attend_paged(*args, P, ctypes.c_size_t(need), None)
    out = (ctypes.c_int * 64)()
    n = device.launches(out)
    assert st == 0, (st, need)
    return list(out[:n]), need > 256
"""


@pytest.fixture(scope="module")
def device(tmp_path_factory):
    from paper_2502_00299_b200 import build
    build.build()
    cuda = os.path.dirname(os.path.dirname(os.path.realpath(build._nvcc())))
    d = tmp_path_factory.mktemp("device")
    (d / "device.cpp").write_text(DEVICE)
    so = str(d / "device.so")
    subprocess.run(["g++", "-shared", "-fPIC", "-isystem", os.path.join(cuda, "include"), "-o", so, str(d / "device.cpp")], check=True)

    def run(widest, code):
        r = subprocess.run([sys.executable, "-c", CALLS + code, build.LIB_PATH, so], env={**os.environ, "LD_PRELOAD": so, "WIDEST": str(widest)}, cwd=ROOT,
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-800:]
    return run


SHORT, LONG = 4000, 14000                     # rows: eight CTAs have room for the first, only 16 for the second


@pytest.mark.parametrize("widest", [16, 8, 0, -1])
def test_clusters_of_sixteen_only_where_they_have_room(device, widest):
    short, long_ = (([16], False),) * 2 if widest == 16 else (([8], False), ([1, 1], True))
    device(widest, f"""
for sums in (0, 1):
    for B, Hq, Hkv in ((1, 4, 1), (3, 24, 2), (1, 28, 7)):
        for d in (64, 128):
            assert call(B, Hq, Hkv, d, {SHORT}, sums) == {short}, (B, Hq, Hkv, d, sums)
            if Hkv == 1: assert call(B, Hq, Hkv, d, {LONG}, sums) == {long_}, (B, Hq, Hkv, d, sums)
assert device.times_asked() == 1
""")


@pytest.mark.parametrize("widest", [16, 8])
def test_smaller_clusters_are_the_same_on_every_device(device, widest):
    device(widest, """
for sums in (0, 1):
    for B, Hkv, rows, want in ((1, 8, 3501, 8), (1, 2, 1500, 8), (5, 4, 2000, 4), (16, 4, 1000, 2), (100, 1, 300, 1), (24, 8, 300, 1)):
        assert call(B, Hkv, Hkv, 128, rows, sums) == ([want], False), (B, Hkv, rows, sums)
    assert call(64, 32, 8, 128, 4160, sums) == ([1, 1], True)
assert device.times_asked() == 0
""")
