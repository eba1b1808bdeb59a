"""The paged-cache calls' scratch without a GPU: what outgrows it stays for the graphs that hold its address, and
nothing is allocated while a stream is being captured."""
import ctypes
import os
import subprocess

import pytest

from paper_2608_05780_gb300.build import CSRC, INCLUDE, nvcc
from test_cache_host import CALLS, EINVAL, _attention, _cache, _draft

# fake_cuda.cpp's cudaFree, counted by address.
FREES = """
#include <set>
#include <cuda_runtime.h>
static std::set<void*> g_freed;
extern "C" cudaError_t __real_cudaFree(void*);
extern "C" cudaError_t __wrap_cudaFree(void* p) { return g_freed.insert(p), __real_cudaFree(p); }
extern "C" int frees() { return static_cast<int>(g_freed.size()); }
"""


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    d = tmp_path_factory.mktemp("fake")
    out, frees = str(d / "libfakescratch.so"), str(d / "frees.cpp")
    with open(frees, "w") as f:
        f.write(FREES)
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc()))), "include")
    here = os.path.dirname(os.path.abspath(__file__))
    subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-I" + INCLUDE, "-I" + CSRC, "-I" + cuda, frees,
                    os.path.join(here, "fake_cuda.cpp"), os.path.join(here, "fake_cache.cpp"),
                    os.path.join(CSRC, "evisel_capi.cpp"), os.path.join(CSRC, "evisel_cache.cpp"), "-o", out,
                    "-Wl,-z,defs", "-Wl,-Bsymbolic", "-Wl,--wrap=cudaFree"], check=True)
    lib = ctypes.CDLL(out)
    lib.evisel_last_error.restype = ctypes.c_char_p
    lib.fake_fail.argtypes = [ctypes.c_char_p, ctypes.c_int]
    lib.fake_calls.argtypes = [ctypes.c_char_p]
    lib.evisel_free.argtypes = [ctypes.c_void_p]
    lib.evisel_workspace_bytes.argtypes = [ctypes.c_void_p]
    lib.evisel_workspace_bytes.restype = ctypes.c_int64
    return lib


def test_outgrown_scratch_stays(fake):
    """Batches one after the other, the smallest first: nothing is freed before the workspace, and what is held stays
    within a few times the largest."""
    ws, n = ctypes.c_void_p(None), fake.frees()
    held = []
    for batch in [*range(1, 40), 400, 3, 400]:
        assert _attention(fake, ctypes.byref(ws), c=_cache(batch=batch)) == 0
        held.append(fake.evisel_workspace_bytes(ws))
    assert fake.frees() == n and held == sorted(held) and held[-1] == held[-3] > held[0]
    alone = ctypes.c_void_p(None)
    assert _attention(fake, ctypes.byref(alone), c=_cache(batch=400)) == 0
    assert held[-1] <= 4.5 * fake.evisel_workspace_bytes(alone)
    fake.evisel_free(alone)
    n = fake.frees()
    fake.evisel_free(ws)
    assert fake.frees() >= n + 3                 # the scratches, the status word


def test_a_failed_growth_keeps_the_scratch(fake):
    ws = ctypes.c_void_p(None)
    assert _attention(fake, ctypes.byref(ws)) == 0
    n, held = fake.frees(), fake.evisel_workspace_bytes(ws)
    fake.fake_fail(b"cudaMalloc", 0)
    assert _attention(fake, ctypes.byref(ws), c=_cache(batch=64)) == -5
    assert fake.frees() == n and fake.evisel_workspace_bytes(ws) == held
    fake.evisel_free(ws)


@pytest.mark.parametrize("call", CALLS)
def test_no_workspace_is_made_in_a_capture(fake, call):
    ws, launches, mallocs = ctypes.c_void_p(None), fake.fake_launches(), fake.fake_calls(b"cudaMalloc")
    fake.fake_capture(1)
    try:
        assert CALLS[call](fake, ctypes.byref(ws)) == EINVAL and b"capture" in fake.evisel_last_error()
    finally:
        fake.fake_capture(0)
    assert ws.value is None and fake.fake_launches() == launches and fake.fake_calls(b"cudaMalloc") == mallocs


def test_scratch_does_not_grow_in_a_capture(fake):
    """The larger call is refused, the workspace as it was; the same size is captured; after the capture it grows."""
    ws = ctypes.c_void_p(None)
    large = dict(c=_cache(batch=64), d=_draft(tokens=200, q_stride=(1 << 20, 3584, 128)))
    assert _attention(fake, ctypes.byref(ws)) == 0
    held, n, launches = fake.evisel_workspace_bytes(ws), fake.frees(), fake.fake_launches()
    fake.fake_capture(1)
    try:
        assert _attention(fake, ctypes.byref(ws), **large) == EINVAL and b"capture" in fake.evisel_last_error()
        assert fake.fake_launches() == launches
        for call in CALLS.values():
            assert call(fake, ctypes.byref(ws)) == 0
    finally:
        fake.fake_capture(0)
    assert fake.evisel_workspace_bytes(ws) == held and fake.frees() == n
    assert _attention(fake, ctypes.byref(ws), **large) == 0
    fake.evisel_free(ws)
