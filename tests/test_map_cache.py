"""Tensor maps kept between calls (csrc/ff_tensor_map.h, FFMapCache), compiled for the host with a driver that only notes what it is
asked for: which maps are encoded again, and that what comes out is always the map asked for, with the address asked for."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_22808_b200", "csrc")
SHIM = r"""
#include <string.h>
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
namespace shim {                         // (names of its own: the library itself may be in the same process)
CUresult replace(CUtensorMap* map, void* base) { map->opaque[0] = (cuuint64_t)base; return CUDA_SUCCESS; }
CUresult encode() { return CUDA_SUCCESS; }
cudaError_t entry_point(const char* name, void** fn, unsigned long long, cudaDriverEntryPointQueryResult*) {
  *fn = strcmp(name, "cuTensorMapReplaceAddress") ? (void*)encode : (void*)replace;
  return cudaSuccess;
}
#define cudaGetDriverEntryPoint entry_point
#include "ff_tensor_map.h"
}
using shim::FFMapCache;
extern "C" {
void* make() { return new FFMapCache(); }
void drop(void* cache) { delete (FFMapCache*)cache; }
int places() { return FFMapCache::N; }
// 1: the map was encoded, 0: it was kept, -1: not the map that was asked for
int get(void* cache, unsigned long long base, int code, int slices) {
  CUtensorMap map = {};
  int encoded = 0;
  const bool ok = ((FFMapCache*)cache)->get(&map, (const void*)base, code, slices, [&] {
    map.opaque[0] = base; map.opaque[1] = (cuuint64_t)code; map.opaque[2] = (cuuint64_t)slices;
    encoded = 1;
    return true;
  });
  return ok && map.opaque[0] == base && map.opaque[1] == (cuuint64_t)code && map.opaque[2] == (cuuint64_t)slices ? encoded : -1;
}
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cxx, nvcc = shutil.which("g++") or shutil.which("c++"), shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    assert cxx, "no C++ compiler"
    folder = tmp_path_factory.mktemp("map_cache")
    source, out = str(folder / "shim.cpp"), str(folder / "shim.so")
    with open(source, "w") as f:
        f.write(SHIM)
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    subprocess.run([cxx, "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-I", include, "-o", out, source], check=True)
    lib = ctypes.CDLL(out)
    lib.make.restype = ctypes.c_void_p
    lib.drop.argtypes = [ctypes.c_void_p]
    lib.get.argtypes = [ctypes.c_void_p, ctypes.c_ulonglong, ctypes.c_int, ctypes.c_int]
    return lib


@pytest.fixture
def cache(lib):
    handle, address = lib.make(), iter(range(1 << 20, 1 << 30, 64))
    yield lambda code, slices: lib.get(handle, next(address), code, slices)
    lib.drop(handle)


def test_as_many_kinds_as_places(lib, cache):
    kinds = [(c, s) for c in range(lib.places() // 2) for s in (3, 70000)]
    assert [cache(*k) for k in kinds] == [1] * len(kinds)
    for _ in range(3):
        assert [cache(*k) for k in kinds] == [0] * len(kinds)


def test_many_token_counts(cache):
    """Weights, whose kinds every call has, are encoded once, however many token counts have been there; a count that comes again soon is
    kept, the latest ones as the first."""
    weights, tokens = [(64, 2048), (64, 5632), (1064, 2048)], [(128, 0), (1128, 0), (32, 0), (1032, 0)]

    def call(M):
        return [cache(*k) for k in weights], [cache(code, M) for code, _ in tokens]
    assert call(1) == ([1] * 3, [1] * 4)
    for M in range(2, 60):
        assert call(M) == ([0] * 3, [1] * 4)
        assert call(M) == ([0] * 3, [0] * 4)
        assert call(M - 1) == ([0] * 3, [0] * 4)
