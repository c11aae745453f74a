"""Several GPUs in one process: what a launch needs set on its device is set on each.  The
library is linked with runtime entry points that only note what they are asked."""

import ctypes
import os
import subprocess

import pytest

from paper_2608_15018_amd import _lib, build

SHIM = r"""
#include <hip/hip_runtime.h>
#include <set>
#include <utility>
#include <vector>
namespace {
int device = 0, missing = 0, launches = 0, sets = 0;
std::set<std::pair<int, const void*>> allowed;
struct Config { dim3 grid, block; size_t lds; hipStream_t stream; };
std::vector<Config> configs;
}
extern "C" {
void shim_device(int d) { device = d; }
int shim_fail = 0;  // the next so many attribute calls fail
int shim_missing() { return missing; }
int shim_launches() { return launches; }
int shim_sets() { return sets; }
hipError_t __wrap_hipGetDevice(int* d) { *d = device; return hipSuccess; }
hipError_t __wrap_hipGetLastError() { return hipSuccess; }
hipError_t __wrap_hipFuncSetAttribute(const void* f, hipFuncAttribute, int) {
  ++sets;
  if (shim_fail > 0) { --shim_fail; return hipErrorOutOfMemory; }
  allowed.insert({device, f});
  return hipSuccess;
}
hipError_t __wrap___hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, hipStream_t s) {
  configs.push_back({g, b, lds, s});
  return hipSuccess;
}
hipError_t __wrap___hipPopCallConfiguration(dim3* g, dim3* b, size_t* lds, hipStream_t* s) {
  const Config c = configs.back();
  configs.pop_back();
  *g = c.grid; *b = c.block; *lds = c.lds; *s = c.stream;
  return hipSuccess;
}
hipError_t __wrap_hipLaunchKernel(const void* f, dim3, dim3, void**, size_t lds, hipStream_t) {
  ++launches;
  if (lds > 65536 && !allowed.count({device, f})) ++missing;
  return hipSuccess;
}
}
"""
WRAPPED = ["hipGetDevice", "hipGetLastError", "hipFuncSetAttribute", "__hipPushCallConfiguration", "__hipPopCallConfiguration", "hipLaunchKernel"]


@pytest.fixture()
def lib(tmp_path):
    objs = [os.path.join(build.OBJDIR, os.path.splitext(s)[0] + ".o") for s in build.SOURCES]
    if not all(os.path.exists(o) for o in objs):
        build.build(verbose=False)
    src, out = tmp_path / "shim.cpp", tmp_path / "libs2moe_shim.so"
    src.write_text(SHIM)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__=1", "-I", build.ROCM_INC, str(src), *objs,
                    *[f"-Wl,--wrap={n}" for n in WRAPPED], "-L", os.path.join(rocm, "lib"), "-lamdhip64",
                    "-Wl,-rpath," + os.path.join(rocm, "lib"), "-o", str(out)], check=True)
    return ctypes.CDLL(str(out))


A, B = 0x10000000, 0x40000000


def prompt(lib, D, n_tokens):
    f = lib.s2moe_prompt_attention
    f.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32] + [ctypes.c_void_p] * 6
    a = _lib.Attn(32, 8, D, _lib.BF16, 0.125, 32 * D, 8 * D, 8 * D, 32 * D)
    return f(ctypes.byref(a), 1, n_tokens, A, A, A, A, B, None)


def tree(lib, D, dtype, nodes):
    f = lib.s2moe_tree_attention
    P = ctypes.c_void_p
    f.argtypes = [P, ctypes.c_int32, P, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, P, P, P, P, P, ctypes.c_size_t, P, P]
    c = _lib.KvCacheStruct(1, 8, D, 8, 16, 4, 4, dtype, A, A, A, A, A)
    a = _lib.Attn(32, 8, D, dtype, 0.125, 32 * D, 0, 0, 32 * D)
    return f(ctypes.byref(c), 0, ctypes.byref(a), 1, nodes, nodes, A, A, A, A, A, 1 << 40, B, None)


def everything(lib):
    """Each kernel that asks for more than 64 KB of LDS."""
    return [prompt(lib, D, n) for D in (64, 128) for n in (100, 9000)] + \
        [tree(lib, D, t, nodes) for D in (64, 128) for t in (_lib.F32, _lib.BF16) for nodes in (1, 64)]


def test_each_device_gets_its_attributes(lib):
    for device in (0, 1, 0, 7):
        lib.shim_device(device)
        assert everything(lib) == [_lib.OK] * 12
    assert lib.shim_launches() > 48 and lib.shim_missing() == 0


def test_an_attribute_is_set_once_on_a_device(lib):
    everything(lib)
    n = lib.shim_sets()
    everything(lib)
    assert lib.shim_sets() == n


def test_a_call_that_could_not_set_it_fails_and_the_next_tries_again(lib):
    fail = ctypes.c_int.in_dll(lib, "shim_fail")
    for call in (lambda: prompt(lib, 128, 9000), lambda: tree(lib, 128, _lib.BF16, 64), lambda: tree(lib, 64, _lib.BF16, 1)):
        fail.value = 1
        assert call() == _lib.EHIP
        assert call() == _lib.OK
    assert lib.shim_missing() == 0
