"""Which kernel a product of 8-bit rows takes, without a GPU: the library linked with runtime
entry points that only note what is launched."""

import ctypes
import os
import re
import subprocess

from paper_2608_15018_amd import _lib, build
from tests import test_attention_devices_cpu as devices

NAMES = r"""
#include <map>
#include <string>
namespace {
std::string launched;
std::map<const void*, std::string>& names() { static std::map<const void*, std::string> m; return m; }
}
extern "C" {
const char* shim_take() { static std::string out; out.swap(launched); launched.clear(); return out.c_str(); }
void __wrap___hipRegisterFunction(void**, const void* f, char*, const char* name, unsigned, void*, void*, void*, void*, int*) { names()[f] = name; }
void shim_note(const void* f) { launched += names()[f]; launched += '\n'; }
}
"""


def _shim(where):
    objs = [os.path.join(build.OBJDIR, os.path.splitext(s)[0] + ".o") for s in build.SOURCES]
    if not all(os.path.exists(o) for o in objs):
        build.build(verbose=False)
    src, out = os.path.join(where, "names.cpp"), os.path.join(where, "libs2moe_names.so")
    text = NAMES + devices.SHIM.replace("  ++launches;\n", "  ++launches;\n  shim_note(f);\n")
    assert "shim_note(f)" in text
    with open(src, "w") as f:
        f.write(text)
    rocm = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "lib")
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__=1", "-I", build.ROCM_INC, src, *objs,
                    *[f"-Wl,--wrap={n}" for n in [*devices.WRAPPED, "__hipRegisterFunction"]], "-L", rocm, "-lamdhip64", "-Wl,-rpath," + rocm,
                    "-o", out], check=True)
    return out


A = 1 << 40


class Forms:
    """kernels(m, n, k, dtype): the kernels of a product, as tuples of a name and its numbers."""

    def __init__(self, where):
        self.lib = ctypes.CDLL(_shim(str(where)))
        P, N, I = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
        self.call = self.lib.s2moe_scaled_matmul
        self.call.argtypes = [I, I, I, P, N, P, N, P, N, P, N, P, N, I, P]
        self.lib.shim_take.restype = ctypes.c_char_p
        self.seen = {}

    def kernels(self, m, n, k, dtype):
        self.lib.shim_take()
        code = {"bf16": _lib.BF16, "f32": _lib.F32}[dtype]
        assert self.call(m, n, k, A, k, 2 * A, m, 3 * A, k, 4 * A, (k + 127) // 128, 5 * A, n, code, None) == _lib.OK
        return [self._name(s) for s in self.lib.shim_take().decode().split()]

    def _name(self, mangled):
        if mangled not in self.seen:
            kind = re.search(r"(stream|few_tokens|small_tiles|tiles)_kernel", mangled).group(1)
            self.seen[mangled] = (kind, *(int(v) for v in re.findall(r"L[ib](\d+)E", mangled)))
        return self.seen[mangled]
