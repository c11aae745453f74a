"""The products' kernels that need more than 64 KB of LDS are allowed it on each device that
they are launched on, and no form needs more than a workgroup can have.  The library is linked
with runtime entry points that only note what they are asked."""

import ctypes

from paper_2608_15018_amd import _lib
from tests.test_attention_devices_cpu import lib  # noqa: F401

A = 1 << 40


def product(lib, m, n, k, out):  # noqa: F811
    f = lib.s2moe_scaled_matmul
    P, N, I = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32
    f.argtypes = [I, I, I, P, N, P, N, P, N, P, N, P, N, I, P]
    return f(m, n, k, A, k, 2 * A, m, 3 * A, k, 4 * A, (k + 127) // 128, 5 * A, n, out, None)


# Every form: from one token to whole prompts.
SIZES = [(1, 512, 1024), (16, 5120, 1024), (16, 32000, 4096), (128, 2048, 1024), (300, 5120, 2880), (768, 5120, 4096), (2048, 2048, 1024),
         (1536, 5120, 1024), (4096, 16384, 4096), (8193, 6144, 4096)]


def test_each_device_gets_its_attributes(lib):  # noqa: F811
    for device in (0, 1, 0, 7):
        lib.shim_device(device)
        for out in (_lib.F32, _lib.BF16):
            assert [product(lib, *s, out) for s in SIZES] == [_lib.OK] * len(SIZES)
    assert lib.shim_missing() == 0 and lib.shim_sets() > 0
    n = lib.shim_sets()
    assert [product(lib, *s, _lib.BF16) for s in SIZES] == [_lib.OK] * len(SIZES) and lib.shim_sets() == n


def test_a_call_that_could_not_set_it_fails_and_the_next_tries_again(lib):  # noqa: F811
    fail = ctypes.c_int.in_dll(lib, "shim_fail")
    fail.value = 1
    assert product(lib, 4096, 16384, 4096, _lib.BF16) == _lib.EHIP
    assert product(lib, 4096, 16384, 4096, _lib.BF16) == _lib.OK
    assert lib.shim_missing() == 0


def test_the_largest_calls_launch(lib):  # noqa: F811
    """The largest arguments that are accepted find a form."""
    before = lib.shim_launches()
    for s in ((1 << 22, 4096, 16), (4096, 1 << 22, 16), (1 << 17, 1 << 17, 144), (1 << 22, 1, 1 << 18), (1, 1 << 22, 1 << 18)):
        assert product(lib, *s, _lib.BF16) == _lib.OK and product(lib, *s, _lib.F32) == _lib.OK
    assert lib.shim_launches() > before
