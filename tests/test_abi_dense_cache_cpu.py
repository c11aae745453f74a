"""Positions and rotated rows are not written over the cache's own arrays, which the same launch
reads or writes: refused before anything is enqueued."""

import ctypes

import pytest

import paper_2608_15018_amd as s2
from paper_2608_15018_amd import _lib

A, B, C, D, E, F, G = (i << 40 for i in range(1, 8))
# 2 layers of 8 pages of 2 heads, 16 slots, 64 wide, in bf16; 4 sequences of up to 4 pages.
CACHE = dict(k=(A, 2 * 8 * 2 * 16 * 64 * 2), v=(B, 2 * 8 * 2 * 16 * 64 * 2), table=(C, 4 * 4 * 4), length=(D, 4 * 4), refs=(E, 8 * 4))
N = 9


@pytest.fixture(scope="module")
def cache():
    return _lib.KvCacheStruct(2, 2, 64, 8, 16, 4, 4, _lib.BF16, *(CACHE[k][0] for k in ("k", "v", "table", "length", "refs")))


def at_both_ends(size, step):
    """Starts of `size` bytes that meet each array of the cache by its first and its last bytes."""
    for at, n in CACHE.values():
        yield at - size + step
        yield at + n - step


def refused(status):
    assert status == _lib.EINVAL and "cache" in _lib.last_error(), _lib.last_error()


@pytest.mark.parametrize("parent", [None, G + 4096])
def test_positions(cache, parent):
    for pos in at_both_ends(4 * N, 4):
        refused(s2.load().s2moe_kv_positions(ctypes.byref(cache), 2, N, G, G + 1024, parent, pos, None))


def test_rotated_rows(cache):
    lib = s2.load()
    q, k, ints = F, F + (1 << 30), G
    # Rows of one array, and of every other 512 elements of one.
    for ld in (256, 512):
        r = _lib.Rotation(4, 64, 0, 256, 128, 128, ld, ld)

        def call(q_out, k_out):
            return lib.s2moe_kv_append_rotated(ctypes.byref(cache), 0, ctypes.byref(r), 2, N, ints, ints + 1024, ints + 2048, ints + 4096, q, k,
                                               k + (1 << 20), q_out, k_out, None)

        for at in at_both_ends((N - 1) * ld * 2 + 256 * 2, 16):
            refused(call(at, None))
            refused(call(at, F + (1 << 35)))
        for at in at_both_ends((N - 1) * ld * 2 + 128 * 2, 16):
            refused(call(F + (1 << 35), at))
