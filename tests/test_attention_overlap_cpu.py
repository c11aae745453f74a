"""Whether an output may lie beside its inputs in one wider array.  Tree attention looks at
its workspace's size after it has looked for overlaps, so a call with a workspace of no size
ends there without a launch, where an overlap ends it before."""

import ctypes

import pytest

import paper_2608_15018_amd as s2
from paper_2608_15018_amd import _lib

A, W = 0x10000000, 0x70000000  # aligned fake addresses
HQ, D, N, LD = 4, 64, 9, 1024  # rows of 512 bytes in an array of 2048-byte rows
ROW, STEP = HQ * D * 2, LD * 2


def tree(q, out, ldq=LD, ldo=LD, n=N):
    lib = s2.load()
    c = _lib.KvCacheStruct(1, 2, D, 8, 16, 4, 4, _lib.BF16, A, A, A, A, A)
    a = _lib.Attn(HQ, 2, D, _lib.BF16, 0.125, ldq, 0, 0, ldo)
    status = lib.s2moe_tree_attention(ctypes.byref(c), 0, ctypes.byref(a), 1, n, n, q, A, A, A, W, 0, out, None)
    return {_lib.EWORKSPACE: "accepted", _lib.EINVAL: "overlaps"}[status] if "overlaps" in _lib.last_error() or status == _lib.EWORKSPACE \
        else pytest.fail(_lib.last_error())


def by_bytes(q, out, ldq, ldo, n):
    """The definition: a byte that both write or read."""
    rows = lambda at, ld: {at + i * ld * 2 + j for i in range(n) for j in range(0, ROW, 16)}  # noqa: E731
    return "overlaps" if rows(q, ldq) & rows(out, ldo) else "accepted"


@pytest.mark.parametrize("first", [0, 256, STEP - ROW])
def test_columns_of_one_array(first):
    """out at every 16 bytes of the rows that q is columns of; 16 bytes in common are refused."""
    q = A + first
    for at in range(-STEP, 2 * STEP, 16):
        out = A + at
        assert tree(q, out) == by_bytes(q, out, LD, LD, N), (first, at)
    free = [at for at in range(0, STEP, 16) if tree(q, A + at) == "accepted"]
    assert free and all((at - first) % STEP >= ROW and (at - first) % STEP <= STEP - ROW for at in free)


def test_before_and_after():
    q = A + 64 * STEP
    for out, want in ((q - N * STEP, "accepted"), (q + N * STEP, "accepted"), (q - (N - 1) * STEP - ROW, "accepted"),
                      (q - (N - 1) * STEP - ROW + 16, "overlaps"), (q + (N - 1) * STEP + ROW, "accepted"),
                      (q + (N - 1) * STEP + ROW - 16, "overlaps")):
        assert tree(q, out) == want == by_bytes(q, out, LD, LD, N)


def test_rows_of_different_steps():
    """Arrays whose extents are apart are accepted; others are refused unless their rows keep step."""
    assert tree(A, A + N * STEP, LD, LD // 2) == "accepted"
    assert tree(A, A + ROW, LD, LD // 2) == "overlaps"
    assert tree(A, A + ROW, LD, LD // 2, n=1) == "accepted"


def test_rows_without_gaps():
    for at in range(-ROW, ROW + 1, 16):
        want = "accepted" if abs(at) >= ROW else "overlaps"
        assert tree(A + 65536, A + 65536 + at, HQ * D, HQ * D, n=1) == want
    assert tree(A, A + N * ROW, HQ * D, HQ * D) == "accepted"
    assert tree(A, A + N * ROW - 16, HQ * D, HQ * D) == "overlaps"
