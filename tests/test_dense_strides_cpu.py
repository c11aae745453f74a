"""Scales whose rows share memory (expanded from one row, or closer together than they are
wide) are refused by the library before anything is launched, as codes are: their strides
reach it as they are.  Tensors on the host that say they are on a GPU stand for tensors
there."""

import pytest

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402
from paper_2608_15018_amd import _lib  # noqa: E402
from tests.test_dense_binding import gpu, lib, rows, weight, zeros  # noqa: E402,F401

E4M3 = s2.E4M3
M, N, K = 6, 300, 400  # three blocks of weight rows, four of k


@pytest.fixture
def here(monkeypatch):
    """The library itself, with its own checks."""
    monkeypatch.setattr(_lib, "_stream", lambda s: 0)
    monkeypatch.setattr(_lib, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)


def shared(n, cols):
    """[n, cols] whose rows are one, and whose rows begin before the last one's end."""
    yield zeros(1, cols).expand(n, cols)
    for step in (1, cols - 1):
        yield torch.as_strided(zeros(n * cols), (n, cols), (step, 1))


def refused(call, name):
    with pytest.raises(s2.S2moeError, match=name) as e:
        call()
    assert e.value.status == _lib.EINVAL


def test_scales_of_products(here):  # noqa: F811
    x, w = rows(M, K), weight(N, K)
    for s in shared(4, M):
        refused(lambda: s2.fp8_matmul(s2.Fp8Rows(x.codes, s), w), "ldxs")
    for s in shared(3, 4):
        refused(lambda: s2.fp8_matmul(x, s2.Fp8Weight(w.codes, s)), "ldws")


@pytest.mark.parametrize("write", [lambda out: s2.quantize(zeros(M, K), out), lambda out: s2.add_norm(zeros(M, K), zeros(K), out=out)])
def test_scales_that_are_written(here, write):  # noqa: F811
    codes = zeros(M, K, dtype=E4M3)
    for s in shared(4, M):
        refused(lambda: write(s2.Fp8Rows(codes, s)), "lds")


def test_codes_rows_and_results(here):
    x, w = rows(M, K), weight(N, K)
    one = zeros(1, K).expand(M, K)
    refused(lambda: s2.fp8_matmul(s2.Fp8Rows(zeros(1, K, dtype=E4M3).expand(M, K), x.scales), w), "ldx")
    refused(lambda: s2.fp8_matmul(x, s2.Fp8Weight(zeros(1, K, dtype=E4M3).expand(N, K), w.scales)), "ldw")
    refused(lambda: s2.fp8_matmul(x, w, out=zeros(1, N).expand(M, N)), "ldo")
    refused(lambda: s2.quantize(one), "ldx")
    refused(lambda: s2.quantize_weight(one), "ldw")
    refused(lambda: s2.add_norm(zeros(M, K), zeros(K), one), "ldr")
    refused(lambda: s2.add_norm(zeros(M, K), zeros(K), out=one), "ldo")


def test_a_single_row_or_block_may_have_any_stride(lib):  # noqa: F811
    """Of one row of scales the stride says nothing, and columns of wider arrays keep theirs."""
    s2.fp8_matmul(s2.Fp8Rows(zeros(M, 64, dtype=E4M3), torch.as_strided(zeros(M), (1, M), (0, 1))), weight(5, 64))
    _, a = lib.calls.pop()
    assert a[6] == M and a[10] == 1
    s2.fp8_matmul(s2.Fp8Rows(zeros(1, K, dtype=E4M3), zeros(4, 9)[:, 2:3]), s2.Fp8Weight(zeros(N, K, dtype=E4M3), zeros(3, 7)[:, :4]))
    _, a = lib.calls.pop()
    assert a[6] == 9 and a[10] == 7


def test_empty_batches_are_taken(here):
    x = s2.quantize(zeros(0, K))
    assert x.scales.shape == (4, 0) and s2.fp8_matmul(x, weight(N, K)).shape == (0, N)
    assert s2.add_norm(zeros(0, K), zeros(K), out=x) is x
