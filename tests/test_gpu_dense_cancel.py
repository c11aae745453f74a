"""Products whose terms cancel: how far bf16 results may be off is bounded by the terms and not
by the result, as documented; fp32 results are sums of exact products."""

import numpy as np
import pytest

from oracle import dense_oracle as do

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402
from tests.test_gpu_dense import DT, HALF, gen, np64  # noqa: E402


def codes(shape, least, g):
    """Any finite codes of magnitude number `least` and more, of either sign."""
    c = torch.randint(least, 127, shape, generator=g, device="cuda", dtype=torch.uint8)
    return (c | torch.randint(0, 2, shape, generator=g, device="cuda", dtype=torch.uint8) << 7).view(DT["e4m3"])


@pytest.mark.parametrize("m,n,k", [(3, 50, 256), (48, 200, 1024), (200, 300, 2304), (600, 1040, 512)])
@pytest.mark.parametrize("least,bound", [(8, 2.0 ** -10), (0, 2.0 ** -7)])  # codes from 8 on are 2^-6 and more
def test_sums_that_cancel(m, n, k, least, bound):
    """The second half of k repeats the first one's rows with weights of the other sign, but for
    their order within eights: every result is what little does not cancel."""
    g = gen(m + n + k)
    x, w = codes((m, k // 2), least, g).view(torch.uint8), codes((n, k // 2), least, g).view(torch.uint8)
    at = torch.randperm(k // 2, generator=g, device="cuda")
    extra = codes((n, 1), least, g).view(torch.uint8)
    other = w[:, at] ^ 128
    other[:, :1] = extra
    x, w = torch.cat((x, x[:, at]), 1).view(DT["e4m3"]), torch.cat((w, other), 1).view(DT["e4m3"])
    one = lambda *s: torch.ones(s, device="cuda")  # noqa: E731
    rows, weight = s2.Fp8Rows(x, one(do.blocks_of(k), m)), s2.Fp8Weight(w, one(do.blocks_of(n), do.blocks_of(k)))
    want, size = do.scaled_matmul(*(np64(t) for t in (*rows, *weight)))
    assert np.median(np.abs(want) / size) < 2.0 ** -6
    slack = size * (2 * 128 + 2 * do.blocks_of(k) + 16) * 2.0 ** -24
    for dtype, lost in (("f32", 0.0), ("bf16", bound)):
        got = np64(s2.fp8_matmul(rows, weight, out_dtype=DT[dtype]))
        off = np.abs(got - want) - (slack + size * lost) * (1 + HALF[dtype]) - np.abs(want) * (HALF[dtype] + 2.0 ** -24)
        assert off.max() <= 0, (dtype, off.max())
