"""8-bit rows and weights: elements half way between two codes, and blocks of every size, against
64 bits."""

import numpy as np
import pytest

from oracle import dense_oracle as do

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402
from tests.test_gpu_dense import DT, check_codes, gen, np64, randn, wide  # noqa: E402


def nearest(y, scales):
    """Codes of y / scales, half way ones to the even neighbour.  y and the largest magnitudes that
    the scales are made of hold bf16 values: a quotient of their whole numbers is a half way
    point exactly or further from it than 64 bits are off."""
    z = y * 448 / (scales * 448).astype(np.float32)
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(z), 2.0 ** -20))), -6) - 3)
    return np.round(z / step) * step, np.abs(z / step - np.floor(z / step) - 0.5) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_elements_half_way_between_codes_go_to_the_even_one(dtype):
    n, K = 160, 2064
    x = randn((n, K), "bf16", gen(21), 3.0).to(DT[dtype])
    y = np64(x)
    want, ties = nearest(y, do.spread_weight(do.weight_scales(y), n, K))
    assert ties.sum() > 200 and np.array_equal(np64(s2.quantize_weight(wide(x, 16)).codes), want)
    x *= torch.exp2(torch.randint(-20, 20, (n, 1), device="cuda", generator=gen(22)).float()).to(DT[dtype])
    y = np64(x)
    want, ties = nearest(y, do.spread_rows(do.row_scales(y), K))
    assert ties.sum() > 200 and np.array_equal(np64(s2.quantize(wide(x, 16)).codes), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_of_every_size(dtype):
    """Blocks from the type's least magnitudes to its largest keep their codes."""
    base = randn((1, 144), "bf16", gen(23)).clamp(-1, 1).float()
    base[0, 5] = base[0, 130] = 1.0
    x = torch.cat([base * 2.0 ** e for e in range(-126, 128, 2)]).to(DT[dtype])
    check_codes(s2.quantize(x), np64(x))
    got = [s2.quantize_weight(x[i:i + 1]) for i in range(len(x))]
    rows = s2.quantize(x)
    assert torch.equal(torch.cat([t.codes.view(torch.uint8) for t in got]), rows.codes.view(torch.uint8))
    assert torch.equal(torch.cat([t.scales for t in got]), rows.scales.t())


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_weights_that_are_not_finite_stay_in_their_block(bad):
    w, x = randn((300, 400), "f32", gen(24)), s2.quantize(randn((20, 400), "f32", gen(25)))
    clean = s2.quantize_weight(w)
    w[130, 270] = bad
    dirty = s2.quantize_weight(w)
    a, b = (t.codes.view(torch.uint8).clone() for t in (clean, dirty))
    a[128:256, 256:384] = b[128:256, 256:384] = 0
    assert torch.equal(a, b)
    s, t = clean.scales.clone(), dirty.scales.clone()
    s[1, 2] = t[1, 2] = 0
    assert torch.equal(s, t)
    y, z = (s2.fp8_matmul(x, t, out_dtype=torch.float32) for t in (clean, dirty))
    assert torch.equal(y[:, :128], z[:, :128]) and torch.equal(y[:, 256:], z[:, 256:]) and torch.isnan(z[:, 130]).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_rows_that_are_not_finite_touch_no_other(bad):
    x = randn((6, 400), "bf16", gen(26))
    clean = s2.quantize(x)
    x[3, 200] = bad
    dirty = s2.quantize(x)
    rest = [0, 1, 2, 4, 5]
    assert torch.equal(clean.codes.view(torch.uint8)[rest], dirty.codes.view(torch.uint8)[rest])
    assert torch.equal(clean.scales[:, rest], dirty.scales[:, rest])
    assert torch.isnan(dirty.codes.float()[3, 200])
