"""Angles next to a whole turn keep their own precision: a position and a frequency whose
product is just below a multiple of 2 pi, or a little below zero, turn by that little.

How far off a sine may be there, relative to it: four units in its last place (2^-21, which
OpenCL allows a sine of half turns), the turn's rounding to fp32 and one product (2^-24 each),
under 2^-20; absolute, position and frequency are multiplied in 64 bits, off by 2^-51 of the
angle; then one rounding to the type."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from tests.test_gpu_rotate import DT, HALF, ints, make, np64  # noqa: E402


def near_whole_turns():
    """(position, frequency) whose product is within 4e-7 of 2 pi times a whole number, or tiny."""
    out = [(-1, 1e-9), (-1, 1e-7), (-3, 2e-5), (-1000, 1e-8), (1, 1e-9), (7, 1e-8)]
    for p in (1, 3, 7, 50, 1021, 65537, 1000003, -1, -5, -777, -100003):
        for turns in (1, 2, 5, 16):
            for step in (-1, 0, 1):
                f = np.float32(2 * np.pi * turns / abs(p))
                out.append((p, float(np.nextafter(f, np.float32(np.inf * step)) if step else f)))
    return out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [8, 1216])  # alone and in groups of eight
def test_angles_next_to_whole_turns(dtype, n):
    D, own = 64, {}
    for p, f in near_whole_turns():
        own.setdefault(p, []).append(f)
    c, _ = make(dtype, 1, D, 16, [0], [n])
    x = torch.zeros((n, 1, D), dtype=DT[dtype], device="cuda")
    x[..., D // 2:] = 1  # (0, 1) becomes (-sin, cos)
    for p, some in own.items():
        freq = np.array(some + [0.0] * (32 - len(some)), dtype=np.float32)
        k_out = torch.empty_like(x)
        got = c.append_rotated(0, x, x, x, ints([0]), ints([0, n]), ints([p] * n), torch.from_numpy(freq).cuda(), k_out=k_out)
        angle = np.longdouble(p) * freq.astype(np.longdouble)
        want = -np.sin(angle).astype(np.float64)
        slack = np.abs(want) * (HALF[dtype] + 2.0 ** -20) + np.abs(angle).astype(np.float64) * 2.0 ** -51
        for t in (got, k_out):
            off = (np.abs(np64(t)[:, 0, :32] - want) - slack).max(0)
            assert off.max() <= 0, (p, freq[off.argmax()], want[off.argmax()], off.max())
