"""What pins the oracle of the dense half: torch's own conversion to e4m3, closed forms, and
invariants."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import dense_oracle as do  # noqa: E402


def test_codes_are_those_of_torch():
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(codes, do.E4M3, equal_nan=True)
    assert np.nanmax(do.E4M3) == 448


def test_half_steps_bound_a_rounding_and_are_reached():
    z = np.random.default_rng(0).standard_normal(20000) * np.exp2(np.random.default_rng(1).integers(-12, 8, 20000))
    z = np.clip(z, -448, 448)
    c = torch.from_numpy(z).float().to(torch.float8_e4m3fn).float().numpy()
    off = np.abs(c - z) / do.half_step(z)
    assert off.max() <= 1 + 1e-6 and off.max() > 0.99


def test_scales_make_the_largest_code_448():
    y = np.random.default_rng(2).standard_normal((5, 300))
    s = do.row_scales(y)
    z = y / do.spread_rows(s, 300)
    assert s.shape == (3, 5)
    for k in range(0, 300, 128):
        assert np.allclose(np.abs(z[:, k:k + 128]).max(1), 448, rtol=1e-14)
    assert do.row_scales(np.zeros((1, 16)))[0, 0] == 2.0 ** -100 / 448
    w = np.random.default_rng(3).standard_normal((130, 140))
    assert np.abs(w / do.spread_weight(do.weight_scales(w), 130, 140)).max() <= 448 * (1 + 1e-14)


def test_norm_has_the_weights_size():
    x = np.random.default_rng(4).standard_normal((3, 64)) * 100
    h, y = do.add_norm(x, -x / 2, np.full(64, 2.0), 1e-12)
    assert np.allclose(h, x / 2) and np.allclose((y * y).mean(1), 4)


def test_product_of_ones():
    x, w = np.ones((2, 144)), np.ones((130, 144))
    xs, ws = np.array([[1.0, 2.0], [10.0, 20.0]]), np.array([[1.0, 0.5], [3.0, 0.25]])
    y, size = do.scaled_matmul(x, xs, w, ws)
    assert np.array_equal(y[:, 0], [128 + 16 * 5, 2 * (128 + 16 * 5)]) and np.array_equal(y, size)
    assert np.array_equal(y[:, 129], [3 * 128 + 16 * 2.5, 2 * (3 * 128 + 16 * 2.5)])


def test_positions_by_hand():
    assert do.positions([10, 0], [3, 2]).tolist() == [10, 11, 12, 0, 1]
    assert do.positions([5], [6], [-1, 0, 0, 1, 9, 4]).tolist() == [5, 6, 6, 7, 5, 6]


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation_keeps_lengths_and_depends_on_differences(neighbours):
    r = np.random.default_rng(5)
    q, k = r.standard_normal((1, 1, 32)), r.standard_normal((1, 1, 32))
    f = np.float32([1.0, 0.3, 0.01, 1e-4])
    dots = []
    for p in (0, 7, 100000):
        a, _ = do.rotate(q, [p + 3], f, neighbours)
        b, _ = do.rotate(k, [p], f, neighbours)
        assert np.isclose((a * a).sum(), (q * q).sum()) and np.array_equal(a[..., 8:], q[..., 8:])
        dots.append((a * b).sum())
    assert np.allclose(dots, dots[0])
    a, _ = do.rotate(np.eye(1, 4)[None], [1], np.float32([np.pi / 2, 0.0]), neighbours)
    assert np.allclose(a[0, 0], [0, 1, 0, 0] if neighbours else [0, 0, 1, 0], atol=1e-7)
