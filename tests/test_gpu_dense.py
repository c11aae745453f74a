"""Norms, 8-bit rows and weights and their products against 64 bits.

How far off results may be: a rounding to a type is off by at most half its step; what
comes before it is fp32, off by at most SLACK of the value: the sum of squares of 72 terms
a lane, one after another, and ten more additions and operations, each 2^-24, halved by the
square root, and six factors: under 2^-18."""

import numpy as np
import pytest

from oracle import dense_oracle as do

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
SLACK = 2.0 ** -18
EPS = 1e-6


def np64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(shape, dtype, g, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(DT[dtype])


def wide(t, extra):
    """The same matrix as columns of a wider array whose other columns are NaN."""
    big = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), device="cuda").to(t.dtype)
    big[:, :t.shape[1]] = t
    return big[:, :t.shape[1]]


def check_codes(rows, y, label=""):
    codes, scales = np64(rows.codes), np64(rows.scales)
    want = do.row_scales(y)
    assert np.all(np.abs(scales - want) <= want * SLACK), label
    z = y / do.spread_rows(want, y.shape[1])
    off = np.abs(codes - z) - do.half_step(z) - np.abs(z) * 2 * SLACK
    assert off.max() <= 0, (label, np.unravel_index(off.argmax(), off.shape), off.max())


def check(got, want, dtype, label=""):
    off = np.abs(np64(got) - want) - np.abs(want) * (HALF[dtype] + SLACK)
    assert off.max() <= 0, (label, off.max())


# ------------------------------------------------------------------------------- norm


@pytest.mark.parametrize("x,r,w,out", [("bf16", "f32", "bf16", "e4m3"), ("bf16", "bf16", "f32", "e4m3"), ("f32", "f32", "f32", "f32"),
                                       ("bf16", "none", "bf16", "bf16"), ("f32", "bf16", "bf16", "bf16"), ("f32", "none", "f32", "e4m3")])
@pytest.mark.parametrize("n,H", [(1, 16), (1, 2048), (3, 48), (5, 512), (7, 528), (2, 1168), (9, 2064), (4, 2880), (3, 4096), (2, 4112),
                                 (3, 8192), (2, 8208), (2, 16384), (130, 256)])
def test_add_norm(x, r, w, out, n, H):
    g = gen(n * 100003 + H)
    xt, wt = randn((n, H), x, g, 3.0), randn((H,), w, g)
    rt = None if r == "none" else randn((n, H), r, g)
    h, y = do.add_norm(np64(xt), None if rt is None else np64(rt), np64(wt), EPS)
    got = s2.add_norm(xt, wt, rt, EPS, out_dtype=DT[out])
    if rt is not None:
        check(rt, h, r, "residual")
    if out == "e4m3":
        assert isinstance(got, s2.Fp8Rows) and got.codes.shape == (n, H) and got.scales.shape == (do.blocks_of(H), n)
        check_codes(got, y)
    else:
        assert got.dtype == DT[out]
        check(got, y, out)


def test_add_norm_strides_and_rows_of_larger_arrays():
    g, n, H = gen(1), 6, 2880
    x, r, w = randn((n, H), "bf16", g), randn((n, H), "f32", g), randn((H,), "f32", g)
    xt, rt = wide(x, 64), wide(r, 16)
    h, y = do.add_norm(np64(x), np64(r), np64(w), EPS)
    codes = torch.zeros((n + 4, H + 32), dtype=torch.uint8, device="cuda").view(DT["e4m3"])
    scales = torch.full((do.blocks_of(H), n + 4), 7.0, device="cuda")
    out = s2.Fp8Rows(codes[2:n + 2, :H], scales[:, 1:n + 1])
    assert s2.add_norm(xt, w, rt, EPS, out=out) is out
    check(rt, h, "f32")
    check_codes(out, y)
    assert (scales[:, 0] == 7).all() and (scales[:, n + 1:] == 7).all()
    assert not codes.view(torch.uint8)[:, H:].any() and not codes.view(torch.uint8)[:2].any() and not codes.view(torch.uint8)[n + 2:].any()
    assert torch.isnan(rt._base[:, H:]).all()


def test_rows_of_zeros_and_of_huge_and_tiny_values():
    H, w = 272, torch.ones(272, device="cuda")
    x = torch.zeros((5, H), device="cuda")
    x[1, 5] = 1e15
    x[2] = 1e-30
    x[3, :128] = 2.0 ** -110
    x[4, 200] = -3.0
    _, y = do.add_norm(np64(x), None, np64(w), EPS)
    check_codes(s2.add_norm(x, w, None, EPS, out_dtype=DT["e4m3"]), y)
    check_codes(s2.quantize(x), np64(x))
    check(s2.add_norm(x, w, None, EPS), y, "f32")
    zero = s2.quantize(torch.zeros((2, 16), device="cuda", dtype=torch.bfloat16))
    assert not zero.codes.view(torch.uint8).any() and (zero.scales == torch.tensor(2.0 ** -100 / 448)).all()
    big = s2.quantize(torch.full((1, 16), 3.0e38, device="cuda"))
    assert (big.codes.float() == 448).all() and torch.isfinite(big.scales).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_row_that_is_not_finite_touches_no_other(bad):
    g, n, H = gen(2), 9, 640
    x, w = randn((n, H), "bf16", g), randn((H,), "bf16", g)
    wq = s2.quantize_weight(randn((40, H), "f32", g))
    clean = s2.add_norm(x, w, out_dtype=DT["e4m3"])
    y = s2.fp8_matmul(clean, wq, out_dtype=torch.float32)
    x[4, 333] = bad
    dirty = s2.add_norm(x, w, out_dtype=DT["e4m3"])
    z = s2.fp8_matmul(dirty, wq, out_dtype=torch.float32)
    rest = [i for i in range(n) if i != 4]
    assert torch.equal(clean.codes.view(torch.uint8)[rest], dirty.codes.view(torch.uint8)[rest])
    assert torch.equal(clean.scales[:, rest], dirty.scales[:, rest]) and torch.equal(y[rest], z[rest])
    assert torch.isnan(z[4]).all()


# ----------------------------------------------------------------------- 8-bit matrices


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,K", [(1, 16), (3, 128), (5, 144), (2, 2880), (33, 512), (7, 528), (1, 20000), (300, 272)])
def test_quantize(dtype, n, K):
    x = randn((n, K), dtype, gen(n + K), 5.0)
    x[:, K // 2] *= 30
    check_codes(s2.quantize(wide(x, 16)), np64(x))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,K", [(1, 16), (17, 144), (128, 128), (129, 272), (300, 2880), (255, 48)])
def test_quantize_weight(dtype, n, K):
    w = randn((n, K), dtype, gen(n + K))
    got = s2.quantize_weight(wide(w, 16))
    want = do.weight_scales(np64(w))
    assert got.codes.shape == (n, K) and np.all(np.abs(np64(got.scales) - want) <= want * SLACK)
    z = np64(w) / do.spread_weight(want, n, K)
    assert (np.abs(np64(got.codes) - z) - do.half_step(z) - np.abs(z) * 2 * SLACK).max() <= 0


# ---------------------------------------------------------------------------- products


def operands(m, n, k, g, full=False):
    """Codes and scales; `full`: any finite code, scales of very different sizes."""
    if full:
        code = lambda shape: torch.randint(0, 127, shape, generator=g, device="cuda", dtype=torch.uint8) \
            | torch.randint(0, 2, shape, generator=g, device="cuda", dtype=torch.uint8) << 7  # noqa: E731
        size = lambda *shape: torch.exp2(torch.randint(-8, 9, shape, generator=g, device="cuda").float()) \
            * (1 + torch.rand(shape, generator=g, device="cuda"))  # noqa: E731
        return (s2.Fp8Rows(code((m, k)).view(DT["e4m3"]), size(do.blocks_of(k), m)),
                s2.Fp8Weight(code((n, k)).view(DT["e4m3"]), size(do.blocks_of(n), do.blocks_of(k))))
    return s2.quantize(randn((m, k), "f32", g)), s2.quantize_weight(randn((n, k), "f32", g))


def check_product(got, x, w, dtype, label=""):
    """In fp32 each of a block's 128 additions is off by at most a whole step; then a factor,
    and one fused addition a block and at most 16 sums of parts.  For bf16 the 8-bit matrix
    instruction's cutting off comes to that."""
    k = x.codes.shape[1]
    args = [np64(t) for t in (*x, *w)]
    want, size = do.scaled_matmul(*args)
    slack = size * (2 * 128 + 2 * do.blocks_of(k) + 16) * 2.0 ** -24
    if dtype == "bf16":
        slack += do.cut_off(*args)
    off = np.abs(np64(got) - want) - slack * (1 + HALF[dtype]) - np.abs(want) * (HALF[dtype] + 2.0 ** -24)
    assert off.max() <= 0, (label, np.unravel_index(off.argmax(), off.shape), off.max())


SIZES = [(1, 1, 16), (1, 16, 128), (1, 17, 144), (1, 500, 2048), (2, 33, 272), (15, 64, 112), (16, 200, 640), (17, 129, 384), (33, 96, 2880),
         (64, 257, 256), (65, 130, 1040), (130, 70, 400), (251, 640, 512), (300, 1000, 144), (513, 260, 336)]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_product(m, n, k, out):
    g = gen(m * 7 + n * 3 + k)
    for full in (False, True):
        x, w = operands(m, n, k, g, full)
        check_product(s2.fp8_matmul(x, w, out_dtype=DT[out]), x, w, out, (m, n, k, full))


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_products_of_small_whole_numbers_are_exact(m, n, k, out):
    """Codes of -2 .. 2 and scales of 1, 2 and 4: every sum is a whole number below 2^24, and
    no product is cut off."""
    g = gen(m + n + k)
    whole = lambda *s: torch.randint(-2, 3, s, generator=g, device="cuda").float().to(DT["e4m3"])  # noqa: E731
    size = lambda *s: torch.exp2(torch.randint(0, 3, s, generator=g, device="cuda").float())  # noqa: E731
    x = s2.Fp8Rows(whole(m, k), size(do.blocks_of(k), m))
    w = s2.Fp8Weight(whole(n, k), size(do.blocks_of(n), do.blocks_of(k)))
    want, _ = do.scaled_matmul(*(np64(t) for t in (*x, *w)))
    assert np.abs(want).max() < 2 ** 24
    assert torch.equal(s2.fp8_matmul(x, w, out_dtype=DT[out]).cpu(), torch.from_numpy(want).float().to(DT[out]))


# Between them every form of the kernel for either type, whole tiles and a few tokens past them.
LARGE = [(257, 512, 400), (384, 2048, 1040), (700, 2050, 1024), (768, 5120, 1040), (1024, 5121, 1024), (1536, 5120, 2064), (2048, 2048, 1024),
         (257, 16400, 1024), (1025, 16384, 1040), (384, 32000, 1024), (2052, 6144, 2880), (90, 32000, 272), (33, 20000, 144), (16, 30001, 1168),
         (1, 9001, 1040), (20, 9000, 272), (27, 5001, 1040), (1, 9000, 272), (17, 9000, 528), (30, 12001, 1168),
         (33, 5001, 272), (50, 5001, 2064), (50, 5001, 528), (1, 9000, 4112), (33, 3000, 2064), (33, 3000, 1040), (17, 5001, 2064),
         (17, 2050, 272), (70, 30001, 1040), (17, 9000, 2064), (200, 5001, 272), (70, 9000, 272), (128, 9000, 272), (128, 20000, 272),
         (1, 20000, 272)]
# A wave's weight scales are 64 blocks at a time: rows of more than that, for each form.
LONG = [(1, 48, 70016), (17, 48, 70016), (1, 5001, 33040), (17, 5001, 33040), (17, 2050, 33040), (33, 3000, 33040), (33, 5001, 33040),
        (33, 9000, 8720), (200, 9000, 8720), (256, 2050, 8720), (600, 5001, 8720), (900, 9000, 8720), (2052, 2050, 8720),
        (128, 9000, 8720), (300, 5001, 8720), (50, 5001, 33040), (20, 9000, 33040), (2052, 3001, 8720)]


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", LARGE + LONG)
def test_large_products(m, n, k, out):
    """Whole numbers exactly, everywhere; other codes at rows and columns drawn."""
    g = gen(m + n + k)
    whole = lambda *s: torch.randint(-2, 3, s, generator=g, device="cuda").float().to(DT["e4m3"])  # noqa: E731
    size = lambda *s: torch.exp2(torch.randint(0, 3, s, generator=g, device="cuda").float())  # noqa: E731
    kb = do.blocks_of(k)
    x, w = s2.Fp8Rows(whole(m, k), size(kb, m)), s2.Fp8Weight(whole(n, k), size(do.blocks_of(n), kb))
    a = x.codes.double() * x.scales.t().repeat_interleave(128, 1)[:, :k]
    b = w.codes.double() * w.scales.repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]
    got = s2.fp8_matmul(x, w, out_dtype=DT[out])
    assert torch.equal(got, (a @ b.t().contiguous()).float().to(DT[out]))
    x, w = operands(m, n, k, g)
    got = s2.fp8_matmul(x, w, out_dtype=DT[out])
    assert torch.equal(got, s2.fp8_matmul(x, w, out_dtype=DT[out]))
    rows = torch.cat([torch.randperm(m, generator=g, device="cuda")[:40], torch.tensor([0, m - 1], device="cuda")])
    cols = torch.cat([torch.randperm(n, generator=g, device="cuda")[:128], torch.tensor([0, n - 1], device="cuda")])
    part = np64(got[rows][:, cols])
    xc, wc = np64(x.codes.float()[rows]), np64(w.codes.float()[cols])
    xs = np64(x.scales[:, rows])
    a, b = xc * do.spread_rows(xs, k), wc * np.repeat(np64(w.scales)[(cols // 128).cpu().numpy()], 128, axis=1)[:, :k]
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    slack = mag * (2 * 128 + 2 * kb + 16) * 2.0 ** -24
    if out == "bf16":  # eight products cut off 13 bits below the largest's exponent, 2^-10 of their sum at most
        slack = slack + mag * 2.0 ** -10
    off = np.abs(part - want) - slack * (1 + HALF[out]) - np.abs(want) * (HALF[out] + 2.0 ** -24)
    assert off.max() <= 0, (np.unravel_index(off.argmax(), off.shape), off.max())


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(2048, 5120, 2064), (1024, 5120, 1024), (384, 2048, 1040), (48, 2048, 1040), (16, 9000, 1040)])
def test_products_while_copies_delay_their_loads(m, n, k, out):
    """A workgroup's waves read what others of them have loaded: the same bits however long
    that takes."""
    g = gen(m + n + k)
    whole = lambda *s: torch.randint(-2, 3, s, generator=g, device="cuda").float().to(DT["e4m3"])  # noqa: E731
    one = lambda *s: torch.ones(s, device="cuda")  # noqa: E731
    kb = do.blocks_of(k)
    x, w = s2.Fp8Rows(whole(m, k), one(kb, m)), s2.Fp8Weight(whole(n, k), one(do.blocks_of(n), kb))
    want = (x.codes.float().double() @ w.codes.float().double().t().contiguous()).float().to(DT[out])
    src, dst = (torch.zeros(2 ** 28, dtype=torch.uint8, device="cuda") for _ in range(2))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(12):
            dst.copy_(src)
    got = [s2.fp8_matmul(x, w, out_dtype=DT[out]) for _ in range(24)]
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in got)


@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(5, 77, 272), (40, 129, 144), (200, 300, 400), (600, 520, 272)])
def test_product_of_parts_of_larger_arrays(m, n, k, out):
    """Rows, scales and results inside arrays whose other elements are NaN, and stay."""
    g = gen(m + n + k)
    x, w = operands(m, n, k, g)
    part = lambda t, r, c: wide(torch.cat([torch.full((r, t.shape[1]), float("nan"), device="cuda").to(t.dtype), t]), c)[r:]  # noqa: E731
    xp = s2.Fp8Rows(part(x.codes, 3, 16), wide(x.scales, 5))
    wp = s2.Fp8Weight(part(w.codes, 2, 48), wide(w.scales, 3))
    for extra in (0, 1, 3, 8):
        big = torch.full((m + 2, n + extra), 7.0, device="cuda", dtype=DT[out])
        s2.fp8_matmul(xp, wp, out=big[:m, :n])
        check_product(big[:m, :n], x, w, out, extra)
        assert (big[m:] == 7).all() and (big[:, n:] == 7).all()
    assert torch.equal(s2.fp8_matmul(xp, wp, out_dtype=DT[out]), s2.fp8_matmul(x, w, out_dtype=DT[out]))


@pytest.mark.parametrize("m", [1, 40, 300])
def test_weights_that_are_nan_reach_their_own_columns_alone(m):
    g = gen(m)
    x, w = operands(m, 300, 400, g)
    y = s2.fp8_matmul(x, w)
    w.codes.view(torch.uint8)[137, 399] = 0x7F
    z = s2.fp8_matmul(x, w)
    rest = [j for j in range(300) if j != 137]
    assert torch.isnan(z[:, 137]).all() and torch.equal(y[:, rest], z[:, rest])


def test_empty_batches():
    w = s2.quantize_weight(torch.ones((20, 32), device="cuda"))
    x = s2.quantize(torch.ones((0, 32), device="cuda"))
    assert x.codes.shape == (0, 32) and x.scales.shape == (1, 0)
    assert s2.fp8_matmul(x, w).shape == (0, 20)
    assert s2.add_norm(torch.ones((0, 32), device="cuda"), torch.ones(32, device="cuda")).shape == (0, 32)


# ------------------------------------------------------------------- streams and graphs


@pytest.mark.parametrize("m", [1, 48, 300])
def test_a_chain_on_another_stream_and_in_a_graph(m):
    """add_norm -> product -> quantize -> product: eager, on a stream of its own, captured and
    replayed on new inputs between eager calls."""
    H, n, g = 640, 384, gen(m)
    w1, w2 = (s2.quantize_weight(randn(s, "f32", g)) for s in ((n, H), (H, n)))
    nw = randn((H,), "bf16", g)
    x0, r0 = randn((m, H), "bf16", g), randn((m, H), "f32", g)

    def chain(x, r, stream=None):
        a = s2.add_norm(x, nw, r, out_dtype=s2.E4M3, stream=stream)
        y = s2.fp8_matmul(a, w1, stream=stream)
        return s2.fp8_matmul(s2.quantize(y, stream=stream), w2, out_dtype=torch.float32, stream=stream)

    def eager(x, r):
        r = r.clone()
        return chain(x, r), r

    want, res = eager(x0, r0)
    side, r1 = torch.cuda.Stream(), r0.clone()
    side.wait_stream(torch.cuda.current_stream())
    got = chain(x0, r1, side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(r1, res)
    x, r = x0.clone(), r0.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = chain(x, r)
    for i in range(4):
        x.copy_(randn((m, H), "bf16", g))
        r.copy_(randn((m, H), "f32", g))
        want, res = eager(x, r)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(r, res), i


# -------------------------------------------------------------------------- past 32 bits


def test_rows_past_four_gigabytes():
    """The same rows far behind others and alone, to the same bits."""
    n, H, tail = 300000, 8192, 3
    g = gen(5)
    x = torch.zeros((n, H), dtype=torch.bfloat16, device="cuda")
    x[-tail:] = randn((tail, H), "bf16", g)
    w, r = randn((H,), "bf16", g), torch.zeros((n, H), dtype=torch.bfloat16, device="cuda")
    alone = s2.add_norm(x[-tail:].clone(), w, torch.zeros((tail, H), dtype=torch.bfloat16, device="cuda"), out_dtype=s2.E4M3)
    far = s2.add_norm(x, w, r, out_dtype=s2.E4M3)
    assert torch.equal(r[-tail:], x[-tail:]) and not r[:-tail].any()
    assert torch.equal(far.codes[-tail:].view(torch.uint8), alone.codes.view(torch.uint8)) and torch.equal(far.scales[:, -tail:], alone.scales)
    del r, far
    alone, far = s2.quantize(x[-tail:].clone()), s2.quantize(x)
    assert torch.equal(far.codes[-tail:].view(torch.uint8), alone.codes.view(torch.uint8)) and torch.equal(far.scales[:, -tail:], alone.scales)


@pytest.mark.parametrize("m,n", [(40000, 32000), (33, 1000000)])
def test_products_past_four_gigabytes(m, n):
    """Results past 2^32 bytes, and weights past 2^32 bytes: exact whole numbers at the end."""
    k = 272 if m > 1000 else 4368
    g = gen(m)
    whole = lambda *s: torch.randint(-2, 3, s, generator=g, device="cuda", dtype=torch.int8).to(DT["e4m3"])  # noqa: E731
    one = lambda *s: torch.ones(s, device="cuda")  # noqa: E731
    kb = do.blocks_of(k)
    x, w = s2.Fp8Rows(whole(m, k), one(kb, m)), s2.Fp8Weight(whole(n, k), one(do.blocks_of(n), kb))
    got = s2.fp8_matmul(x, w, out_dtype=torch.float32)
    rows, cols = slice(max(0, m - 300), m), slice(n - 1000, n)
    want = x.codes[rows].float().double() @ w.codes[cols].float().double().t().contiguous()
    assert torch.equal(got[rows, cols], want.float())
    want = x.codes[:40].float().double() @ w.codes[cols].float().double().t().contiguous()
    assert torch.equal(got[:40, cols], want.float())
