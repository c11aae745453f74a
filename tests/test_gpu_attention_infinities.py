"""Infinities and NaN among the values that rows see: the answer is the formula's, the same
wherever the token lies, and nothing else changes.

A coordinate of a row is a sum of weight times value over the tokens that the row sees, with
weights above zero: one infinity makes it that infinity, both signs or a NaN make it NaN.
Every other coordinate, and every other row, keeps its bits."""

import numpy as np
import pytest

from oracle import attention_oracle as ao
from tests.test_gpu_attention import DT, check, ints, random_parents, run_prompt, run_tree

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402

INF, NAN = float("inf"), float("nan")
# What two tokens' values are at one coordinate, and what a row gets that sees the first, the second, both.
PAIRS = [(INF, INF, INF, INF, INF), (-INF, -INF, -INF, -INF, -INF), (INF, -INF, INF, -INF, NAN), (-INF, INF, -INF, INF, NAN),
         (NAN, INF, NAN, INF, NAN), (-INF, NAN, -INF, NAN, NAN)]


def same(got, want):
    return torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0))


def expected(out, d, sees_a, sees_b, pair):
    """out with coordinate d of the rows (a boolean each [n]) replaced."""
    want = out.clone()
    for rows, value in ((sees_a & ~sees_b, pair[2]), (~sees_a & sees_b, pair[3]), (sees_a & sees_b, pair[4])):
        want[rows, :, d] = value
    return want


# Heads of at most 16 rows (keys split over the waves) and of more, D = 64 and 128; all query heads of a kv head.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,T", [((2, 1, 64), 7), ((2, 1, 128), 7), ((4, 2, 64), 40), ((4, 2, 128), 40), ((8, 1, 64), 40), ((8, 1, 128), 20)])
def test_tree_infinite_values(dtype, heads, T):
    """Tokens deep in the context (steps without masks), in its last, broken step, and in the tree."""
    n, P = 300, 16
    par = random_parents([T], 5)
    cache, att, args, out, _ = run_tree(dtype, heads, P, [n], [T], par, seed=5)
    seen, _ = ao.tree_visible(par)
    slots = [3, 130, 287, 290, 299, n, n + 2, n + T - 1]
    D = heads[2]

    def value(slot, d, x):
        page = int(cache.table[0, slot // P])
        old = cache.v[0, page, :, slot % P // 8, d, slot % 8].clone()
        cache.v[0, page, :, slot % P // 8, d, slot % 8] = x
        return old

    def sees(slot):
        return torch.tensor(np.ones(T, dtype=bool) if slot < n else seen[:, slot - n], device="cuda")

    for i, a in enumerate(slots):
        b = slots[(i + 3) % len(slots)]
        for j, pair in enumerate(PAIRS):
            d = (7 * i + 13 * j) % D
            old = value(a, d, pair[0]), value(b, d, pair[1])
            got = att(*args)
            assert same(got, expected(out, d, sees(a), sees(b), pair)), (a, b, pair)
            value(a, d, old[0]), value(b, d, old[1])
    assert torch.equal(att(*args), out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,lens", [((4, 2, 64), [60, 131, 30]), ((4, 2, 128), [60, 131, 30]), ((32, 8, 64), [40] * 60), ((32, 8, 128), [40] * 60),
                                        ((64, 32, 64), [1187, 1290]), ((64, 32, 128), [1187, 1290])])
def test_prompt_infinite_values(dtype, heads, lens):
    """Rows near such a token see it in a step with masks, later ones in a step without."""
    q, k, v, off, out = run_prompt(dtype, heads, lens, seed=6, wide=False)
    first, n = lens[0], lens[1]  # the second prompt
    row = torch.arange(sum(lens), device="cuda") - first
    at = [0, 5, 31, 32, n // 2, n - 3, n - 1]
    for i, a in enumerate(at):
        b = at[(i + 2) % len(at)]
        for j, pair in enumerate(PAIRS[i % 2::2]):
            d = (11 * i + 13 * j) % heads[2]
            w = v.clone()
            w[first + a, :, d], w[first + b, :, d] = pair[0], pair[1]
            inside = row < n
            got = s2.prompt_attention(q, k, w, off)
            assert same(got, expected(out, d, inside & (row >= a), inside & (row >= b), pair)), (a, b, pair)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_an_infinity_of_no_weight_is_treated_alike(dtype):
    """A weight that underflows to zero times an infinity: NaN in a step with masks as in one without."""
    n, D = 400, 64
    g = torch.Generator(device="cuda").manual_seed(7)
    q = torch.ones((n, 2, D), device="cuda").to(DT[dtype])
    k = torch.zeros((n, 1, D), device="cuda")
    k[1:, 0, 0] = -1000.0
    v = torch.randn((n, 1, D), generator=g, device="cuda").to(DT[dtype])
    v[100, 0, 9] = INF  # token 0 outweighs it by e^1000
    out = s2.prompt_attention(q, k.to(DT[dtype]), v, ints([0, n]), scale=1.0)
    assert out[100:, :, 9].isnan().all() and out[:100].isfinite().all()
    out[100:, :, 9] = 0
    assert out.isfinite().all()


# Forms of the prompt kernels: few rows and short, many rows and short, many rows and long.
FORMS = [((4, 2, 64), [60, 131, 30]), ((4, 2, 128), [60, 131, 30]), ((32, 8, 64), [40] * 60), ((32, 8, 128), [40] * 60),
         ((64, 32, 64), [1187, 1290]), ((64, 32, 128), [1187, 1290])]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,lens", FORMS)
def test_prompt_rows_of_scores_of_minus_infinity(dtype, heads, lens):
    """Keys that weigh nothing: the rows that see no other get zeros, the later ones what the others give."""
    q, k, v, off, _ = run_prompt(dtype, heads, lens, seed=8, wide=False)
    first, n, hidden = lens[0], lens[1], 37
    q[:, :, 0] = q[:, :, 0].abs() + 0.25
    k2 = k.clone()
    k2[first:first + hidden, :, 0] = -INF
    out = s2.prompt_attention(q, k2, v, off)
    assert not out[first:first + hidden].any()
    cut = ints([0, n - hidden])
    part = [t[first + hidden:first + n].contiguous() for t in (q, k, v)]
    want = ao.prompt_attention(*(t.double().cpu().numpy() for t in part), cut.tolist(), heads[2] ** -0.5)
    check(out[first + hidden:first + n], want, dtype)
    assert torch.equal(out[:first], s2.prompt_attention(q, k, v, off)[:first])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,T", [((2, 1, 64), 7), ((2, 1, 128), 7), ((4, 2, 64), 40), ((4, 2, 128), 40)])
def test_tree_rows_of_scores_of_minus_infinity(dtype, heads, T):
    cache, att, args, _, _ = run_tree(dtype, heads, 16, [300], [T], seed=9)
    layer, q, *rest = args
    q = q.clone()
    q[:, :, 0] = q[:, :, 0].abs() + 0.25
    cache.k[0, :, :, :, 0] = -INF
    assert not att(layer, q, *rest).any()
