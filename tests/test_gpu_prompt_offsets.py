"""Prompt attention with offsets that make no sense: nothing outside the arrays, and no row
written twice."""

import pytest

from tests.test_gpu_attention import ints, run_prompt

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 2, 128)])
def test_offsets_that_do_not_ascend_write_nothing(dtype, heads):
    q, k, v, off, out = run_prompt(dtype, heads, [40, 50, 30], wide=False)
    for wrong in ([0, 90, 40, 120], [120, 0], [0, 40, 39, 120], [5, -3, 120, 120], list(range(0, 100)) + [7], [0, 120] * 512):
        dst = torch.full_like(out, 7.0)
        s2.prompt_attention(q, k, v, ints(wrong), out=dst)
        assert (dst == 7.0).all(), wrong[:4]
    # Ascending, but partly outside: the prompts that lie inside.
    for wrong, first, last in (([-5, 0, 40, 130], 0, 40), ([0, 40, 2000000000], 0, 40), ([-2**31, 0, 40], 0, 40), ([40, 90], 40, 90)):
        dst = torch.full_like(out, 7.0)
        s2.prompt_attention(q, k, v, ints(wrong), out=dst)
        assert torch.equal(dst[first:last], out[first:last]), wrong
        dst[first:last] = 7.0
        assert (dst == 7.0).all(), wrong
    assert torch.equal(s2.prompt_attention(q, k, v, off), out)
