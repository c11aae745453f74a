"""Cache and attention calls on a stream other than the current one."""

import pytest

from oracle import attention_oracle as ao
from tests.test_gpu_attention import check, ints, run_tree

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402

SLEEP = 100_000_000  # clock ticks: tens of milliseconds


def handles(s):
    """The ways to name a stream."""
    return s, s.cuda_stream


@pytest.mark.parametrize("way", [0, 1])
def test_a_result_does_not_take_memory_that_the_current_stream_still_uses(way):
    g = torch.Generator(device="cuda").manual_seed(1)
    n, Hq, Hkv, D = 500, 8, 2, 128
    q, k, v = (torch.randn((n, h, D), generator=g, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
    off = ints([0, n])
    want = s2.prompt_attention(q, k, v, off)
    ref = ao.prompt_attention(*(t.double().cpu().numpy() for t in (q, k, v)), [0, n], D ** -0.5)
    s, other = torch.cuda.Stream(), q.flip(0).contiguous()
    torch.cuda.synchronize()
    for _ in range(3):
        a = torch.full_like(want, 7.0)
        torch.cuda._sleep(SLEEP)
        b = a.clone()
        del a  # its block is free for the current stream's next allocation, after the copy
        out = s2.prompt_attention(q, k, v, off, stream=handles(s)[way])
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda._sleep(SLEEP)
        c = out.clone()
        del out  # and this one must not go back to the other stream before the copy
        s2.prompt_attention(other, k, v, off, stream=handles(s)[way])
        torch.cuda.synchronize()
        assert (b == 7.0).all() and torch.equal(c, want)
    check(want, ref, "bf16")


@pytest.mark.parametrize("way", [0, 1])
def test_tree_results_on_another_stream(way):
    cache, att, args, want, _ = run_tree("bf16", (32, 8, 128), 64, [1500, 30, 700], [16, 1, 9])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        a = torch.full_like(want, 7.0)
        torch.cuda._sleep(SLEEP)
        b = a.clone()
        del a
        out = att(*args, stream=handles(s)[way])
        torch.cuda.current_stream().wait_stream(s)
        c = out.clone()
        torch.cuda.synchronize()
        assert (b == 7.0).all() and torch.equal(c, want)


def test_the_default_stream_by_its_handle():
    cache, att, args, want, _ = run_tree("bf16", (8, 2, 64), 16, [50], [4])
    assert torch.equal(att(*args, stream=0), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = att(*args, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_calls_on_two_streams_at_once():
    """One object, its calls interleaved on two streams: each keeps its parts in a workspace of its own."""
    cache, att, args, want, _ = run_tree("bf16", (32, 8, 128), 64, [9000, 4000], [16, 9])
    layer, q, seqs, off, par = args
    swapped = (layer, torch.cat([q[16:], q[:16]]), ints([1, 0]), ints([0, 9, 25]), torch.cat([par[16:], par[:16]]))
    first = att(*swapped)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    out = [(torch.empty_like(want), torch.empty_like(first)) for _ in range(30)]
    for x, y in out:
        att(*args, out=x, stream=a)
        att(*swapped, out=y, stream=b)
    torch.cuda.synchronize()
    for x, y in out:
        assert torch.equal(x, want) and torch.equal(y, first)


def test_a_replay_beside_eager_calls():
    cache, att, args, want, _ = run_tree("bf16", (32, 8, 128), 64, [9000, 4000], [16, 9])
    layer, q, seqs, off, par = args
    swapped = (layer, torch.cat([q[16:], q[:16]]), ints([1, 0]), ints([0, 9, 25]), torch.cat([par[16:], par[:16]]))
    first = att(*swapped)
    dst, s = torch.empty_like(want), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        att(*args, out=dst)
    for _ in range(20):
        dst.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graph.replay()
        got = [att(*swapped) for _ in range(3)]
        torch.cuda.synchronize()
        assert torch.equal(dst, want) and all(torch.equal(g, first) for g in got)
    with torch.cuda.stream(s):
        again = att(*args)
    torch.cuda.synchronize()
    assert torch.equal(again, want)
