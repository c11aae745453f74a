"""The append with rotation for many tokens at once, which writes the cache in groups of eight
slots (from 1200 tokens on; from 4096 on a wave has two kv heads): the cache against the plain
append, bit for bit, keys and queries against 64 bits, and in place."""

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402
from tests.test_gpu_rotate import DT, check_turned, freqs, ints, make, offsets, twin  # noqa: E402

ARRAYS = ("k", "v", "table", "length", "refs")
# Requests that begin at the end, in the middle and at the beginning of a group and of a page;
# long ones, one token, a few, and none, beside each other.
SOME = ([3, 0, 13, 15, 7, 8, 1, 0, 31], [1, 0, 700, 1, 513, 1, 3, 0, 40])
MANY = ([5, 16, 3, 0, 15, 9, 255], [2049, 1, 0, 1500, 2, 777, 9])


def compare(dtype, Hq, Hkv, D, P, rot, neighbours, lengths, counts, seed=0):
    c, g = make(dtype, Hkv, D, P, lengths, [a + b for a, b in zip(lengths, counts)], seed)
    plain, own = twin(c), twin(c)
    n = sum(counts)
    qkv = torch.randn((n, Hq + 2 * Hkv, D), generator=g, device="cuda").to(DT[dtype])
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    seqs, off, f = ints(list(range(len(counts)))), ints(offsets(counts)), freqs(rot)
    pos = c.positions(seqs, off, n)
    given = qkv.clone()
    k_out = torch.empty((n, Hkv, D), dtype=DT[dtype], device="cuda")
    q_out = c.append_rotated(1, q, k, v, seqs, off, pos, f, neighbours, k_out=k_out)
    assert torch.equal(qkv, given)
    check_turned(q_out, q, pos.tolist(), f, neighbours, dtype, "q")
    check_turned(k_out, k, pos.tolist(), f, neighbours, dtype, "k")
    plain.append(1, k_out, v, seqs, off)
    for name in ARRAYS:
        assert torch.equal(getattr(c, name), getattr(plain, name)), name
    # In place, and without the keys kept: the same bits.
    own.append_rotated(1, given[:, :Hq], given[:, Hq:Hq + Hkv], given[:, Hq + Hkv:], seqs, off, pos, f, neighbours, out=given[:, :Hq],
                       k_out=given[:, Hq:Hq + Hkv])
    assert torch.equal(given[:, :Hq], q_out) and torch.equal(given[:, Hq:Hq + Hkv], k_out) and torch.equal(given[:, Hq + Hkv:], v)
    assert torch.equal(own.k, c.k) and torch.equal(own.v, c.v)
    own.k.zero_()
    own.v.zero_()
    assert torch.equal(own.append_rotated(1, q, k, v, seqs, off, pos, f, neighbours), q_out)
    plain.k.zero_()
    plain.v.zero_()
    plain.append(1, k_out, v, seqs, off)
    assert torch.equal(own.k, plain.k) and torch.equal(own.v, plain.v)


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 48), (128, 128), (128, 16)])
@pytest.mark.parametrize("requests", [SOME, MANY], ids=["some", "many"])
def test_against_the_plain_append(requests, D, rot, dtype, neighbours):
    compare(dtype, 4, 3, D, 16, rot, neighbours, *requests)


@pytest.mark.parametrize("P", [32, 256])
@pytest.mark.parametrize("Hkv", [1, 2, 5, 8])
@pytest.mark.parametrize("requests", [SOME, MANY], ids=["some", "many"])
def test_kv_heads_and_pages(requests, Hkv, P):
    compare("bf16", Hkv, Hkv, 64, P, 64, False, *requests, seed=Hkv)


# A wave's loads of queries go round more than once.
@pytest.mark.parametrize("dtype,D,Hq", [("f32", 128, 64), ("f32", 128, 33), ("f32", 64, 70), ("bf16", 128, 72), ("bf16", 64, 130), ("bf16", 128, 1)])
def test_query_heads(dtype, D, Hq):
    compare(dtype, Hq, 1, D, 16, D, False, *SOME)


@pytest.mark.parametrize("n", [1199, 1200, 4095, 4096])
def test_either_side_of_the_rules(n):
    compare("bf16", 8, 3, 64, 64, 64, False, [7, 2], [n - 5, 5])


def test_tokens_without_a_page_and_rows_outside():
    """No page from some slot on, a shared page, an unknown sequence: keys are turned but not kept;
    rows outside the requests stay as they were."""
    D, P, Hkv = 64, 16, 3
    lengths, room, counts = [5, 3, 0, 9], [600, 700, 0, 40], [900, 640, 300, 20, 100]
    c, g = make("bf16", Hkv, D, P, lengths, room, maxp=60)
    c.refs[c.table[1, 10].long()] = 2
    c.refs[c.table[1, 11].long()] = 0
    plain = twin(c)
    seqs, off = ints([0, 1, 2, 3, 99]), ints([3 + x for x in offsets(counts)])
    n = sum(counts) + 7
    q, k, v = (torch.randn((n, h, D), generator=g, device="cuda").to(torch.bfloat16) for h in (4, Hkv, Hkv))
    pos = ints(list(range(1000, 1000 + n)))
    out, k_out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    c.append_rotated(0, q, k, v, seqs, off, pos, freqs(D), out=out, k_out=k_out)
    inside = slice(3, n - 4)
    check_turned(out[inside], q[inside], pos[inside].tolist(), freqs(D), False, "bf16")
    check_turned(k_out[inside], k[inside], pos[inside].tolist(), freqs(D), False, "bf16")
    for t in (out, k_out):
        assert (t[:3] == 7).all() and (t[n - 4:] == 7).all()
    plain.append(0, k_out, v, seqs, off)
    for name in ARRAYS:
        assert torch.equal(getattr(c, name), getattr(plain, name)), name


def test_offsets_that_make_no_sense_stay_inside():
    c, g = make("bf16", 1, 64, 16, [3, 9], [16, 16])
    n = 1300
    q, k, v = (torch.randn((n, 1, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    refs = c.refs.clone()
    for off in ([0, 5000, n], [-5, 7, 2 ** 31 - 1], [900, 3, 1], [-2 ** 31, -3, -1], [2000, 2001, 2002], [0, n, 0]):
        c.append_rotated(0, q, k, v, ints([0, 1]), ints(off), ints([5] * n), freqs(64), k_out=torch.empty_like(k))
    torch.cuda.synchronize()
    assert torch.equal(c.refs, refs)


def test_rows_past_four_gigabytes():
    """One prompt whose rows pass 2^32 bytes: its cache against the plain append, its last keys
    and queries against the same tokens alone."""
    n, tail, Hq, Hkv, D, P = 600000, 5, 16, 8, 128, 256
    g = torch.Generator(device="cuda").manual_seed(4)
    qkv = torch.empty((n, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    pages = -(-(n + 3) // P)
    c = s2.KVCache(1, Hkv, D, pages, P, 1, pages)
    c.table[0] = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    c.refs.fill_(1)
    c.length.fill_(3)
    c.k.zero_()
    c.v.zero_()
    plain = twin(c)
    seqs, off, f = ints([0]), ints([0, n]), freqs(D)
    pos = c.positions(seqs, off, n)
    k_out = torch.empty((n, Hkv, D), dtype=torch.bfloat16, device="cuda")
    q_out = c.append_rotated(0, q, k, v, seqs, off, pos, f, k_out=k_out)
    plain.append(0, k_out, v, seqs, off)
    assert torch.equal(c.k, plain.k) and torch.equal(c.v, plain.v)
    few = s2.KVCache(1, Hkv, D, 2, P, 1, 2)
    few.refs.fill_(1)
    few.table[0] = ints([0, 1])
    kept = torch.empty((tail, Hkv, D), dtype=torch.bfloat16, device="cuda")
    for at in (0, n // 2, n - tail):
        part = slice(at, at + tail)
        turned = few.append_rotated(0, q[part], k[part], v[part], seqs, ints([0, tail]), pos[part].clone(), f, k_out=kept)
        assert torch.equal(q_out[part], turned) and torch.equal(k_out[part], kept)
        check_turned(kept, k[part], pos[part].tolist(), f, False, "bf16")


def test_a_captured_prompt():
    c, g = make("bf16", 3, 64, 16, SOME[0], [a + b + 4 for a, b in zip(*SOME)])
    n = sum(SOME[1])
    q, k, v = (torch.randn((n, h, 64), generator=g, device="cuda").to(torch.bfloat16) for h in (4, 3, 3))
    seqs, off, f, other = ints(list(range(9))), ints(offsets(SOME[1])), freqs(64), twin(c)

    def step(cache):
        pos = cache.positions(seqs, off, n)
        return pos, cache.append_rotated(0, q, k, v, seqs, off, pos, f)

    step(other)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(other)
    for i in range(3):
        for t in (q, k, v):
            t.normal_(generator=g)
        c.length.add_(1)
        for name in ARRAYS:
            getattr(other, name).copy_(getattr(c, name))
        want = step(c)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(c.k, other.k) and torch.equal(c.v, other.v), i

