"""Positions and the append with rotation against 64 bits and against the plain append.

How far off a turned element may be: the turn is rounded once to fp32 below 1 (2 pi 2^-25
of an angle), sine and cosine by 2^-22, three fp32 operations, and the product of position
and frequency in 64 bits; then one rounding to the type."""

import numpy as np
import pytest

from oracle import dense_oracle as do

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def np64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def freqs(rot, theta=1e4):
    return (theta ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)).float().cuda()


def check_turned(got, x, pos, freq, neighbours, dtype, label=""):
    f = freq.cpu().numpy()
    want, size = do.rotate(np64(x), pos, f, neighbours)
    angle = np.abs(np.asarray(pos, dtype=np.float64)).max() * np.abs(f).max()
    slack = 2 * np.pi * 2.0 ** -25 + 2.0 ** -22 + 4 * 2.0 ** -24 + angle * 2.0 ** -51
    rot = 2 * len(f)
    off = np.abs(np64(got) - want)[..., :rot] - size[..., :rot] * slack - np.abs(want)[..., :rot] * HALF[dtype]
    assert off.max() <= 0, (label, np.unravel_index(off.argmax(), off.shape), off.max())
    assert torch.equal(got[..., rot:], x[..., rot:]), label


def make(dtype, Hkv, D, P, lengths, room, seed=0, extra_pages=3, maxp=None):
    """A cache whose sequences hold `lengths` tokens and have pages for `room`, all slots filled."""
    need = [-(-r // P) for r in room]
    c = s2.KVCache(2, Hkv, D, sum(need) + extra_pages, P, len(lengths), maxp or max(max(need), 1), dtype=DT[dtype])
    g = torch.Generator(device="cuda").manual_seed(seed)
    c.k.normal_(generator=g)
    c.v.normal_(generator=g)
    order, at = torch.randperm(sum(need), generator=g, device="cuda").to(torch.int32), 0
    for i, n in enumerate(need):
        c.table[i, :n] = order[at:at + n]
        at += n
    c.refs[:sum(need)] = 1
    c.length.copy_(ints(lengths))
    return c, g


def twin(c):
    t = s2.KVCache(c.n_layers, c.n_kv_heads, c.head_dim, c.n_pages, c.page_size, c.max_seqs, c.max_pages, dtype=c.dtype,
                   **{n: getattr(c, n).clone() for n in ("k", "v", "table", "length", "refs")})
    return t


def offsets(counts):
    return np.concatenate([[0], np.cumsum(counts)]).astype(int).tolist()


# --------------------------------------------------------------------------- positions


@pytest.mark.parametrize("counts", [[1], [5, 0, 3], [700, 1, 255, 256, 257], [4000]])
def test_positions_of_prompts(counts):
    lengths = [(17 * i) % 50 for i in range(len(counts))]
    c, _ = make("bf16", 1, 64, 16, lengths, [n + 1 for n in lengths])
    off = offsets(counts)
    got = c.positions(ints(list(range(len(counts)))), ints(off), off[-1])
    assert got.dtype == torch.int32 and got.tolist() == do.positions(lengths, counts).tolist()


def draw_parents(n, r, chain=0.6):
    return [-1 if i == 0 else (i - 1 if r.random() < chain else int(r.integers(-1, i))) for i in range(n)]


@pytest.mark.parametrize("counts", [[1], [8], [16, 0, 1, 64], [255, 256, 257, 3], [1000, 700]])
@pytest.mark.parametrize("chain", [0.0, 0.6, 1.0])
def test_positions_of_trees(counts, chain):
    r = np.random.default_rng(len(counts))
    lengths = [5 + 3 * i for i in range(len(counts))]
    c, _ = make("bf16", 1, 64, 16, lengths, [n + 1 for n in lengths])
    parent = sum([draw_parents(n, r, chain) for n in counts], [])
    off = offsets(counts)
    got = c.positions(ints(list(range(len(counts)))), ints(off), off[-1], ints(parent))
    assert got.tolist() == do.positions(lengths, counts, parent).tolist()


def test_positions_with_bad_parents_ids_and_rows_outside():
    c, _ = make("bf16", 1, 64, 16, [10, 20], [11, 21])
    parent = [-1, 0, 5, 2, -7, 4, 6, 2 ** 31 - 1]
    out = torch.full((12,), -99, dtype=torch.int32, device="cuda")
    got = c.positions(ints([1, 7]), ints([2, 10, 10]), 12, ints([0, 0] + parent + [0, 0]), out=out)
    assert got is out
    assert out.tolist() == [-99, -99] + do.positions([20], [8], parent).tolist() + [-99, -99]
    assert c.positions(ints([9]), ints([0, 3]), 3).tolist() == [0, 1, 2]
    assert c.positions(ints([]), ints([0]), 0).shape == (0,)


# ------------------------------------------------------------------------- the rotation


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,rot", [(64, 64), (64, 16), (64, 48), (128, 128), (128, 64), (128, 112)])
@pytest.mark.parametrize("neighbours", [False, True])
def test_against_the_plain_append(dtype, D, rot, neighbours):
    """The cache holds what the plain append makes of the turned keys, bit for bit; queries and
    keys are turned; whole groups of eight and parts of them, pages that end inside."""
    Hkv, Hq, P = 2, 6, 16
    for lengths, counts in (([13, 0, 7], [29, 8, 1]), ([3, 40, 0, 9, 15, 16], [1, 1, 3, 1, 0, 2]), ([0], [1])):
        c, g = make(dtype, Hkv, D, P, lengths, [a + b for a, b in zip(lengths, counts)])
        t = twin(c)
        off = offsets(counts)
        n = off[-1]
        qkv = torch.randn((n, Hq + 2 * Hkv, D), generator=g, device="cuda").to(DT[dtype])
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        seqs, to, f = ints(list(range(len(counts)))), ints(off), freqs(rot)
        pos = c.positions(seqs, to, n)
        k_out = torch.empty((n, Hkv, D), dtype=DT[dtype], device="cuda")
        q_out = c.append_rotated(1, q, k, v, seqs, to, pos, f, neighbours, k_out=k_out)
        check_turned(q_out, q, pos.tolist(), f, neighbours, dtype, "q")
        check_turned(k_out, k, pos.tolist(), f, neighbours, dtype, "k")
        t.append(1, k_out, v, seqs, to)
        for name in ("k", "v", "table", "length", "refs"):
            assert torch.equal(getattr(c, name), getattr(t, name)), (lengths, name)
        # In place gives the same bits.
        u = twin(t)
        own = qkv.clone()
        got = u.append_rotated(1, own[:, :Hq], own[:, Hq:Hq + Hkv], own[:, Hq + Hkv:], seqs, to, pos, f, neighbours,
                               out=own[:, :Hq], k_out=own[:, Hq:Hq + Hkv])
        assert torch.equal(own[:, :Hq], q_out) and torch.equal(own[:, Hq:Hq + Hkv], k_out) and torch.equal(own[:, Hq + Hkv:], v)
        assert got.data_ptr() == own.data_ptr() and torch.equal(u.k, c.k) and torch.equal(u.v, c.v)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 7), (32, 8), (64, 8), (33, 11)])
@pytest.mark.parametrize("D", [64, 128])
def test_head_counts(Hq, Hkv, D):
    for counts in ([1] * 5, [37, 12]):
        lengths = [11 * i for i in range(len(counts))]
        c, g = make("bf16", Hkv, D, 32, lengths, [a + b for a, b in zip(lengths, counts)])
        t = twin(c)
        off = offsets(counts)
        q, k, v = (torch.randn((off[-1], h, D), generator=g, device="cuda").to(torch.bfloat16) for h in (Hq, Hkv, Hkv))
        seqs, to, f = ints(list(range(len(counts)))), ints(off), freqs(D)
        pos = c.positions(seqs, to, off[-1])
        k_out = torch.empty_like(k)
        check_turned(c.append_rotated(0, q, k, v, seqs, to, pos, f, k_out=k_out), q, pos.tolist(), f, False, "bf16")
        check_turned(k_out, k, pos.tolist(), f, False, "bf16")
        t.append(0, k_out, v, seqs, to)
        assert torch.equal(c.k, t.k) and torch.equal(c.v, t.v)
        again = twin(t)
        again.append_rotated(0, q, k, v, seqs, to, pos, f)  # without k_out
        assert torch.equal(again.k, c.k) and torch.equal(again.v, c.v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions(dtype):
    c, g = make(dtype, 1, 64, 16, [0], [16])
    pos = [0, 1, -1, 1000, 131071, 10 ** 6, 16777217, 2 ** 31 - 1, -2 ** 31, 123456789]
    n = len(pos)
    q, k, v = (torch.randn((n, 1, 64), generator=g, device="cuda").to(DT[dtype]) for _ in range(3))
    for f in (freqs(64), freqs(64, 1e6) * 3.7):
        k_out = torch.empty_like(k)
        got = c.append_rotated(0, q, k, v, ints([0]), ints([0, n]), ints(pos), f, k_out=k_out)
        for i, p in enumerate(pos):  # one at a time, as the bound grows with the angle
            check_turned(got[i:i + 1], q[i:i + 1], [p], f, False, dtype, p)
            check_turned(k_out[i:i + 1], k[i:i + 1], [p], f, False, dtype, p)
        assert torch.equal(got[0], q[0])


def test_tokens_without_a_page_and_rows_outside():
    """No page, a shared page, an unknown sequence: keys are turned but not kept; rows outside
    the requests stay as they were."""
    c, g = make("bf16", 2, 64, 16, [14, 5, 0], [16, 16, 0], extra_pages=2)
    c.refs[c.table[1, 0].long()] = 2
    before = c.k.clone(), c.v.clone()
    n = 14
    q, k, v = (torch.randn((n, 2, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    seqs, off = ints([0, 1, 2, 77]), ints([1, 5, 8, 10, 12])
    out, k_out = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    pos = ints(list(range(100, 100 + n)))
    c.append_rotated(0, q, k, v, seqs, off, pos, freqs(64), out=out, k_out=k_out)
    check_turned(out[1:12], q[1:12], range(101, 112), freqs(64), False, "bf16")
    check_turned(k_out[1:12], k[1:12], range(101, 112), freqs(64), False, "bf16")
    for t in (out, k_out):
        assert (t[:1] == 7).all() and (t[12:] == 7).all()
    page = int(c.table[0, 0])
    assert torch.equal(c.k[0, page, :, 14:16].transpose(0, 1), k_out[1:3])  # the two slots that are left
    before[0][0, page, :, 14:16] = c.k[0, page, :, 14:16]
    before[1][0, page, :, 1, :, 6:] = c.v[0, page, :, 1, :, 6:]
    assert torch.equal(c.k, before[0]) and torch.equal(c.v, before[1])


def test_offsets_that_make_no_sense_stay_inside():
    c, g = make("bf16", 1, 64, 16, [3, 9], [16, 16])
    q, k, v = (torch.randn((20, 1, 64), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    for off in ([0, 500, 20], [-5, 7, 2 ** 31 - 1], [9, 3, 1], [-2 ** 31, -3, -1], [30, 40, 50]):
        pos = c.positions(ints([0, 1]), ints(off), 20)
        c.append_rotated(0, q, k, v, ints([0, 1]), ints(off), ints([5] * 20), freqs(64), k_out=torch.empty_like(k))
        assert pos.shape == (20,)
    torch.cuda.synchronize()


def test_streams_and_graphs():
    c, g = make("bf16", 2, 128, 32, [10, 33], [60, 90])
    q, k, v = (torch.randn((20, h, 128), generator=g, device="cuda").to(torch.bfloat16) for h in (4, 2, 2))
    seqs, off, f = ints([0, 1]), ints([0, 9, 20]), freqs(128)
    parent = ints(draw_parents(9, np.random.default_rng(0)) + draw_parents(11, np.random.default_rng(1)))

    def step(cache, stream=None):
        pos = cache.positions(seqs, off, 20, parent, stream=stream)
        return pos, cache.append_rotated(0, q, k, v, seqs, off, pos, f, stream=stream)

    want = step(c)
    side, other = torch.cuda.Stream(), twin(c)
    other.k.zero_()
    other.v.zero_()
    side.wait_stream(torch.cuda.current_stream())
    got = step(other, side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(other)
    for i in range(4):
        for t in (q, k, v):
            t.normal_(generator=g)
        c.length.add_(1)
        other.length.copy_(c.length)
        want = step(c)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        for s in (0, 1):
            n = int(c.length[s])
            for j in range(n, n + (9, 11)[s]):
                p = int(c.table[s, j // 32])
                assert torch.equal(c.k[0, p, :, j % 32], other.k[0, p, :, j % 32])
                assert torch.equal(c.v[0, p, :, j % 32 // 8, :, j % 8], other.v[0, p, :, j % 32 // 8, :, j % 8])


def test_rows_and_pages_past_four_gigabytes():
    """The last tokens of many, and pages at the end of a long cache, as the same tokens alone
    in a short one."""
    n, tail, Hq, Hkv, D, P = 300000, 5, 64, 1, 128, 256
    long, short = (s2.KVCache(2, 8, D, pages, P, 1, 2) for pages in (5200, 2))
    for c in (long, short):
        c.table[0, :2] = ints([c.n_pages - 1, c.n_pages - 2])
        c.refs[-2:] = 1
        c.length.fill_(P - 2)
        c.k.zero_()
        c.v.zero_()
    f, g = freqs(D), torch.Generator(device="cuda").manual_seed(3)
    pos = ints([7, 100, 3, 2000, 65])
    q, k, v = (torch.randn((tail, h, D), generator=g, device="cuda").to(torch.bfloat16) for h in (16, 8, 8))
    want = short.append_rotated(1, q, k, v, ints([0]), ints([0, tail]), pos, f)
    assert torch.equal(long.append_rotated(1, q, k, v, ints([0]), ints([0, tail]), pos, f), want)
    for t in ("k", "v"):
        assert torch.equal(getattr(long, t)[1, -2:], getattr(short, t)[1, -2:]) and getattr(long, t)[1, -2:].any()
        assert not getattr(long, t)[0].any() and not getattr(long, t)[1, :-2].any()
    del long
    c = s2.KVCache(1, Hkv, D, 2, P, 1, 2)
    q = torch.zeros((n, Hq, D), dtype=torch.bfloat16, device="cuda")
    k = torch.zeros((n, Hkv, D), dtype=torch.bfloat16, device="cuda")
    q[-tail:].normal_(generator=g)
    pos_all = torch.zeros(n, dtype=torch.int32, device="cuda")
    pos_all[-tail:] = pos
    args = k[-tail:].clone(), k[-tail:].clone(), ints([0]), ints([0, tail]), pos, f
    want = c.append_rotated(0, q[-tail:].clone(), *args)
    got = c.append_rotated(0, q, k, k.clone(), ints([0]), ints([0, n]), pos_all, f)
    assert torch.equal(got[-tail:], want) and not got[:1000].any()
