"""Page operations and appends against the host model of the cache: whole
numbers equal, pools equal bit for bit."""

import numpy as np
import pytest

from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pair:
    """The cache on the device and its model on the host, driven alike."""

    def __init__(self, dtype="bf16", layers=2, Hkv=2, D=64, pages=40, P=16, seqs=12, maxp=6, seed=0):
        self.dev = s2.KVCache(layers, Hkv, D, pages, P, seqs, maxp, dtype=DT[dtype])
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dev.k.normal_(generator=g)
        self.dev.v.normal_(generator=g)
        self.g, self.dtype = g, DT[dtype]
        self.host = ao.Cache(*(self.np(t) for t in (self.dev.k, self.dev.v, self.dev.table, self.dev.length, self.dev.refs)))

    def np(self, t):
        t = t.cpu()
        return (t.view(torch.int16) if t.dtype == torch.bfloat16 else t.view(torch.int32) if t.dtype == torch.float32 else t).numpy()

    def same(self, status, n, label):
        got = self.dev.status[:n].tolist()
        assert got == list(status), f"{label}: status {got}, {status} wanted"
        for name in ("table", "length", "refs", "k", "v"):
            a, b = self.np(getattr(self.dev, name)), getattr(self.host, name)
            assert np.array_equal(a, b), f"{label}: {name} differs at {np.argwhere(a != b)[:3].tolist()}"
        # Every reference is some sequence's, and a row's pages lie together.
        t = self.host.table
        assert np.array_equal(np.bincount(t[t >= 0], minlength=len(self.host.refs)), self.host.refs), label
        assert not ((t[:, 1:] >= 0) & (t[:, :-1] < 0)).any(), label

    def fork(self, src, dst):
        self.dev.fork(ints(src), ints(dst))
        st = self.host.fork(src, dst)
        self.same(st, len(src), f"fork {src} {dst}")
        return st

    def reserve(self, seqs, extra):
        self.dev.reserve(ints(seqs), ints(extra))
        st, copied = self.host.reserve(seqs, extra)
        self.same(st, len(seqs), f"reserve {seqs} {extra}")
        assert self.dev.copied[:len(seqs)].tolist() == copied.tolist()
        return st

    def append(self, layer, seqs, counts, wide=False):
        off = np.concatenate([[0], np.cumsum(counts)]).astype(int).tolist()
        Hkv, D = self.dev.n_kv_heads, self.dev.head_dim
        x = torch.randn((off[-1], 3 * Hkv, D), generator=self.g, device="cuda").to(self.dtype)
        k, v = (x[:, Hkv:2 * Hkv], x[:, 2 * Hkv:]) if wide else (x[:, :Hkv].contiguous(), x[:, Hkv:2 * Hkv].contiguous())
        self.dev.append(layer, k, v, ints(seqs), ints(off))
        self.host.append(layer, self.np(k.contiguous()), self.np(v.contiguous()), seqs, off)
        self.same(self.dev.status[:0].tolist(), 0, f"append {seqs} {counts}")

    def commit(self, seqs, path, acc):
        p = None
        if path is not None:
            most = max([len(x) for x in path] + [0])
            p = ints([list(x) + [-7] * (most - len(x)) for x in path]).view(len(path), most)
        self.dev.commit(ints(seqs), p, ints(acc))
        st = self.host.commit(seqs, None if path is None else p.tolist(), acc)
        self.same(st, len(seqs), f"commit {seqs} {path} {acc}")
        return st

    def free(self, seqs):
        self.dev.free(ints(seqs))
        st = self.host.free(seqs)
        self.same(st, len(seqs), f"free {seqs}")
        return st


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P,D,Hkv", [(16, 64, 2), (32, 128, 1), (64, 64, 3), (256, 128, 2)])
def test_a_branched_decoding(dtype, P, D, Hkv):
    c = Pair(dtype, P=P, D=D, Hkv=Hkv, maxp=4)
    assert c.reserve([0, 3], [P + 5, 2 * P]) == [0, 0]
    for layer in (0, 1):
        c.append(layer, [0, 3], [P + 5, 2 * P], wide=layer == 1)
    assert c.commit([0, 3], None, [P + 5, 2 * P]) == [0, 0]
    assert c.fork([0, 0, 3], [1, 2, 4]) == [0, 0, 0]
    assert c.reserve([0, 1, 2, 3, 4], [9, 3, 8, 4, 1]) == [0] * 5
    c.append(1, [1, 0, 4], [3, 9, 1])
    assert c.commit([0, 1, 2, 4], [[0, 2, 3, 8], [1], [], [0]], [4, 1, 0, 1]) == [0] * 4
    assert c.reserve([2], [2]) == [0]  # the last holder of the shared page writes in place
    assert c.free([3, 0]) == [0, 0]
    assert c.free([3, 1, 2, 4]) == [0] * 4
    assert not c.dev.refs.any() and (c.dev.table == -1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seed", range(4))
def test_random_programs(dtype, seed):
    r = np.random.default_rng(seed)
    S, maxp, P = 10, 5, [16, 32, 64, 16][seed]
    c = Pair(dtype, P=P, pages=[30, 18, 24, 50][seed], seqs=S, maxp=maxp, seed=seed)
    for step in range(60):
        n = int(r.integers(1, 6))
        seqs = r.integers(-1, S + 1, n).tolist() if r.random() < 0.2 else r.permutation(S)[:n].tolist()
        op = r.integers(0, 5)
        if op == 0:
            c.reserve(seqs, r.integers(0, 2 * P, n).tolist())
        elif op == 1:
            c.fork(r.integers(0, S, n).tolist(), seqs)
        elif op == 2:
            seqs = r.permutation(S)[:n].tolist()
            counts = r.integers(0, 20, n).tolist()
            if r.random() < 0.7:
                c.reserve(seqs, counts)
            c.append(int(r.integers(0, 2)), seqs, counts, wide=bool(r.integers(0, 2)))
        elif op == 3:
            path = [sorted(r.permutation(20)[:int(r.integers(0, 7))].tolist()) for _ in range(n)]
            c.commit(seqs, path if r.random() < 0.8 else None, [len(p) for p in path])
        else:
            c.free(seqs[:2])


def test_grants_end_with_the_pages():
    c = Pair(pages=10, maxp=6)
    assert c.reserve([0, 1, 2, 3, 4], [16 * 4, 16 * 5, 16 * 2, 0, 16]) == [0, 0, ao.NO_PAGES, 0, ao.NO_PAGES]
    assert c.reserve([2], [16]) == [0]
    assert c.reserve([2], [17]) == [ao.NO_PAGES]
    assert c.free([1]) == [0]
    assert c.reserve([2, 5], [40, 33]) == [0, 0]


def test_a_copy_that_finds_no_page_changes_nothing():
    c = Pair(pages=2)
    c.reserve([0], [20])
    c.commit([0], None, [20])
    c.fork([0], [1])
    assert c.reserve([1, 0], [1, 1]) == [ao.NO_PAGES, 0]
    assert c.reserve([1], [1]) == [ao.NO_PAGES]


def test_refusals_on_the_device():
    c = Pair(maxp=3)
    assert c.reserve([0, 0, -1, 12, 1, 2], [5, 5, 5, 5, -1, 49]) == [0, 4, 4, 4, 2, 2]
    c.commit([0], None, [5])
    assert c.fork([0, 0, 0, 1, 5, -1, 99], [1, 1, 0, 3, 12, 6, 7]) == [4, 4, 4, 4, 4, 4, 4]
    assert c.fork([0, 0, 7], [1, 2, 3]) == [0, 0, 0]
    assert c.fork([0], [1]) == [ao.BUSY]
    c.reserve([5], [3])
    assert c.fork([0], [5]) == [ao.BUSY]  # reserved pages count
    c.reserve([0], [20])
    bad = [[1, 1], [2, 1], [-1, 0], [0, 43]]
    for p in bad:
        assert c.commit([0], [p], [2]) == [ao.BAD_PATH], p
    assert c.commit([0], [[0, 1]], [3]) == [ao.BAD_PATH]
    assert c.commit([0], [[0, 1]], [-1]) == [ao.BAD_PATH]
    assert c.commit([0], None, [44]) == [ao.BAD_PATH]
    assert c.commit([0, 0, 33], [[0], [1], [0]], [1, 1, 1]) == [0, 4, 4]
    assert c.free([0, 0, 44]) == [0, 4, 4]


def test_longest_paths_and_no_requests():
    c = Pair(pages=40, P=16, maxp=20)
    c.reserve([0], [270])
    c.append(0, [0], [270])
    c.commit([0], None, [11])
    c.reserve([0], [256])
    r = np.random.default_rng(0)
    path = sorted(r.permutation(256)[:200].tolist())
    assert c.commit([0], [path], [200]) == [0]
    c.reserve([0], [100])
    assert c.commit([0], [list(range(100))], [100]) == [0]
    e = ints([])
    c.dev.fork(e, e), c.dev.reserve(e, e), c.dev.free(e), c.dev.commit(e, None, e)
    c.dev.append(0, torch.empty((0, 2, 64), dtype=c.dtype, device="cuda"), torch.empty((0, 2, 64), dtype=c.dtype, device="cuda"), ints([0]),
                 ints([0, 0]))
    c.same([], 0, "no requests")


def test_many_requests_and_a_large_pool():
    """1024 requests in one call over more pages than one sweep of the grants covers."""
    n = 1024
    c = Pair(layers=1, Hkv=1, pages=50000, P=16, seqs=2 * n, maxp=64)
    r = np.random.default_rng(1)
    first = r.integers(0, 700, n).tolist()
    seqs = r.permutation(n).tolist()
    assert not any(c.reserve(seqs, first))
    assert not any(c.commit(seqs, None, first))
    assert not any(c.free(seqs[::3]))
    keep = [s for i, s in enumerate(seqs) if i % 3]
    assert not any(c.fork(keep, [n + s for s in keep]))
    both = [n + s for s in keep[:500]] + keep[:500]
    assert not any(c.reserve(both, r.integers(0, 100, 1000).tolist()))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_appends_of_every_length_and_place(dtype):
    """Whole and broken groups of eight slots, across pages, from every starting slot."""
    c = Pair(dtype, pages=200, P=16, seqs=40, maxp=8)
    starts = list(range(0, 34))
    c.reserve(list(range(34)), [s + 60 for s in starts])
    c.commit(list(range(34)), None, starts)
    c.reserve(list(range(34)), [60] * 34)
    c.append(0, list(range(34)), [(7 * s) % 61 for s in starts])
    c.append(1, list(range(33, -1, -1)), [1] * 34, wide=True)
    c.append(1, [0, 1], [100, 200])  # past the reserved pages: dropped


def test_append_to_unknown_sequences_is_dropped():
    c = Pair()
    c.reserve([3], [30])
    k = torch.randn((12, 2, 64), device="cuda").to(c.dtype)
    c.dev.append(0, k, k, ints([-1, 50, 3]), ints([0, 4, 8, 12]))
    c.host.append(0, c.np(k)[8:], c.np(k)[8:], [3], [0, 4])
    c.same([], 0, "append")


def test_pools_past_32_bits():
    """Copies, moves and writes in pages and layers beyond 2^31 elements."""
    Hkv, D, P = 8, 128, 256
    pages = (1 << 31) // (Hkv * D * P) + 4
    c = s2.KVCache(2, Hkv, D, pages, P, 3, 2)
    c.refs[:pages - 4] = 1  # only the last pages are free
    c.reserve(ints([0]), ints([300]))
    assert c.table[0].tolist() == [pages - 4, pages - 3]
    x = torch.randn((300, 2 * Hkv, D), device="cuda").to(torch.bfloat16)
    c.append(1, x[:, :Hkv], x[:, Hkv:], ints([0]), ints([0, 300]))
    c.commit(ints([0]), None, ints([290]))
    c.fork(ints([0]), ints([1]))
    c.reserve(ints([1]), ints([10]))
    assert c.table[1].tolist() == [pages - 4, pages - 2] and c.copied[0].tolist() == [pages - 3, pages - 2]
    c.append(1, x[290:, :Hkv], x[290:, Hkv:], ints([1]), ints([0, 10]))
    c.commit(ints([1]), ints([[3, 7]]), ints([2]))
    want = torch.cat([x[:290], x[293:294], x[297:298]])
    for page, lo, hi in ((pages - 4, 0, 256), (pages - 2, 256, 292)):
        assert torch.equal(c.k[1, page, :, :hi - lo].transpose(0, 1), want[lo:hi, :Hkv])
        v = c.v[1, page].permute(1, 3, 0, 2).reshape(P, Hkv, D)
        assert torch.equal(v[:hi - lo], want[lo:hi, Hkv:])


def test_a_step_in_a_graph():
    """free, fork, reserve, append and commit captured once and replayed."""
    c = Pair(pages=60)
    c.reserve([0, 1], [37, 64])
    c.commit([0, 1], None, [37, 64])
    src, dst, room = ints([0, 0, 1]), ints([4, 5, 6]), ints([8, 8, 8])
    path, acc = ints([[0, 2, 5], [1, 3, 0], [4, 0, 0]]), ints([3, 2, 1])
    off = ints([0, 8, 16, 24])
    k = torch.empty((24, 2, 64), dtype=c.dtype, device="cuda")
    v = torch.empty_like(k)

    def step():
        c.dev.free(dst)
        c.dev.fork(src, dst)
        c.dev.reserve(dst, room)
        c.dev.append(1, k, v, dst, off)
        c.dev.commit(dst, path, acc)

    k.normal_(), v.normal_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        k.normal_(), v.normal_()
        graph.replay()
        c.host.free([4, 5, 6])
        c.host.fork([0, 0, 1], [4, 5, 6])
        c.host.reserve([4, 5, 6], room.tolist())
        c.host.append(1, c.np(k), c.np(v), [4, 5, 6], [0, 8, 16, 24])
        c.same(c.host.commit([4, 5, 6], path.tolist(), [3, 2, 1]), 3, f"replay {i}")
        if i == 1:
            room.fill_(20)
