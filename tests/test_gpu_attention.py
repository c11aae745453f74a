"""Tree and prompt attention against the fp64 oracle.

Tolerances.  fp32: a score of D products carries about sqrt(D) 2^-24 of the
score's size, the same relative error in each weight, and sums of thousands of
weights little more: 1e-5 of the row.  bf16: the output's rounding is at most
2^-8 of an element and 1.7e-3 in the 2-norm, and so is that of the weights, whose
errors are independent (2.4e-3 together): 4e-3 over all rows, and 1e-2 for a
single row of 64 elements."""

import numpy as np
import pytest

from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL_ALL = {"f32": 1e-5, "bf16": 4e-3}
TOL_ROW = {"f32": 3e-5, "bf16": 1e-2}


def check(got, ref, dtype, label=""):
    """got [n, H, D] on the device against ref; rows that are zero have to be zero."""
    g = got.double().cpu().numpy()
    assert np.isfinite(g).all(), label
    norm = np.linalg.norm(ref)
    if norm:
        err = np.linalg.norm(g - ref) / norm
        assert err <= TOL_ALL[dtype], f"{label}: {err:.3e}"
    rows = np.linalg.norm(ref, axis=-1)
    off = np.linalg.norm(g - ref, axis=-1)
    bad = off > TOL_ROW[dtype] * rows
    assert not bad.any(), f"{label}: rows {np.argwhere(bad)[:4].tolist()} off by {(off / np.maximum(rows, 1e-30)).max():.3e}"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def fill(cache, lengths, rooms, g, poison=False):
    """Pages for rooms[s] slots of each sequence, scattered over the pool, all slots random (or, where no token lies, NaN)."""
    P = cache.page_size
    order = torch.randperm(cache.n_pages, generator=torch.Generator().manual_seed(7)).tolist()
    cache.k.normal_(generator=g)
    cache.v.normal_(generator=g)
    table = torch.full((cache.max_seqs, cache.max_pages), -1, dtype=torch.int32)
    at = 0
    used = torch.zeros((cache.n_pages, P), dtype=torch.bool)
    for s, room in enumerate(rooms):
        for j in range(-(-room // P)):
            table[s, j] = order[at]
            used[order[at], :max(0, min(P, room - j * P))] = True
            at += 1
    cache.table.copy_(table)
    cache.length.copy_(torch.tensor(list(lengths) + [0] * (cache.max_seqs - len(lengths)), dtype=torch.int32))
    cache.refs.zero_()
    cache.refs[torch.tensor(order[:at], dtype=torch.long, device="cuda")] = 1
    if poison:
        bad = (~used).cuda()
        cache.k[:, bad.nonzero()[:, 0], :, bad.nonzero()[:, 1]] = float("nan")
        p, x = bad.nonzero()[:, 0], bad.nonzero()[:, 1]
        cache.v[:, p, :, x // 8, :, x % 8] = float("inf")


def random_parents(counts, seed, chain=0.6):
    r = np.random.default_rng(seed)
    out = []
    for n in counts:
        out += [i - 1 if r.random() < chain else int(r.integers(-1, i)) if i else -1 for i in range(n)]
    return out


def tree_reference(cache, layer, q, lengths, counts, parents, scale):
    """Oracle output of every sequence, packed."""
    k = cache.k[layer].double().cpu().numpy()[None]
    v = cache.v[layer].double().cpu().numpy()[None]
    oc = ao.Cache(k, v, cache.table.cpu().numpy(), cache.length.cpu().numpy(), cache.refs.cpu().numpy())
    out, at = [], 0
    for s, (n, t) in enumerate(zip(lengths, counts)):
        if t == 0:
            continue
        kk, vv = oc.tokens(0, s, n + t)
        out.append(ao.tree_attention(q[at:at + t].double().cpu().numpy(), kk, vv, n, parents[at:at + t], scale))
        at += t
    return np.concatenate(out)


def run_tree(dtype, heads, P, lengths, counts, parents=None, poison=False, layers=1, layer=0, scale=None, seed=0, max_nodes=None, qscale=1.0):
    Hq, Hkv, D = heads
    g = torch.Generator(device="cuda").manual_seed(seed)
    rooms = [a + b for a, b in zip(lengths, counts)]
    pages = sum(-(-r // P) for r in rooms) + 2
    cache = s2.KVCache(layers, Hkv, D, pages, P, len(lengths) + 1, max(-(-r // P) for r in rooms) + 1, dtype=DT[dtype])
    fill(cache, lengths, rooms, g, poison)
    off = np.concatenate([[0], np.cumsum(counts)]).tolist()
    parents = random_parents(counts, seed) if parents is None else parents
    q = torch.randn((off[-1], Hq, D), generator=g, device="cuda").mul_(qscale).to(DT[dtype])
    att = s2.TreeAttention(cache, Hq, len(lengths), max_nodes or max(max(counts), 1), scale)
    args = (layer, q, ints(list(range(len(lengths)))), ints(off), ints(parents))
    out = att(*args)
    ref = tree_reference(cache, layer, q, lengths, counts, parents, scale or D ** -0.5)
    check(out, ref, dtype, f"{dtype} {heads} P {P}")
    return cache, att, args, out, ref


HEADS = [(4, 2, 64), (32, 8, 128), (8, 8, 128), (16, 1, 64), (10, 2, 64), (3, 1, 128)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("P", [16, 64])
def test_tree_heads_and_pages(dtype, heads, P):
    run_tree(dtype, heads, P, [37, 0, 130, 63], [5, 3, 16, 1], seed=heads[0] + P)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("D", [64, 128])
def test_tree_lengths_at_the_edges(dtype, P, D):
    """Contexts and trees that end at, before and after pages and tiles; one token; nothing cached."""
    edges = [0, 1, 7, 8, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513]
    run_tree(dtype, (4, 2, D), P, edges, [1 + (3 * i) % 5 for i in range(len(edges))], seed=P + D, poison=True)
    run_tree(dtype, (8, 2, D), P, edges, [1] * len(edges), seed=P + D + 1, poison=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 128, 200, 256])
def test_tree_sizes(dtype, T):
    run_tree(dtype, (8, 4, 64), 32, [70, 3], [T, max(1, T // 3)], seed=T, poison=True)
    run_tree(dtype, (8, 1, 128), 16, [9], [T], seed=T + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ["chain", "star", "pairs"])
def test_tree_shapes(dtype, shape):
    T = 100
    par = {"chain": list(range(-1, T - 1)), "star": [-1] * T, "pairs": [(i - 1) // 2 if i else -1 for i in range(T)]}[shape]
    run_tree(dtype, (4, 2, 64), 32, [41], [T], par, poison=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_long_context_few_rows(dtype):
    run_tree(dtype, (8, 2, 128), 64, [9001], [1], seed=1)
    run_tree(dtype, (8, 2, 64), 16, [6007, 1, 800], [3, 1, 2], seed=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_ragged_batch(dtype):
    r = np.random.default_rng(3)
    n = 70
    run_tree(dtype, (8, 2, 64), 32, r.integers(0, 400, n).tolist(), r.integers(0, 9, n).tolist(), seed=4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_many_sequences(dtype):
    r = np.random.default_rng(5)
    run_tree(dtype, (2, 1, 64), 16, r.integers(0, 40, 1024).tolist(), [1] * 1024, seed=6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_rows_that_see_nothing(dtype):
    """Nodes below an invalid parent get zeros, whatever the others get."""
    par = [-1, 0, 2, 2, 7, 1, -2, 6, 3, 5]
    _, _, _, out, ref = run_tree(dtype, (4, 2, 64), 16, [20], [10], par)
    dead = [2, 3, 4, 6, 7, 8]
    assert not ref[dead].any() and not out[dead].any().item()
    _, _, _, out, _ = run_tree(dtype, (4, 2, 64), 16, [0], [3], [5, 0, 1])
    assert not out.any().item()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_what_masked_nodes_hold_does_not_matter(dtype):
    """Infinities and NaN in the slots of nodes that a row does not see."""
    lengths, counts = [45], [40]
    par = random_parents(counts, 9)
    cache, att, args, out, ref = run_tree(dtype, (8, 2, 64), 16, lengths, counts, par, seed=9)
    seen, _ = ao.tree_visible(par)
    node = max(range(5, 40), key=lambda j: int(seen[:, j].sum()) if seen[:, j].sum() < 20 else 0)
    at = int(cache.table[0, (45 + node) // 16]), (45 + node) % 16
    for kk, vv in ((float("nan"), float("nan")), (float("inf"), float("-inf")), (3e38, 3e38)):
        cache.k[0, at[0], :, at[1]] = kk
        cache.v[0, at[0], :, at[1] // 8, :, at[1] % 8] = vv
        got = att(*args)
        blind = ~torch.tensor(seen[:, node], device="cuda")
        assert torch.equal(got[blind], out[blind]), "a masked node changed a row"
        if kk != kk:
            assert torch.isnan(got[~blind]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_large_scores(dtype):
    """Scores of hundreds: the running maximum moves by far more than exp can take."""
    run_tree(dtype, (8, 2, 64), 32, [300, 40], [6, 17], seed=11, qscale=40.0 if dtype == "bf16" else 8.0, scale=0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tree_strides_layers_and_slices(dtype):
    """q a slice of a wider array, out another, id arrays at odd addresses, a middle layer."""
    Hq, Hkv, D = 6, 2, 64
    cache, att, args, out, _ = run_tree(dtype, (Hq, Hkv, D), 16, [50, 20], [7, 4], layers=3, layer=1)
    _, q, seqs, off, par = args
    wide = torch.full((11, Hq + 5, D), float("nan"), dtype=DT[dtype], device="cuda")
    wide[:, 2:2 + Hq] = q
    shift = lambda x: torch.cat([ints([99]), x])[1:]  # noqa: E731
    dst = torch.zeros((11, 2 * Hq, D), dtype=DT[dtype], device="cuda")
    att(1, wide[:, 2:2 + Hq], shift(seqs), shift(off), shift(par), out=dst[:, Hq:])
    assert torch.equal(dst[:, Hq:], out) and not dst[:, :Hq].any()
    # Sequences by any id, in any order.
    r = att(1, torch.cat([q[7:], q[:7]]), ints([1, 0]), ints([0, 4, 11]), torch.cat([par[7:], par[:7]]))
    assert torch.equal(torch.cat([r[4:], r[:4]]), out) or dtype == "bf16"
    check(torch.cat([r[4:], r[:4]]), out.double().cpu().numpy(), dtype)


def test_tree_same_bits_every_time_and_on_another_stream():
    cache, att, args, out, _ = run_tree("bf16", (32, 8, 128), 64, [1500, 30, 700], [16, 1, 9])
    for _ in range(5):
        assert torch.equal(att(*args), out)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = att(*args)
    s.synchronize()
    assert torch.equal(again, out)
    other = att(*args, stream=s)
    s.synchronize()
    assert torch.equal(other, out)


def test_tree_workspace_contents_do_not_matter():
    cache, att, args, out, _ = run_tree("bf16", (32, 4, 128), 64, [5000, 3], [4, 1])
    att.workspace.fill_(255)
    assert torch.equal(att(*args), out)


def test_tree_smaller_trees_than_announced_and_empty_ones():
    run_tree("bf16", (8, 2, 64), 16, [50, 20, 7, 0], [3, 0, 2, 0], max_nodes=200)


def test_tree_zero_tokens():
    cache = s2.KVCache(1, 1, 64, 4, 16, 2, 2)
    att = s2.TreeAttention(cache, 2, 2, 4)
    assert att(0, torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda"), ints([0]), ints([0, 0]), ints([])).shape == (0, 2, 64)


def test_tree_offsets_past_32_bits():
    """Pages beyond 2^31 elements of the pool."""
    Hkv, D, P = 8, 128, 256
    pages = (1 << 31) // (Hkv * D * P) + 40
    cache = s2.KVCache(1, Hkv, D, pages, P, 1, 8)
    g = torch.Generator(device="cuda").manual_seed(0)
    ids = [pages - 1, pages - 7, 3, pages - 30]
    for p in ids:
        cache.k[0, p].normal_(generator=g)
        cache.v[0, p].normal_(generator=g)
    cache.table[0, :4] = ints(ids)
    cache.length[0] = 1000
    q = torch.randn((2, 16, D), generator=g, device="cuda").to(torch.bfloat16)
    out = s2.TreeAttention(cache, 16, 1, 2)(0, q, ints([0]), ints([0, 2]), ints([-1, -1]))
    sub = torch.tensor(ids, device="cuda")
    k = cache.k[0, sub].permute(0, 2, 1, 3).reshape(-1, Hkv, D)[:1002].double().cpu().numpy()
    v = cache.v[0, sub].permute(0, 2, 4, 1, 3).reshape(-1, Hkv, D)[:1002].double().cpu().numpy()
    check(out, ao.tree_attention(q.double().cpu().numpy(), k, v, 1000, [-1, -1], D ** -0.5), "bf16")


def test_tree_in_a_graph():
    """Captured once, replayed while lengths, tables and inputs change under it."""
    cache, att, args, out, _ = run_tree("bf16", (8, 2, 128), 32, [400, 90], [5, 3])
    layer, q, seqs, off, par = args
    dst = torch.empty_like(out)
    att(*args, out=dst)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        att(*args, out=dst)
    for n in ([400, 90], [17, 0], [1, 60], [333, 89]):
        cache.length[:2] = ints(n)
        q.normal_()
        dst.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dst, att(*args))
        check(dst, tree_reference(cache, 0, q, n, [5, 3], par.tolist(), 128 ** -0.5), "bf16")


# -------------------------------------------------------------------- prompts


def run_prompt(dtype, heads, lens, seed=0, wide=True, scale=None, qscale=1.0, first=0):
    Hq, Hkv, D = heads
    g = torch.Generator(device="cuda").manual_seed(seed)
    off = (first + np.concatenate([[0], np.cumsum(lens)])).tolist()
    n = off[-1]
    if wide:
        x = torch.randn((n, Hq + 2 * Hkv, D), generator=g, device="cuda")
        x[:, :Hq] *= qscale
        x = x.to(DT[dtype])
        q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    else:
        q, k, v = (torch.randn((n, h, D), generator=g, device="cuda").to(DT[dtype]) for h in (Hq, Hkv, Hkv))
    out = s2.prompt_attention(q, k, v, ints(off), scale=scale)
    ref = ao.prompt_attention(*(t.double().cpu().numpy() for t in (q, k, v)), off, scale or D ** -0.5)
    check(out[first:], ref[first:], dtype, f"{dtype} {heads} {lens[:4]}")
    return q, k, v, ints(off), out


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", HEADS)
def test_prompt_heads(dtype, heads):
    run_prompt(dtype, heads, [70, 1, 0, 33, 140], seed=heads[0])
    run_prompt(dtype, heads, [5], seed=heads[0], wide=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_prompt_lengths_at_the_edges(dtype, D):
    run_prompt(dtype, (4, 2, D), [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 0], seed=D)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 1, 128), (2, 2, 64)])
def test_prompt_long(dtype, heads):
    run_prompt(dtype, heads, [1531], seed=1)
    run_prompt(dtype, heads, [1, 1024, 511], seed=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_many(dtype):
    r = np.random.default_rng(8)
    run_prompt(dtype, (2, 1, 64), r.integers(0, 9, 1024).tolist(), seed=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_large_scores(dtype):
    run_prompt(dtype, (8, 2, 64), [300, 40], seed=11, qscale=40.0 if dtype == "bf16" else 8.0, scale=0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_rising_scores(dtype):
    """Each key outweighs all before it: the maximum moves at every step."""
    D, n = 64, 400
    k = torch.zeros((n, 1, D), device="cuda")
    k[:, 0, 0] = torch.arange(n, device="cuda") // 2
    g = torch.Generator(device="cuda").manual_seed(3)
    v = torch.randn((n, 1, D), generator=g, device="cuda").to(DT[dtype])
    q = torch.ones((n, 2, D), device="cuda").to(DT[dtype])
    k = k.to(DT[dtype])
    out = s2.prompt_attention(q, k, v, ints([0, n]), scale=3.0)
    check(out, ao.prompt_attention(*(t.double().cpu().numpy() for t in (q, k, v)), [0, n], 3.0), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("at", [0, 40, 95, 130])
def test_prompt_later_tokens_do_not_matter(dtype, at):
    """Infinities and NaN in k and v of a token leave every earlier row, and every other prompt, as it was."""
    q, k, v, off, out = run_prompt(dtype, (4, 2, 64), [60, 131, 30], wide=False)
    for kk, vv in ((float("nan"), float("nan")), (float("inf"), float("-inf"))):
        k2, v2 = k.clone(), v.clone()
        k2[60 + at], v2[60 + at] = kk, vv
        got = s2.prompt_attention(q, k2, v2, off)
        assert torch.equal(got[:60 + at], out[:60 + at]) and torch.equal(got[191:], out[191:])
        if kk != kk:
            assert torch.isnan(got[60 + at:191]).all()


def test_prompt_rows_outside_the_offsets_are_left_alone():
    q, k, v, off, out = run_prompt("bf16", (4, 2, 64), [40, 50], wide=False)
    dst = torch.full_like(out, 7.0)
    s2.prompt_attention(q, k, v, ints([11, 40, 75]), out=dst)
    assert (dst[:11] == 7.0).all() and (dst[75:] == 7.0).all()
    ref = ao.prompt_attention(*(t.double().cpu().numpy() for t in (q, k, v)), [11, 40, 75], 64 ** -0.5)
    check(dst[11:75], ref[11:75], "bf16")


def test_prompt_same_bits_every_time_and_in_a_graph():
    q, k, v, off, out = run_prompt("bf16", (8, 2, 128), [300, 1, 77], wide=False)
    dst = torch.empty_like(out)
    s2.prompt_attention(q, k, v, off, out=dst)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s2.prompt_attention(q, k, v, off, out=dst)
    for _ in range(4):
        q.normal_()
        dst.zero_()
        graph.replay()
        assert torch.equal(dst, s2.prompt_attention(q, k, v, off))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = s2.prompt_attention(q, k, v, off, out=torch.empty_like(out), stream=s)
    s.synchronize()
    assert torch.equal(got, dst)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_offsets_past_32_bits(dtype):
    """Rows beyond 2^31 elements (bf16) and bytes (fp32) of the arrays they are slices of."""
    n, D = 70000, 64
    ld = (1 << 31) // n + 200
    ld -= ld % 64
    if dtype == "f32":
        ld //= 2
        ld -= ld % 64
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.empty((n, ld // D, D), dtype=DT[dtype], device="cuda")
    x[-90:, :6].normal_(generator=g)
    q, k, v = x[:, :4], x[:, 4:5], x[:, 5:6]
    out = torch.zeros((n, 4, D), dtype=DT[dtype], device="cuda")
    s2.prompt_attention(q, k, v, ints([n - 90, n - 80, n]), out=out)
    ref = ao.prompt_attention(*(t[-90:].double().cpu().numpy() for t in (q, k, v)), [0, 10, 90], D ** -0.5)
    check(out[-90:], ref, dtype)
    assert not out[:-90].any()


# Many heads and long prompts: 64 rows a wave in bf16, in fp32 the keys split over the waves.
WIDE = [(64, 32, 128), (64, 32, 64)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads", WIDE)
def test_prompt_many_rows(dtype, heads):
    run_prompt(dtype, heads, [1187, 1290], seed=21)


@pytest.mark.parametrize("heads", WIDE)
def test_prompt_many_rows_large_scores(heads):
    run_prompt("bf16", heads, [1187, 1290], seed=22, qscale=40.0, scale=0.5)


@pytest.mark.parametrize("heads", WIDE)
def test_prompt_many_rows_rising_scores(heads):
    Hq, Hkv, D = heads
    n = 1201
    g = torch.Generator(device="cuda").manual_seed(23)
    k = torch.zeros((2 * n, Hkv, D), device="cuda")
    k[:, :, 0] = (torch.arange(2 * n, device="cuda") % n // 8)[:, None]
    q = torch.ones((2 * n, Hq, D), device="cuda").bfloat16()
    k, v = k.bfloat16(), torch.randn((2 * n, Hkv, D), generator=g, device="cuda").bfloat16()
    out = s2.prompt_attention(q, k, v, ints([0, n, 2 * n]), scale=3.0)
    check(out, ao.prompt_attention(*(t.double().cpu().numpy() for t in (q, k, v)), [0, n, 2 * n], 3.0), "bf16")


@pytest.mark.parametrize("heads", WIDE)
@pytest.mark.parametrize("at", [0, 700, 1180])
def test_prompt_many_rows_later_tokens_do_not_matter(heads, at):
    Hq, Hkv, D = heads
    g = torch.Generator(device="cuda").manual_seed(24)
    q, k, v = (torch.randn((2477, h, D), generator=g, device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
    off = ints([0, 1187, 2477])
    out = s2.prompt_attention(q, k, v, off)
    k[at], v[at] = float("nan"), float("nan")
    got = s2.prompt_attention(q, k, v, off)
    assert torch.equal(got[:at], out[:at]) and torch.equal(got[1187:], out[1187:])
    assert torch.isnan(got[at:1187]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_prompt_f32_many_short(D):
    """Short prompts, but many rows: a wave takes rows of its own."""
    r = np.random.default_rng(25)
    run_prompt("f32", (32, 8, D), [0, 1, 255] + r.integers(0, 130, 40).tolist(), seed=25)
