"""Performance cases of the cache and attention operators of a speculative-decoding program.

Four kinds of call:
  tree    attention of drafted tokens over the cache (`TreeAttention`): each sequence's draft tree
          attends to its cached tokens and, within the tree, to its ancestors.  One node is plain decoding.
  prompt  causal attention over whole prompts, packed one after another (`prompt_attention`).
  append  the keys and values of new tokens written into a layer's pages (`KVCache.append`).
  pages   a step of branched decoding: the branches of the last step are freed, new ones forked from
          their parents, given room for drafted tokens (which copies the pages they share and would
          write to), and their accepted paths made contiguous, over all layers.

`own` chooses between the framework's calls and a plain form of elementary operations in 32 bits.

The cache: K [layer, page, kv head, slot, D], V [layer, page, kv head, slot / 8, D, slot % 8],
table [sequence, page of the sequence] (-1: none), length [sequence], refs [page].
"""

import math
import random

import torch

own = False

DEVICE = "cuda" if torch.cuda.is_available() else "cpu"

# (query heads, kv heads, head size) of the model shapes the repository's workloads are named after; "tiny" goes with
# the fp32 layer of hidden size 256.
HEADS = {
    "tiny": (4, 2, 64),
    "mixtral": (32, 8, 128),
    "qwen3": (32, 4, 128),
    "olmoe": (16, 16, 128),
    "gptoss": (64, 8, 64),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# --------------------------------------------------------------------- cases


def listed():
    return [
        # The fp32 parity layer's attention: one short sequence, a tree of 8 nodes.  Latency alone counts.
        dict(name="tree f32 tiny 8 nodes", kind="tree", heads="tiny", dtype="f32", seqs=1, ctx_lo=200, ctx_hi=200, nodes_lo=8,
             nodes_hi=8, page=16, mix=1),
        # Decoding one token of one conversation: the smallest call of a serving program.
        dict(name="tree decode 1 token", kind="tree", heads="mixtral", dtype="bf16", seqs=1, ctx_lo=2047, ctx_hi=2047, nodes_lo=1,
             nodes_hi=1, page=64, mix=2),
        # The verify batch of the Mixtral-shaped workload: 16 drafted tokens of one conversation.
        dict(name="tree verify 16 nodes", kind="tree", heads="mixtral", dtype="bf16", seqs=1, ctx_lo=4093, ctx_hi=4093, nodes_lo=16,
             nodes_hi=16, page=64, mix=3),
        # A serving batch of verifications: 64 conversations of very different lengths, 1 to 9 nodes each.
        dict(name="tree batch 64 ragged", kind="tree", heads="qwen3", dtype="bf16", seqs=64, ctx_lo=300, ctx_hi=6000, nodes_lo=1,
             nodes_hi=9, page=32, mix=4),
        # One long document with a large tree: the long axis has to be split.
        dict(name="tree long 64 nodes", kind="tree", heads="gptoss", dtype="bf16", seqs=1, ctx_lo=65537, ctx_hi=65537, nodes_lo=64,
             nodes_hi=64, page=128, mix=5),
        # fp32 prompts of a few words.
        dict(name="prompt f32 tiny", kind="prompt", heads="tiny", dtype="f32", seqs=3, len_lo=1, len_hi=150, mix=6),
        # A batch of short chat prompts.
        dict(name="prompt 24 ragged", kind="prompt", heads="gptoss", dtype="bf16", seqs=24, len_lo=1, len_hi=1024, mix=7),
        # One long document: bound by the matrix cores.
        dict(name="prompt 12289", kind="prompt", heads="qwen3", dtype="bf16", seqs=1, len_lo=12289, len_hi=12289, mix=8),
        # The new token of every conversation of a decoding batch.
        dict(name="append 48 tokens", kind="append", heads="mixtral", dtype="bf16", seqs=48, ctx_lo=100, ctx_hi=2000, new_lo=1,
             new_hi=1, page=16, mix=9),
        # The prompts of several conversations entering the cache.
        dict(name="append prompts", kind="append", heads="mixtral", dtype="bf16", seqs=5, ctx_lo=0, ctx_hi=70, new_lo=1000,
             new_hi=5000, page=64, mix=10),
        # Two conversations with two branches each, fp32.
        dict(name="pages f32 tiny", kind="pages", heads="tiny", dtype="f32", layers=2, parents=2, branches=2, ctx_lo=20, ctx_hi=90,
             nodes_lo=4, nodes_hi=8, page=16, mix=11),
        # Sixteen conversations with four branches each over all layers of the 24-layer workload.
        dict(name="pages 64 branches", kind="pages", heads="mixtral", dtype="bf16", layers=24, parents=16, branches=4, ctx_lo=100,
             ctx_hi=600, nodes_lo=4, nodes_hi=16, page=64, mix=12),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("tree", "tree", "prompt", "prompt", "append", "pages"))
    c = dict(kind=kind, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")), mix=rng.randrange(1 << 20))
    c["heads"] = rng.choice([h for h in HEADS if h != "tiny"]) if c["dtype"] == "bf16" else rng.choice(("tiny", "mixtral", "gptoss"))
    page = rng.choice((16, 32, 64, 128))
    if kind == "tree":
        ctx = _log_int(rng, 1, 32768)
        seqs = _log_int(rng, 1, max(1, min(64, 131072 // ctx)))
        nodes = _log_int(rng, 1, 64 if seqs <= 8 else 16)
        c.update(seqs=seqs, ctx_lo=_log_int(rng, max(1, ctx // 8), ctx), ctx_hi=ctx, nodes_lo=_log_int(rng, 1, nodes), nodes_hi=nodes, page=page)
    elif kind == "prompt":
        n = _log_int(rng, 1, 8192 if c["dtype"] == "bf16" else 2048)
        c.update(seqs=_log_int(rng, 1, max(1, min(32, 12000 // n))), len_lo=_log_int(rng, max(1, n // 8), n), len_hi=n)
    elif kind == "append":
        n = _log_int(rng, 1, 4096)
        c.update(seqs=_log_int(rng, 1, max(1, min(64, 16384 // n))), ctx_lo=0, ctx_hi=rng.randrange(0, 500), new_lo=_log_int(rng, max(1, n // 4), n),
                 new_hi=n, page=page)
    else:
        ctx = _log_int(rng, 16, 600)
        nodes = _log_int(rng, 2, 16)
        c.update(layers=rng.randint(1, 16), parents=rng.randint(1, 12), branches=rng.randint(1, 4), ctx_lo=_log_int(rng, max(1, ctx // 4), ctx), ctx_hi=ctx,
                 nodes_lo=_log_int(rng, 1, nodes), nodes_hi=nodes, page=page)
    return c


def _ragged(case, n, lo, hi, key):
    """n whole numbers of the case's own between lo and hi; the first is hi."""
    rng = random.Random(case["mix"] * 1009 + key)
    return [hi] + [rng.randint(lo, hi) for _ in range(n - 1)]


def _offsets(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


# ------------------------------------------------------------------- prepare


def _gen(*key):
    g = torch.Generator(device=DEVICE)
    s = 0
    for k in key:
        s = (s * 1000003 + int(k) + 12345) % (1 << 62)
    g.manual_seed(s)
    return g


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEVICE)


def _randn(shape, dtype, g, std=1.0):
    x = torch.randn(shape, generator=g, device=DEVICE, dtype=dtype)
    return x.mul_(std) if std != 1.0 else x


def _cache(layers, heads, dtype, page, lengths, rows, max_pages, spare, g):
    """A cache in use: the first len(lengths) sequences hold that many tokens, with pages for what `rows` says, scattered
    over the pool; every slot, used or not, holds something."""
    _, kvh, D = HEADS[heads]
    need = [-(-r // page) for r in rows]
    total = sum(need) + spare
    order = torch.randperm(total, generator=g, device=DEVICE).to(torch.int32)
    table = torch.full((len(lengths), max_pages), -1, dtype=torch.int32, device=DEVICE)
    refs = torch.zeros(total, dtype=torch.int32, device=DEVICE)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    refs[order[:at].long()] = 1
    return {"k": _randn((layers, total, kvh, page, D), dtype, g), "v": _randn((layers, total, kvh, page // 8, D, 8), dtype, g),
            "table": table, "length": _ints(lengths), "refs": refs}


def _parents(counts, g):
    """Draft trees, one after another: a node hangs below the one before it, or below an earlier one or the last verified token (-1)."""
    at = torch.cat([torch.arange(n, device=DEVICE) for n in counts])
    u = torch.rand((2, at.numel()), generator=g, device=DEVICE)
    return torch.where(u[0] < 0.6, at - 1, (u[1] * (at + 1)).long().clamp(max=at.numel()) - 1).clamp(min=-1).minimum(at - 1).to(torch.int32)


def _handle(cache):
    """The framework's view of these tensors, which a program keeps."""
    import paper_2608_15018_amd as s2

    L, n_pages, kvh, P, D = cache["k"].shape
    S, maxp = cache["table"].shape
    return s2.KVCache(L, kvh, D, n_pages, P, S, maxp, dtype=cache["k"].dtype, **cache)


def prepare(case, seed):
    dt = DTYPES[case["dtype"]]
    qh, kvh, D = HEADS[case["heads"]]
    g = _gen(seed, case["mix"])
    st = {"kind": case["kind"]}
    if case["kind"] == "prompt":
        lens = _ragged(case, case["seqs"], case["len_lo"], case["len_hi"], 1)
        n = sum(lens)
        qkv = _randn((n, qh + 2 * kvh, D), dt, g)  # one projection's output, as a layer has it
        st.update(q=qkv[:, :qh], k=qkv[:, qh:qh + kvh], v=qkv[:, qh + kvh:], off=_ints(_offsets(lens)), most=max(lens))
        return st
    if case["kind"] == "pages":
        n, b, P = case["parents"], case["branches"], case["page"]
        ctx = _ragged(case, n, case["ctx_lo"], case["ctx_hi"], 1)
        nodes = _ragged(case, n * b, case["nodes_lo"], case["nodes_hi"], 2)
        maxp = -(-(case["ctx_hi"] + case["nodes_hi"]) // P) + 1
        c = _cache(case["layers"], case["heads"], dt, P, ctx + [0] * (n * b), ctx + [0] * (n * b), maxp, n * b * (2 + case["nodes_hi"] // P), g)
        # The accepted path of a branch: ascending nodes, each kept with probability 0.7.
        keep = torch.rand((n * b, case["nodes_hi"]), generator=g, device=DEVICE) < 0.7
        at = torch.arange(case["nodes_hi"], device=DEVICE)
        keep &= at < _ints(nodes)[:, None]
        path = torch.where(keep, at, 1 << 20).sort(dim=1).values
        path = torch.where(path < (1 << 20), path, -1).to(torch.int32)
        src = torch.arange(n, device=DEVICE).repeat_interleave(b).to(torch.int32)
        dst = torch.arange(n, n + n * b, device=DEVICE).to(torch.int32)
        st.update(cache=c, src=src, dst=dst, nodes=_ints(nodes), path=path, accepted=keep.sum(1).to(torch.int32))
        st["handle"] = _handle(c) if own else None
        return st
    n, P = case["seqs"], case["page"]
    ctx = _ragged(case, n, case["ctx_lo"], case["ctx_hi"], 1)
    new = _ragged(case, n, case["nodes_lo"], case["nodes_hi"], 2) if case["kind"] == "tree" else _ragged(case, n, case["new_lo"], case["new_hi"], 2)
    room = [a + b for a, b in zip(ctx, new)]
    c = _cache(1, case["heads"], dt, P, ctx, room, -(-max(room) // P), 3, g)
    st.update(cache=c, seqs=torch.arange(n, device=DEVICE).to(torch.int32), off=_ints(_offsets(new)), most=max(new))
    if case["kind"] == "append":
        kv = _randn((sum(new), 2 * kvh, D), dt, g)
        st.update(k=kv[:, :kvh], v=kv[:, kvh:])
    else:
        st.update(q=_randn((sum(new), qh, D), dt, g), parent=_parents(new, g))
    if own:
        st["handle"] = _handle(c)
        if case["kind"] == "tree":
            import paper_2608_15018_amd as s2

            st["attention"] = s2.TreeAttention(st["handle"], qh, n, st["most"])
    return st


# ----------------------------------------------------------------------- run


def run(state):
    if own:
        return _run_own(state)
    return {"tree": _plain_tree, "prompt": _plain_prompt, "append": _plain_append, "pages": _plain_pages}[state["kind"]](state)


def _state_of(c):
    return {n: c[n] for n in ("k", "v", "table", "length", "refs")}


def _run_own(st):
    import paper_2608_15018_amd as s2

    if st["kind"] == "tree":
        return st["attention"](0, st["q"], st["seqs"], st["off"], st["parent"])
    if st["kind"] == "prompt":
        return s2.prompt_attention(st["q"], st["k"], st["v"], st["off"])
    h = st["handle"]
    if st["kind"] == "append":
        h.append(0, st["k"], st["v"], st["seqs"], st["off"])
        return {"k": st["cache"]["k"], "v": st["cache"]["v"]}
    h.free(st["dst"])
    h.fork(st["src"], st["dst"])
    h.reserve(st["dst"], st["nodes"])
    h.commit(st["dst"], st["path"], st["accepted"])
    return _state_of(st["cache"])


def _padded(x, off, most):
    """Packed rows [n, ...] as [sequences, most, ...] in 32 bits, zero past each end, and which rows are real."""
    at = torch.arange(most, device=x.device)
    first, count = off[:-1].long(), (off[1:] - off[:-1]).long()
    real = at < count[:, None]
    rows = torch.where(real, first[:, None] + at, 0)
    return torch.where(real[(...,) + (None,) * (x.dim() - 1)], x[rows].float(), 0.0), real


def _softmax(s):
    """Softmax over the last axis, in place; a row of -inf alone gives zeros."""
    top = s.amax(-1, keepdim=True)
    s.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = s.sum(-1, keepdim=True)
    return s.div_(torch.where(total == 0, 1.0, total))


def _plain_prompt(st):
    q, real = _padded(st["q"], st["off"], st["most"])
    k, v = _padded(st["k"], st["off"], st["most"])[0], _padded(st["v"], st["off"], st["most"])[0]
    n, m, qh, D = q.shape
    kvh = k.shape[2]
    q = q.reshape(n, m, kvh, qh // kvh, D).permute(0, 2, 3, 1, 4).reshape(n, kvh, -1, D).contiguous()
    k, v = k.permute(0, 2, 3, 1).contiguous(), v.permute(0, 2, 1, 3).contiguous()
    s = torch.matmul(q, k).mul_(D ** -0.5).view(n, kvh, qh // kvh, m, m)
    at = torch.arange(m, device=q.device)
    s.masked_fill_(at[None, :] > at[:, None], -math.inf)
    o = torch.matmul(_softmax(s).view(n, kvh, -1, m), v).view(n, qh, m, D).permute(0, 2, 1, 3)
    return o[real].to(st["q"].dtype)


def _plain_tree(st):
    c = st["cache"]
    _, _, kvh, P, D = c["k"].shape
    q, real = _padded(st["q"], st["off"], st["most"])
    par = _padded(st["parent"], st["off"], st["most"])[0].long()
    n, T, qh, _ = q.shape
    dev = q.device
    length = c["length"][st["seqs"].long()].long()
    pages = c["table"][st["seqs"].long()].long().clamp(min=0)
    m = pages.shape[1] * P
    k = c["k"][0][pages].float().permute(0, 2, 4, 1, 3).reshape(n, kvh, D, m).contiguous()
    v = c["v"][0][pages].float().permute(0, 2, 1, 3, 5, 4).reshape(n, kvh, m, D).contiguous()
    at = torch.arange(m, device=dev)
    node = torch.arange(T, device=dev)
    # above[i, j]: node j is node i or an ancestor of it.  Squaring the relation doubles the steps it covers.
    above = (node[:, None] == node[None, :]) | (par[..., None] == node)
    above = above.float()
    for _ in range(max(1, (T - 1).bit_length())):
        above = torch.matmul(above, above).clamp_(max=1.0)
    live = at < (length + (st["off"][1:] - st["off"][:-1]))[:, None]
    slot = (at - length[:, None]).clamp(0, T - 1)
    seen = torch.where((at < length[:, None])[:, None], True, above.gather(2, slot[:, None].expand(n, T, m)) > 0) & live[:, None]
    q = q.reshape(n, T, kvh, qh // kvh, D).permute(0, 2, 1, 3, 4).reshape(n, kvh, -1, D).contiguous()
    s = torch.matmul(q, k).mul_(D ** -0.5).view(n, kvh, T, qh // kvh, m)
    s.masked_fill_(~seen[:, None, :, None], -math.inf)
    o = torch.matmul(_softmax(s).view(n, kvh, -1, m), v).view(n, kvh, T, qh // kvh, D).permute(0, 2, 1, 3, 4).reshape(n, T, qh, D)
    return o[real].to(st["q"].dtype)


def _plain_append(st):
    c = st["cache"]
    P = c["k"].shape[3]
    count = (st["off"][1:] - st["off"][:-1]).long()
    total = st["k"].shape[0]
    seq = torch.repeat_interleave(torch.arange(count.numel(), device=count.device), count, output_size=total)
    s = st["seqs"].long()[seq]
    pos = c["length"].long()[s] + torch.arange(total, device=count.device) - st["off"].long()[seq]
    page, slot = c["table"][s, pos // P].long(), pos % P
    c["k"][0][page, :, slot] = st["k"]
    c["v"][0][page, :, slot // 8, :, slot % 8] = st["v"]
    return {"k": c["k"], "v": c["v"]}


def _plain_free(c, ids):
    rows = c["table"][ids]
    c["refs"].index_add_(0, rows.clamp(min=0).reshape(-1), -(rows >= 0).to(torch.int32).reshape(-1))
    c["table"][ids] = -1
    c["length"][ids] = 0


def _plain_fork(c, src, dst):
    P, maxp = c["k"].shape[3], c["table"].shape[1]
    held = (torch.arange(maxp, device=src.device) * P) < c["length"][src][:, None]
    rows = torch.where(held, c["table"][src], -1)
    c["refs"].index_add_(0, rows.clamp(min=0).reshape(-1), held.to(torch.int32).reshape(-1))
    c["table"][dst] = rows
    c["length"][dst] = c["length"][src]


def _plain_reserve(c, ids, extra):
    """Pages for extra more tokens; a last page that others hold too is copied (its used tokens, in groups of eight)."""
    P, maxp = c["k"].shape[3], c["table"].shape[1]
    rows, length, n = c["table"][ids], c["length"][ids].long(), ids.numel()
    held = (rows >= 0).sum(1)
    new = ((length + extra + P - 1) // P - held).clamp(min=0)
    last = (length // P).clamp(max=maxp - 1)
    page = rows.gather(1, last[:, None])[:, 0].long().clamp(min=0)
    may = (extra > 0) & (length % P != 0) & (c["refs"][page] > 1)
    before = torch.arange(n, device=ids.device)
    rank = ((page[:, None] == page[None, :]) & may[None, :] & (before[None, :] < before[:, None])).sum(1)
    copy = (may & (c["refs"][page] - rank > 1)).long()
    take = new + copy
    first = take.cumsum(0) - take
    free = torch.argsort((c["refs"] != 0).to(torch.int32), stable=True)
    # The copied page's place first, then the new pages.
    j = torch.arange(maxp, device=ids.device)
    fresh = free[(first[:, None] + copy[:, None] + j - held[:, None]).clamp(0, free.numel() - 1)].to(torch.int32)
    rows = torch.where((j >= held[:, None]) & (j < (held + new)[:, None]), fresh, rows)
    to = free[first.clamp(max=free.numel() - 1)]
    rows = torch.where((copy[:, None] > 0) & (j == last[:, None]), to[:, None].to(torch.int32), rows)
    c["table"][ids] = rows
    c["refs"].index_add_(0, rows.clamp(min=0).reshape(-1).long(),
                         ((j >= held[:, None]) & (j < (held + new)[:, None])).to(torch.int32).reshape(-1))
    c["refs"].index_add_(0, to, copy.to(torch.int32))
    c["refs"].index_add_(0, page, -copy.to(torch.int32))
    # Copies land in pages nobody else holds; where there is none, the page is copied onto itself.
    to, used = torch.where(copy > 0, to, page), -(-(length % P) // 8)
    for name, group in (("k", torch.arange(P, device=ids.device) // 8), ("v", torch.arange(P // 8, device=ids.device))):
        pool = c[name]
        mask = (group < used[:, None])[None, :, None].view(1, n, 1, -1, *([1] * (pool.dim() - 4)))
        pool[:, to] = torch.where(mask, pool[:, page], pool[:, to])


def _plain_commit(c, ids, path, accepted):
    P, maxp = c["k"].shape[3], c["table"].shape[1]
    n, m = path.shape
    length = c["length"][ids].long()
    j = torch.arange(m, device=ids.device)
    take = j < accepted[:, None]
    src = torch.where(take, length[:, None] + path.long(), 0)
    dst = torch.where(take, length[:, None] + j, 0)
    rows = c["table"][ids].long()
    pick = take.reshape(-1).nonzero()[:, 0]
    sp, dp = (rows.gather(1, x // P).reshape(-1)[pick] for x in (src, dst))
    ss, ds = (x.reshape(-1)[pick] % P for x in (src, dst))
    c["k"][:, dp, :, ds] = c["k"][:, sp, :, ss]
    c["v"][:, dp, :, ds // 8, :, ds % 8] = c["v"][:, sp, :, ss // 8, :, ss % 8]
    length = length + accepted
    c["length"][ids] = length.to(torch.int32)
    over = (torch.arange(maxp, device=ids.device) >= ((length + P - 1) // P)[:, None]) & (rows >= 0)
    c["refs"].index_add_(0, rows.clamp(min=0).reshape(-1), -over.to(torch.int32).reshape(-1))
    c["table"][ids] = torch.where(over, -1, rows).to(torch.int32)


def _plain_pages(st):
    c, src, dst = st["cache"], st["src"].long(), st["dst"].long()
    _plain_free(c, dst)
    _plain_fork(c, src, dst)
    _plain_reserve(c, dst, st["nodes"].long())
    _plain_commit(c, dst, st["path"], st["accepted"])
    return _state_of(c)


# ---------------------------------------------------------------------- work


def work(case):
    """Each cached or new token's keys and values read once (for a page that several branches hold, once for each copy),
    queries read and outputs written once."""
    qh, kvh, D = HEADS[case["heads"]]
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "prompt":
        lens = _ragged(case, case["seqs"], case["len_lo"], case["len_hi"], 1)
        return {"bytes": sum(lens) * (2 * qh + 2 * kvh) * D * e, "flops": sum(2 * n * (n + 1) for n in lens) * qh * D}
    if case["kind"] == "pages":
        n, b, P = case["parents"], case["branches"], case["page"]
        ctx = _ragged(case, n, case["ctx_lo"], case["ctx_hi"], 1)
        nodes = _ragged(case, n * b, case["nodes_lo"], case["nodes_hi"], 2)
        # Every branch but the parent's own copy moves: the parent keeps its page, so each branch copies its used slots; of the
        # drafted tokens 0.7 are kept, and nearly all of those move.
        tokens = sum(b * (a % P) for a in ctx) + sum(0.7 * t for t in nodes)
        return {"bytes": max(1, 4 * tokens * case["layers"] * kvh * D * e), "flops": 0}
    ctx = _ragged(case, case["seqs"], case["ctx_lo"], case["ctx_hi"], 1)
    if case["kind"] == "append":
        new = _ragged(case, case["seqs"], case["new_lo"], case["new_hi"], 2)
        return {"bytes": 4 * sum(new) * kvh * D * e, "flops": 0}
    new = _ragged(case, case["seqs"], case["nodes_lo"], case["nodes_hi"], 2)
    return {"bytes": (2 * sum(a + t for a, t in zip(ctx, new)) * kvh + 2 * sum(new) * qh) * D * e,
            "flops": sum(4 * t * (a + t) for a, t in zip(ctx, new)) * qh * D}


# --------------------------------------------------------------------- exact


def _token(c, layer, s, pos):
    """Keys and values [positions, kv head, D] of sequence s in 64 bits."""
    P = c["k"].shape[3]
    page, slot = c["table"][s].long()[pos // P], pos % P
    return c["k"][layer][page, :, slot].double(), c["v"][layer][page, :, slot // 8, :, slot % 8].double()


def _attend(q, k, v, seen):
    """q [t, D] over k, v [m, D] with seen [t, m], in 64 bits."""
    s = (q @ k.T) * q.shape[1] ** -0.5
    p = torch.exp(s - s.masked_fill(~seen, -math.inf).amax(1, keepdim=True)) * seen
    return (p @ v) / p.sum(1, keepdim=True)


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "prompt":
        off, q = st["off"].tolist(), st["q"]
        group = q.shape[1] // st["k"].shape[1]
        out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
        for a, b in zip(off[:-1], off[1:]):
            for h in range(q.shape[1]):
                k, v = st["k"][a:b, h // group].double(), st["v"][a:b, h // group].double()
                for i in range(a, b, 2048):  # rows at a time
                    e = min(b, i + 2048)
                    at = torch.arange(i - a, e - a, device=q.device)
                    out[i:e, h] = _attend(q[i:e, h].double(), k[:e - a], v[:e - a], torch.arange(e - a, device=q.device) <= at[:, None])
        return out
    c = st["cache"]
    if case["kind"] == "tree":
        off, par, q = st["off"].tolist(), st["parent"].tolist(), st["q"]
        group = q.shape[1] // c["k"].shape[2]
        out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
        for i, (a, b) in enumerate(zip(off[:-1], off[1:])):
            n = int(c["length"][i])
            seen = torch.zeros((b - a, n + b - a), dtype=torch.bool)
            seen[:, :n] = True
            for t in range(b - a):
                j = t
                while j >= 0:
                    seen[t, n + j] = True
                    j = par[a + j]
            seen = seen.to(q.device)
            k, v = _token(c, 0, i, torch.arange(n + b - a, device=q.device))
            for h in range(q.shape[1]):
                out[a:b, h] = _attend(q[a:b, h].double(), k[:, h // group], v[:, h // group], seen)
        return out
    return None  # copied values and whole numbers, which have to be equal
