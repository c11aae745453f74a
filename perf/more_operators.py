"""Performance cases of the dense half of a verify layer: norms, 8-bit products, and the rotation that goes before the cache.

Four kinds of call, in the order in which a layer makes them:
  norm      a layer's output added to the residual stream and normalised by its root mean square (`add_norm`), in 8 bits with
            scales where a product follows, in bf16 or fp32 where the experts or a program's own code do.
  matmul    a product of 8-bit floating point rows and weights with a scale for each block of 128 (`fp8_matmul`): projections and logits.
  rotate    the positions of a step's new tokens (`KVCache.positions`), their queries and keys rotated by them, the keys and values
            written into the cache's pages (`KVCache.append_rotated`).
  quantize  rows in 8 bits with scales (`quantize`), as the output projection takes the attention's.

`own` chooses between the framework's calls and a plain form of elementary operations in 32 bits.

Rows in 8 bits: codes [rows, K] (e4m3), scales [ceil(K / 128), rows]: the scale of a row's block is its largest magnitude / 448.
Weights: codes [N, K], scales [ceil(N / 128), ceil(K / 128)].  The cache: K [layer, page, kv head, slot, D], V [layer, page,
kv head, slot / 8, D, slot % 8], table [sequence, page of the sequence] (-1: none), length [sequence], refs [page].
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
E4M3 = torch.float8_e4m3fn
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": E4M3}
BYTES = {"f32": 4, "bf16": 2, "e4m3": 1}
BLOCK, LARGEST, FLOOR = 128, 448.0, 2.0 ** -100
EPS = 1e-6


# --------------------------------------------------------------------- cases


def listed():
    return [
        # One token between two layers of a draft step, on its way into the query, key and value projection: latency alone counts.
        dict(name="norm 1 token", kind="norm", rows=1, hidden=2048, x="bf16", res="f32", w="bf16", out="e4m3"),
        # A verify batch on its way to the experts, whose hidden size is no multiple of 128.
        dict(name="norm verify 251 tokens", kind="norm", rows=251, hidden=2880, x="bf16", res="f32", w="bf16", out="e4m3"),
        # Several prompts at once, the residual stream in bf16.
        dict(name="norm prompt 8193 tokens", kind="norm", rows=8193, hidden=4096, x="bf16", res="bf16", w="f32", out="e4m3"),
        # The attention's output of one verified tree.
        dict(name="quantize 16 tokens", kind="quantize", rows=16, hidden=4096, x="bf16"),
        # The attention's output of a long document.
        dict(name="quantize 12289 tokens", kind="quantize", rows=12289, hidden=4096, x="bf16"),
        # Query, key and value projection of one token: the weights are read, and that is all.
        dict(name="matmul 1 token", kind="matmul", m=1, n=5120, k=2048, out="bf16"),
        # Logits of the 16 nodes of a drafted tree: the largest weights of a step.
        dict(name="matmul logits 16 nodes", kind="matmul", m=16, n=32000, k=4096, out="f32"),
        # A serving batch of trees.
        dict(name="matmul verify 251 tokens", kind="matmul", m=251, n=5120, k=2880, out="bf16"),
        # Several prompts at once: bound by the matrix cores.
        dict(name="matmul prompt 8193 tokens", kind="matmul", m=8193, n=6144, k=4096, out="bf16"),
        # The fp32 parity layer's attention: one drafted tree of 8 nodes.
        dict(name="rotate f32 tiny 8 nodes", kind="rotate", heads="tiny", dtype="f32", seqs=1, ctx_lo=200, ctx_hi=200, new_lo=8, new_hi=8, page=16,
             rot=64, pairs=False, tree=True, keep=False, mix=1),
        # The new token of every conversation of a decoding batch.
        dict(name="rotate 48 tokens", kind="rotate", heads="mixtral", dtype="bf16", seqs=48, ctx_lo=100, ctx_hi=4000, new_lo=1, new_hi=1, page=64,
             rot=128, pairs=False, tree=False, keep=False, mix=2),
        # Prompts entering the cache, their rotated keys kept for the prompts' own attention.
        dict(name="rotate prompts", kind="rotate", heads="qwen3", dtype="bf16", seqs=5, ctx_lo=0, ctx_hi=0, new_lo=1000, new_hi=5000, page=64, rot=128,
             pairs=False, tree=False, keep=True, mix=3),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "quantize", "matmul", "matmul", "matmul", "rotate", "rotate"))
    if kind in ("norm", "quantize"):
        rows = _log_int(rng, 1, 12289)
        c = dict(kind=kind, rows=rows, hidden=16 * _log_int(rng, 2, min(512, 8193 * 256 // rows)), x=rng.choice(("bf16", "bf16", "f32")))
        if kind == "norm":
            c.update(res=rng.choice(("f32", "bf16", "none")), w=rng.choice(("f32", "bf16")), out=rng.choice(("e4m3", "e4m3", "bf16", "f32")))
        return c
    if kind == "matmul":
        m, k = _log_int(rng, 1, 8193), 16 * _log_int(rng, 8, 512)
        most = min(32000 * 4096 // k, 8193 * 6144 * 4096 // (m * k))
        return dict(kind=kind, m=m, n=_log_int(rng, 17, min(32000, most)), k=k, out=rng.choice(("bf16", "bf16", "f32")))
    c = dict(kind=kind, dtype=rng.choice(("bf16", "bf16", "bf16", "f32")), page=rng.choice((16, 32, 64, 128)), mix=rng.randrange(1 << 20))
    c["heads"] = rng.choice([h for h in HEADS if h != "tiny"]) if c["dtype"] == "bf16" else rng.choice(("tiny", "mixtral", "gptoss"))
    D = HEADS[c["heads"]][2]
    c["rot"] = rng.choice((D, D, D // 2, 16 * rng.randint(1, D // 16)))
    c["pairs"] = rng.random() < 0.4
    c["tree"] = rng.random() < 0.5
    new = _log_int(rng, 1, 64 if c["tree"] else 4096)
    c["seqs"] = _log_int(rng, 1, max(1, min(64, 8192 // new)))
    ctx = 0 if new > 256 else _log_int(rng, 1, max(2, 65536 // c["seqs"]))
    c.update(ctx_lo=min(ctx, _log_int(rng, max(1, ctx // 8), max(1, ctx))), ctx_hi=ctx, new_lo=_log_int(rng, max(1, new // 4), new), new_hi=new,
             keep=rng.random() < 0.5)
    return c


def _ragged(case, lo, hi, key):
    """A whole number between lo and hi for each sequence of the case; the first is hi."""
    rng = random.Random(case["mix"] * 1009 + key)
    return [hi] + [rng.randint(lo, hi) for _ in range(case["seqs"] - 1)]


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


def _activations(rows, hidden, dtype, g):
    """Hidden states: rows of different size, some coordinates far larger than the others."""
    x = _randn((rows, hidden), torch.float32, g)
    x *= torch.exp(_randn((rows, 1), torch.float32, g, 0.5))
    x *= torch.where(torch.rand((hidden,), generator=g, device=DEVICE) < 0.01, 20.0, 1.0)
    return x.to(dtype)


def prepare(case, seed):
    kind = case["kind"]
    if kind in ("norm", "quantize"):
        rows, hidden = case["rows"], case["hidden"]
        g = _gen(seed, rows, hidden)
        st = {"kind": kind, "x": _activations(rows, hidden, DTYPES[case["x"]], g)}
        if kind == "norm":
            st["w"] = (1 + _randn((hidden,), torch.float32, g, 0.1)).to(DTYPES[case["w"]])
            st["residual"] = None if case["res"] == "none" else (4 * _activations(rows, hidden, torch.float32, g)).to(DTYPES[case["res"]])
            st["out"] = DTYPES[case["out"]]
        return st
    if kind == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        g = _gen(seed, m, n, k)
        x, sx = _codes(_activations(m, k, torch.float32, g))
        w = _randn((n, k), torch.float32, g, k ** -0.5)
        w *= torch.exp(_randn((n, 1), torch.float32, g, 0.3))
        w, sw = _weight_codes(w)
        return {"kind": kind, "x": x, "sx": sx, "w": w, "sw": sw, "out": DTYPES[case["out"]]}
    return _prepare_rotate(case, seed)


def _prepare_rotate(case, seed):
    dt, P = DTYPES[case["dtype"]], case["page"]
    qh, kvh, D = HEADS[case["heads"]]
    g = _gen(seed, case["mix"])
    ctx, new = _ragged(case, case["ctx_lo"], case["ctx_hi"], 1), _ragged(case, case["new_lo"], case["new_hi"], 2)
    need = [-(-(a + b) // P) for a, b in zip(ctx, new)]
    total, seqs = sum(need) + 3, case["seqs"]
    order = torch.randperm(total, generator=g, device=DEVICE).to(torch.int32)
    table = torch.full((seqs, max(need)), -1, dtype=torch.int32, device=DEVICE)
    refs = torch.zeros(total, dtype=torch.int32, device=DEVICE)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    refs[order[:at].long()] = 1
    cache = {"k": _randn((1, total, kvh, P, D), dt, g), "v": _randn((1, total, kvh, P // 8, D, 8), dt, g), "table": table, "length": _ints(ctx),
             "refs": refs}
    off = [0]
    for n in new:
        off.append(off[-1] + n)
    qkv = _randn((off[-1], qh + 2 * kvh, D), dt, g)  # one projection's output, as a layer has it
    st = {"kind": "rotate", "cache": cache, "seqs": torch.arange(seqs, device=DEVICE).to(torch.int32), "off": _ints(off), "most": max(new),
          "q": qkv[:, :qh], "k": qkv[:, qh:qh + kvh], "v": qkv[:, qh + kvh:], "keep": case["keep"], "pairs": case["pairs"], "parent": None}
    st["freq"] = (1e6 ** (-torch.arange(case["rot"] // 2, device=DEVICE, dtype=torch.float64) * 2 / case["rot"])).float()
    if case["tree"]:
        # A node hangs below the one before it, or below an earlier one or the last kept token (-1).
        node = torch.cat([torch.arange(n, device=DEVICE) for n in new])
        u = torch.rand((2, node.numel()), generator=g, device=DEVICE)
        st["parent"] = torch.where(u[0] < 0.6, node - 1, (u[1] * (node + 1)).long() - 1).clamp(min=-1).minimum(node - 1).to(torch.int32)
    if own:
        import paper_2608_15018_amd as s2

        st["handle"] = s2.KVCache(1, kvh, D, total, P, seqs, max(need), dtype=dt, **cache)
    return st


# ----------------------------------------------------------------------- run


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _plain_norm, "quantize": _plain_quantize, "matmul": _plain_matmul, "rotate": _plain_rotate}[state["kind"]](state)


def _run_own(st):
    import paper_2608_15018_amd as s2

    if st["kind"] == "norm":
        y = s2.add_norm(st["x"], st["w"], st["residual"], EPS, out_dtype=st["out"])
        return {"residual": st["residual"], "y": tuple(y) if st["out"] is E4M3 else y}
    if st["kind"] == "quantize":
        return tuple(s2.quantize(st["x"]))
    if st["kind"] == "matmul":
        return s2.fp8_matmul(s2.Fp8Rows(st["x"], st["sx"]), s2.Fp8Weight(st["w"], st["sw"]), out_dtype=st["out"])
    cache = st["handle"]
    pos = cache.positions(st["seqs"], st["off"], st["q"].shape[0], st["parent"])
    k_out = torch.empty(st["k"].shape, dtype=st["k"].dtype, device=st["k"].device) if st["keep"] else None
    q = cache.append_rotated(0, st["q"], st["k"], st["v"], st["seqs"], st["off"], pos, st["freq"], st["pairs"], k_out=k_out)
    return {"pos": pos, "q": q, "k_out": k_out, "k": cache.k, "v": cache.v}


def _codes(y):
    """Rows y in 8 bits: codes of y's shape, scales [blocks, rows]."""
    rows, K = y.shape
    pad = -K % BLOCK
    b = torch.nn.functional.pad(y, (0, pad)).view(rows, -1, BLOCK)
    scale = b.abs().amax(-1).clamp(min=FLOOR) / LARGEST
    codes = (b / scale[..., None]).to(E4M3).view(rows, -1)
    return (codes[:, :K].contiguous() if pad else codes), scale.t().contiguous()


def _weight_codes(w):
    N, K = w.shape
    b = torch.nn.functional.pad(w, (0, -K % BLOCK, 0, -N % BLOCK))
    b = b.view(b.shape[0] // BLOCK, BLOCK, -1, BLOCK)
    scale = b.abs().amax((1, 3)).clamp(min=FLOOR) / LARGEST
    codes = (b / scale[:, None, :, None]).to(E4M3).view(b.shape[0] * BLOCK, -1)
    return codes[:N, :K].contiguous(), scale


def _plain_norm(st):
    h = st["x"].float()
    if st["residual"] is not None:
        h = h + st["residual"].float()
        st["residual"].copy_(h)
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * st["w"].float()
    return {"residual": st["residual"], "y": _codes(y) if st["out"] is E4M3 else y.to(st["out"])}


def _plain_quantize(st):
    return _codes(st["x"].float())


def _plain_matmul(st):
    m, k = st["x"].shape
    n = st["w"].shape[0]
    x = st["x"].float() * st["sx"].t().repeat_interleave(BLOCK, 1)[:, :k]
    w = st["w"].float() * st["sw"].repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]
    return torch.matmul(x, w.t()).to(st["out"])


def _rotated(x, cos, sin, pairs):
    """Rows x [n, heads, D] turned by the angles of their positions (cos, sin [n, rot / 2]) in 32 bits."""
    half = cos.shape[1]
    y = x.float()
    a, b = (y[..., 0:2 * half:2], y[..., 1:2 * half:2]) if pairs else (y[..., :half], y[..., half:2 * half])
    c, s = cos[:, None], sin[:, None]
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack((a, b), -1).flatten(-2) if pairs else torch.cat((a, b), -1)
    return torch.cat((turned, y[..., 2 * half:]), -1).to(x.dtype)


def _plain_rotate(st):
    c, total = st["cache"], st["q"].shape[0]
    off, dev = st["off"].long(), st["q"].device
    count = off[1:] - off[:-1]
    seq = torch.repeat_interleave(torch.arange(count.numel(), device=dev), count, output_size=total)
    s = st["seqs"].long()[seq]
    row = torch.arange(total, device=dev)
    begin = c["length"].long()[s]
    slot = begin + row - off[seq]
    if st["parent"] is None:
        pos = slot
    else:
        # Depths by doubling: after each step `up` is twice as many ancestors away, and depth counts those passed.
        parent = st["parent"].long()
        up = torch.where(parent < 0, total, off[seq] + parent)
        up = torch.cat((up, up.new_full((1,), total)))
        depth = (up < total).long()
        for _ in range(max(1, (st["most"] - 1).bit_length())):
            depth = depth + depth[up]
            up = up[up]
        pos = begin + depth[:total]
    angle = pos.double()[:, None] * st["freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    q, k = (_rotated(st[name], cos, sin, st["pairs"]) for name in ("q", "k"))
    P = c["k"].shape[3]
    page, at = c["table"][s, slot // P].long(), slot % P
    c["k"][0][page, :, at] = k
    c["v"][0][page, :, at // 8, :, at % 8] = st["v"]
    return {"pos": pos.to(torch.int32), "q": q, "k_out": k if st["keep"] else None, "k": c["k"], "v": c["v"]}


# --------------------------------------------------------------------- exact


def exact(case, seed):
    """What run() returns for these inputs, from the definitions in 64 bits."""
    st = prepare(case, seed)
    if st["kind"] == "quantize":
        return _exact_codes(st["x"].double())
    if st["kind"] == "norm":
        h = st["x"].double()
        if st["residual"] is not None:
            h += st["residual"].double()
        length = torch.linalg.vector_norm(h, dim=1) / math.sqrt(h.shape[1])
        y = h / torch.sqrt(length.square() + EPS)[:, None] * st["w"].double()
        return {"residual": None if st["residual"] is None else h, "y": _exact_codes(y) if case["out"] == "e4m3" else y}
    if st["kind"] == "matmul":
        y = 0
        for b in range(st["sx"].shape[0]):
            part = slice(b * BLOCK, (b + 1) * BLOCK)
            rows = torch.div(torch.arange(st["w"].shape[0], device=DEVICE), BLOCK, rounding_mode="floor")
            left = st["x"][:, part].double() * st["sx"][b].double()[:, None]
            y = y + left @ (st["w"][:, part].double() * st["sw"][rows, b].double()[:, None]).t().contiguous()
        return y
    return _exact_rotate(case, st)


def _exact_codes(y):
    K = y.shape[1]
    codes, scales = torch.empty_like(y), []
    for k in range(0, K, BLOCK):
        part = y[:, k:k + BLOCK]
        scale = torch.clamp(part.abs().max(1).values, min=FLOOR) / LARGEST
        z = part / scale[:, None]
        # Three bits below the leading one, whose exponent is at least -6.
        step = torch.exp2(torch.clamp(torch.frexp(z).exponent.double() - 1, min=-6) - 3)
        codes[:, k:k + BLOCK] = torch.round(z / step) * step
        scales.append(scale)
    return codes, torch.stack(scales)


def _exact_rotate(case, st):
    c, off = st["cache"], st["off"].tolist()
    lengths, P = c["length"].tolist(), case["page"]
    k_pool, v_pool = c["k"].double(), c["v"].double()
    parents = None if st["parent"] is None else st["parent"].tolist()
    pos = []
    for i, n in enumerate(lengths):
        depth = []
        for j in range(off[i + 1] - off[i]):
            up = j - 1 if parents is None else parents[off[i] + j]
            depth.append(0 if up < 0 else depth[up] + 1)
        pos += [n + d for d in depth]
    turn = torch.tensor(pos, dtype=torch.float64, device=DEVICE)[:, None] * st["freq"].double()
    turn = torch.polar(torch.ones_like(turn), turn)[:, None]

    def turned(x):
        y, rot = x.double(), case["rot"]
        part = y[..., :rot]
        z = part.unflatten(-1, (rot // 2, 2)) if case["pairs"] else part.unflatten(-1, (2, rot // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        y[..., :rot] = (z if case["pairs"] else z.transpose(-1, -2)).flatten(-2)
        return y

    q, k = turned(st["q"]), turned(st["k"])
    for i, n in enumerate(lengths):
        new = off[i + 1] - off[i]
        at = torch.arange(n, n + new, device=DEVICE)
        page = c["table"][i].long()[at // P]
        k_pool[0, page, :, at % P] = k[off[i]:off[i + 1]]
        v_pool[0, page, :, at % P // 8, :, at % 8] = st["v"][off[i]:off[i + 1]].double()
    return {"pos": None, "q": q, "k_out": k if st["keep"] else None, "k": k_pool, "v": v_pool}


# ---------------------------------------------------------------------- work


def work(case):
    """Inputs read once, outputs written once; of the cache, what is written."""
    if case["kind"] in ("norm", "quantize"):
        rows, hidden = case["rows"], case["hidden"]
        out = case.get("out", "e4m3")
        n = rows * hidden * (BYTES[case["x"]] + BYTES[out]) + (4 * rows * -(-hidden // BLOCK) if out == "e4m3" else 0)
        if case["kind"] == "norm":
            n += hidden * BYTES[case["w"]] + (2 * rows * hidden * BYTES[case["res"]] if case["res"] != "none" else 0)
        return {"bytes": n, "flops": rows * hidden * (6 if case["kind"] == "norm" else 2)}
    if case["kind"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        blocks = -(-k // BLOCK)
        return {"bytes": (m + n) * k + 4 * blocks * (m + -(-n // BLOCK)) + m * n * BYTES[case["out"]], "flops": 2 * m * n * k}
    qh, kvh, D = HEADS[case["heads"]]
    tokens = sum(_ragged(case, case["new_lo"], case["new_hi"], 2))
    heads = 2 * qh + 4 * kvh + (kvh if case["keep"] else 0)
    return {"bytes": tokens * heads * D * BYTES[case["dtype"]] + 4 * tokens, "flops": 3 * tokens * (qh + kvh) * case["rot"]}
