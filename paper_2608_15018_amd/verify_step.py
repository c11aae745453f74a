"""One speculative-decoding step through whole layers: attention over the cache and
the verify-MoE layer, from prompts to the accepted path.

    python -m paper_2608_15018_amd.verify_step [--layers 4] [--seqs 8] [--nodes 16] [--steps 4]
                                               [--dense bf16|fp8]

A layer is: query, key and value projections, attention, output projection, and the
MoE layer, each added to the residual stream, with an RMS norm before either half.
With dense="bf16" attention, the cache and the MoE layer are the library's, the
projections and the norm torch's, and positions do not enter.  With dense="fp8" all is
the library's: norms that add to the residual stream and hand on 8-bit rows, projections
in 8 bits with a scale for each block of 128, and queries and keys rotated by their
positions on their way to attention and cache.  Weights are random, so drafted trees and
accepted paths are drawn, not predicted: what a step does, and what it costs, do not
depend on them.
"""

from __future__ import annotations

import argparse

import torch

from . import _lib, dense as d8
from .attention import KVCache, TreeAttention, prompt_attention
from .pipeline import VerifyPass, pack_expert_weights

MAX_BATCH = 256  # tokens of one verify-MoE call


def _norm(x):
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


class VerifyStack:
    """Layers of random weights with their cache, for up to `seqs` sequences of up to
    `max_tokens` tokens and drafted trees of up to `nodes` nodes."""

    def __init__(self, layers=4, hidden=2048, ffn=1024, n_experts=64, top_k=8, n_heads=16,
                 n_kv_heads=4, head_dim=128, seqs=8, nodes=16, max_tokens=4096, page_size=64,
                 seed=0, device="cuda", dense="bf16", theta=1e6):
        if dense not in ("bf16", "fp8"):
            raise ValueError(f"dense: expected bf16 or fp8, got {dense}")
        g = torch.Generator(device=device).manual_seed(seed)

        def weight(*shape):
            w = torch.randn(shape, generator=g, device=device, dtype=torch.bfloat16)
            return w.mul_(shape[-1] ** -0.5)

        self.heads = (n_heads, n_kv_heads, head_dim)
        self.qkv = [weight((n_heads + 2 * n_kv_heads) * head_dim, hidden) for _ in range(layers)]
        self.out = [weight(hidden, n_heads * head_dim) for _ in range(layers)]
        self.router = [weight(n_experts, hidden) for _ in range(layers)]
        self.experts = [pack_expert_weights(({"gate": weight(n_experts, ffn, hidden),
                                              "up": weight(n_experts, ffn, hidden),
                                              "down": weight(n_experts, hidden, ffn)}, {}), "bf16")
                        for _ in range(layers)]
        self.layer = _lib.make_layer(hidden=hidden, ffn=ffn, n_experts=n_experts, top_k=top_k,
                                     cap=top_k, alpha=0.0, flags=_lib.PACKED_WEIGHTS)
        self.dense = dense
        if dense == "fp8":
            self.qkv, self.out = ([d8.quantize_weight(w) for w in ws] for ws in (self.qkv, self.out))
            self.norm = torch.ones(hidden, dtype=torch.bfloat16, device=device)
            at = torch.arange(head_dim // 2, device=device, dtype=torch.float64)
            self.inv_freq = (theta ** (-2 * at / head_dim)).float()
        pages = -(-(max_tokens + nodes) // page_size)
        self.cache = KVCache(layers, n_kv_heads, head_dim, seqs * pages, page_size, seqs, pages,
                             device=device)
        self.attention = TreeAttention(self.cache, n_heads, seqs, nodes)
        self.passes = {}
        self.conf = torch.ones(MAX_BATCH, device=device)

    def _moe(self, l, x):
        """The MoE layer over any number of tokens, in verify batches."""
        y = torch.empty(x.shape, dtype=torch.float32, device=x.device)
        for i in range(0, x.shape[0], MAX_BATCH):
            part = x[i:i + MAX_BATCH]
            n = part.shape[0]
            if n not in self.passes:
                self.passes[n] = VerifyPass(self.layer, n, x.device, fused=True)
            y[i:i + n] = self.passes[n](part, self.router[l], self.conf[:n], self.experts[l][1])
        return y

    def _layers_fp8(self, x, seqs, tok_off, parent, attend, prompt):
        Hq, Hkv, D = self.heads
        n = x.shape[0]
        pos = self.cache.positions(seqs, tok_off, n, parent)
        res = x.to(torch.float32, copy=True)  # the residual stream, which the norms add to
        y = None
        for l in range(len(self.qkv)):
            a = (d8.add_norm(res, self.norm, out_dtype=d8.E4M3) if y is None else
                 d8.add_norm(y, self.norm, res, out_dtype=d8.E4M3))
            qkv = d8.fp8_matmul(a, self.qkv[l]).view(n, Hq + 2 * Hkv, D)
            q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
            # In place; attention of prompts takes the turned keys from here, not from the cache.
            self.cache.append_rotated(l, q, k, v, seqs, tok_off, pos, self.inv_freq, out=q,
                                      k_out=k if prompt else None)
            o = d8.quantize(attend(l, q, k, v).view(n, Hq * D))
            h = d8.add_norm(d8.fp8_matmul(o, self.out[l]), self.norm, res, out_dtype=torch.bfloat16)
            y = self._moe(l, h)
        return res if y is None else res.add_(y)

    def _layers(self, x, seqs, tok_off, parent, attend, prompt=False):
        if self.dense == "fp8":
            return self._layers_fp8(x, seqs, tok_off, parent, attend, prompt)
        Hq, Hkv, D = self.heads
        x = x.float()
        for l in range(len(self.qkv)):
            qkv = (_norm(x) @ self.qkv[l].T).view(-1, Hq + 2 * Hkv, D)
            q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
            self.cache.append(l, k, v, seqs, tok_off)
            o = attend(l, q, k, v)
            x = x + (o.reshape(x.shape[0], -1) @ self.out[l].T).float()
            x = x + self._moe(l, _norm(x))
        return x

    def prefill(self, x, seqs, tok_off):
        """Whole prompts x [n_tokens, hidden], packed, into empty sequences; returns the
        last layer's output."""
        counts = tok_off[1:] - tok_off[:-1]
        self.cache.reserve(seqs, counts)
        y = self._layers(x, seqs, tok_off, None,
                         lambda l, q, k, v: prompt_attention(q, k, v, tok_off), prompt=True)
        self.cache.commit(seqs, None, counts)
        return y

    def verify(self, x, seqs, tok_off, parent):
        """Drafted trees x [n_tokens, hidden], packed, over what the sequences hold;
        returns the last layer's output.  Nothing is kept until commit."""
        self.cache.reserve(seqs, tok_off[1:] - tok_off[:-1])
        return self._layers(x, seqs, tok_off, parent,
                            lambda l, q, k, v: self.attention(l, q, seqs, tok_off, parent))

    def commit(self, seqs, path, n_accept):
        """Keeps the accepted path of every tree."""
        self.cache.commit(seqs, path, n_accept)


def draw_trees(seqs, nodes, generator):
    """Trees of `nodes` nodes and, of each, the path to a drawn node: parent [seqs *
    nodes], path [seqs, nodes] (ascending, padded with -1), n_accept [seqs], on the host."""
    parent, path, accept = [], [], []
    for _ in range(seqs):
        u = torch.rand(nodes, generator=generator).tolist()
        p = [i - 1 if u[i] < 0.6 else int(torch.randint(-1, max(i, 1), (1,), generator=generator))
             if i else -1 for i in range(nodes)]
        node, up = int(torch.randint(0, nodes, (1,), generator=generator)), []
        while node >= 0:
            up.append(node)
            node = p[node]
        parent += p
        path.append(up[::-1] + [-1] * (nodes - len(up)))
        accept.append(len(up))
    i32 = torch.int32
    return (torch.tensor(parent, dtype=i32), torch.tensor(path, dtype=i32),
            torch.tensor(accept, dtype=i32))


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--seqs", type=int, default=8)
    ap.add_argument("--nodes", type=int, default=16)
    ap.add_argument("--steps", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=1000)
    ap.add_argument("--dense", choices=("bf16", "fp8"), default="bf16")
    a = ap.parse_args(argv)
    hidden = 2048
    m = VerifyStack(layers=a.layers, hidden=hidden, seqs=a.seqs, nodes=a.nodes,
                    max_tokens=a.prompt + a.steps * a.nodes, dense=a.dense)
    g = torch.Generator().manual_seed(1)
    ids = torch.arange(a.seqs, dtype=torch.int32, device="cuda")
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]

    def timed(f, *args):
        ev[0].record()
        y = f(*args)
        ev[1].record()
        torch.cuda.synchronize()
        return y, ev[0].elapsed_time(ev[1])

    # Once untimed: the libraries load and the buffers are allocated.
    x = torch.randn((a.seqs * a.prompt, hidden), device="cuda")
    off = torch.arange(0, a.seqs * a.prompt + 1, a.prompt, dtype=torch.int32, device="cuda")
    m.prefill(x, ids, off)
    m.cache.free(ids)
    _, ms = timed(m.prefill, x, ids, off)
    print(f"prefill: {a.seqs} prompts of {a.prompt} tokens, {a.layers} layers: {ms:.2f} ms")
    off = torch.arange(0, a.seqs * a.nodes + 1, a.nodes, dtype=torch.int32, device="cuda")
    for step in range(a.steps):
        parent, path, accept = (t.cuda() for t in draw_trees(a.seqs, a.nodes, g))
        x = torch.randn((a.seqs * a.nodes, hidden), device="cuda")
        _, ms = timed(m.verify, x, ids, off, parent)
        _, kept = timed(m.commit, ids, path, accept)
        print(f"step {step}: verified {a.seqs * a.nodes} drafted tokens in {ms:.2f} ms, kept "
              f"{int(accept.sum())} in {kept:.3f} ms, lengths {m.cache.length.tolist()}")


if __name__ == "__main__":
    main()
