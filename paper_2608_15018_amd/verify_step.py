"""One speculative-decoding step through whole layers: attention over the cache and
the verify-MoE layer, from prompts to the accepted path.

    python -m paper_2608_15018_amd.verify_step [--layers 4] [--seqs 8] [--nodes 16] [--steps 4]

A layer is: query, key and value projections, attention, output projection, and the
MoE layer, each added to the residual stream, with an RMS norm before either half.
Attention, the cache and the MoE layer are the library's; the projections and the norm
are torch's.  Weights are random, so drafted trees and accepted paths are drawn, not
predicted: what a step does, and what it costs, do not depend on them.
"""

from __future__ import annotations

import argparse

import torch

from . import _lib
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
                 seed=0, device="cuda"):
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

    def _layers(self, x, seqs, tok_off, attend):
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
        y = self._layers(x, seqs, tok_off, lambda l, q, k, v: prompt_attention(q, k, v, tok_off))
        self.cache.commit(seqs, None, counts)
        return y

    def verify(self, x, seqs, tok_off, parent):
        """Drafted trees x [n_tokens, hidden], packed, over what the sequences hold;
        returns the last layer's output.  Nothing is kept until commit."""
        self.cache.reserve(seqs, tok_off[1:] - tok_off[:-1])
        return self._layers(x, seqs, tok_off,
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
    a = ap.parse_args(argv)
    hidden = 2048
    m = VerifyStack(layers=a.layers, hidden=hidden, seqs=a.seqs, nodes=a.nodes,
                    max_tokens=a.prompt + a.steps * a.nodes)
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
