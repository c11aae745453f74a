"""The attention side of a verify step: the paged cache of keys and values, the
attention of drafted trees over it, and that of whole prompts.  Argument
marshalling only; every step is a call into libs2moe.so.

A verify step of one layer, for sequences `seqs` whose trees' tokens are packed
one after another (`tok_off` their offsets, `parent` the index of each node's
parent within its tree, -1 below the last kept token):

    cache.reserve(seqs, n_nodes)                  # once per step, all layers
    cache.append(layer, k, v, seqs, tok_off)      # the drafted tokens' K and V
    o = attention(layer, q, seqs, tok_off, parent)
    ...                                           # the layer's experts, the other layers
    cache.commit(seqs, path, n_accept)            # once per step: keep the accepted path

Calls are made with the cache's GPU current.  With `stream`, the inputs have to be
ready there, and kept (or recorded on it) until it is done with them, as with any torch
tensor that another stream reads.
"""

from __future__ import annotations

import ctypes
import threading

import torch

from . import _lib

KV_NO_PAGES, KV_TOO_LONG, KV_BAD_SEQ, KV_BUSY, KV_BAD_PATH = 1, 2, 4, 8, 16
KV_MAX_REQUESTS = 1024

_CODES = {torch.float32: _lib.F32, torch.bfloat16: _lib.BF16}


def _code(dtype) -> int:
    if dtype not in _CODES:
        raise TypeError(f"expected torch.float32 or torch.bfloat16, got {dtype}")
    return _CODES[dtype]


_I32 = torch.int32


# The checks are on every call's path to the GPU, which at the smallest sizes waits
# for them: each property is read once.
def _ints(t, name, n):
    """Pointer of int32 [n]."""
    if t.dtype is not _I32 or t.dim() != 1 or t.size(0) != n or not t.is_contiguous():
        raise ValueError(f"{name}: expected contiguous int32 [{n}], got {t.dtype} {tuple(t.shape)}")
    return t.data_ptr()


def _rows(t, name, heads, head_dim, dtype):
    """(pointer, elements from one token to the next, tokens) of [n, heads,
    head_dim] whose heads lie together."""
    shape = t.shape
    if t.dtype is not dtype or len(shape) != 3 or shape[1] != heads or shape[2] != head_dim:
        raise ValueError(f"{name}: expected {dtype} [n, {heads}, {head_dim}], got {t.dtype} "
                         f"{tuple(shape)}")
    s0, s1, s2 = t.stride()
    if s2 != 1 or (s1 != head_dim and heads > 1):
        raise ValueError(f"{name}: the heads of a token must lie together (strides {t.stride()})")
    n = shape[0]
    return t.data_ptr(), s0 if n > 1 else heads * head_dim, n


def _refuse(gpu, **tensors):
    """Says which of the tensors, which the kernels would read by their pointers, is
    not on GPU `gpu`."""
    for name, t in tensors.items():
        if gpu < 0 or t.get_device() != gpu:
            where = f"GPU {gpu}" if gpu >= 0 else "a GPU"
            raise _lib.S2moeError(_lib.EINVAL, f"{name} is on {t.device}, not on {where}")


def _other(stream, device):
    """`stream` as torch's object, or None if it is the current one."""
    if _lib._stream(stream) == _lib._stream(None):
        return None
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(stream), device=device)


def _result(like, shape, other):
    """Memory for what a stream writes.  From that stream's pool: the current
    stream's may hold blocks that work queued there still uses.  The caller goes on
    with it on the current stream, so it is not given back while work there has it."""
    if other is None:
        return like.new_empty(shape)
    with torch.cuda.stream(other):
        out = like.new_empty(shape)
    out.record_stream(torch.cuda.current_stream())
    return out


class KVCache:
    """Pages of keys and values of `n_layers` layers for up to `max_seqs`
    sequences of up to `max_pages` pages each.  Allocates the arrays that are
    not given and then empties the cache; given all five (k, v, table, length,
    refs) it takes them as they are.

    `status` holds one word per request of the last page operation (bits KV_*,
    0: done) and `copied` the pages that the last reserve copied, both on the
    device; every operation writes them.  Threads may share a cache; operations on
    different streams, which all read and write its table, lengths and counts, are the
    caller's to order."""

    def __init__(self, n_layers: int, n_kv_heads: int, head_dim: int, n_pages: int,
                 page_size: int, max_seqs: int, max_pages: int, dtype=torch.bfloat16,
                 device="cuda", k=None, v=None, table=None, length=None, refs=None):
        code = _code(dtype)
        i32 = torch.int32
        want = {"k": ((n_layers, n_pages, n_kv_heads, page_size, head_dim), dtype),
                "v": ((n_layers, n_pages, n_kv_heads, page_size // 8, head_dim, 8), dtype),
                "table": ((max_seqs, max_pages), i32), "length": ((max_seqs,), i32),
                "refs": ((n_pages,), i32)}
        given = {"k": k, "v": v, "table": table, "length": length, "refs": refs}
        fresh = any(t is None for t in given.values())
        for name, (shape, dt) in want.items():
            t = given[name]
            if t is None:
                t = torch.empty(shape, dtype=dt, device=device)
            else:
                _lib._expect(t, name, dt, shape)
            setattr(self, name, t)
        self.n_layers, self.n_kv_heads, self.head_dim = n_layers, n_kv_heads, head_dim
        self.n_pages, self.page_size = n_pages, page_size
        self.max_seqs, self.max_pages, self.dtype = max_seqs, max_pages, dtype
        dev = self.k.device
        self._gpu = self.k.get_device()
        _refuse(self._gpu, **{name: getattr(self, name) for name in want})
        self.status = torch.zeros(KV_MAX_REQUESTS, dtype=i32, device=dev)
        self.copied = torch.full((KV_MAX_REQUESTS, 2), -1, dtype=i32, device=dev)
        self.struct = _lib.KvCacheStruct(n_layers, n_kv_heads, head_dim, n_pages, page_size,
                                         max_seqs, max_pages, code,
                                         *[_lib._ptr(getattr(self, n))
                                           for n in ("k", "v", "table", "length", "refs")])
        self._ref = ctypes.byref(self.struct)
        self._lib = _lib.load()
        self._lock = threading.Lock()  # the launches of an operation before another's
        self._rotations = {}  # argument structs of append_rotated by what they hold
        self._status, self._copied = self.status.data_ptr(), self.copied.data_ptr()
        if fresh:
            self.clear()

    def clear(self, stream=None):
        """Every sequence empty, every page free."""
        with self._lock:
            _lib._check(self._lib.s2moe_kv_init(self._ref, _lib._stream(stream)))

    def fork(self, src, dst, stream=None):
        """Sequence dst[i] becomes a copy of src[i] on the same pages."""
        n = src.shape[0]
        ps, pd = _ints(src, "src", n), _ints(dst, "dst", n)
        if src.get_device() != self._gpu or dst.get_device() != self._gpu:
            _refuse(self._gpu, src=src, dst=dst)
        with self._lock:
            _lib._check(self._lib.s2moe_kv_fork(self._ref, n, ps, pd, self._status,
                                                _lib._stream(stream)))

    def reserve(self, seqs, extra, stream=None):
        """Pages for extra[i] more tokens of seqs[i]; a shared page that they
        would be written to is copied."""
        n = seqs.shape[0]
        ps, pe = _ints(seqs, "seqs", n), _ints(extra, "extra", n)
        if seqs.get_device() != self._gpu or extra.get_device() != self._gpu:
            _refuse(self._gpu, seqs=seqs, extra=extra)
        with self._lock:
            _lib._check(self._lib.s2moe_kv_reserve(self._ref, n, ps, pe, self._copied,
                                                   self._status, _lib._stream(stream)))

    def append(self, layer: int, k, v, seqs, tok_off, stream=None):
        """New tokens' keys and values [n_tokens, n_kv_heads, head_dim] into
        the slots after the lengths."""
        n = seqs.shape[0]
        kp, ldk, t = _rows(k, "k", self.n_kv_heads, self.head_dim, self.dtype)
        vp, ldv, tv = _rows(v, "v", self.n_kv_heads, self.head_dim, self.dtype)
        if tv != t:
            raise ValueError(f"v holds {tv} tokens, k {t}")
        ps, po = _ints(seqs, "seqs", n), _ints(tok_off, "tok_off", n + 1)
        g = self._gpu
        if not (g == k.get_device() == v.get_device() == seqs.get_device() == tok_off.get_device()):
            _refuse(g, k=k, v=v, seqs=seqs, tok_off=tok_off)
        _lib._check(self._lib.s2moe_kv_append(self._ref, layer, n, t, ps, po, kp, ldk, vp, ldv,
                                              _lib._stream(stream)))

    def positions(self, seqs, tok_off, n_tokens: int, parent=None, out=None, stream=None):
        """Positions [n_tokens] int32 of new tokens, once per step for all layers: the
        sequence's length plus the token's place among its new ones, or with `parent` plus
        its depth in the drafted tree."""
        n = seqs.shape[0]
        ps, po = _ints(seqs, "seqs", n), _ints(tok_off, "tok_off", n + 1)
        pp = None if parent is None else _ints(parent, "parent", n_tokens)
        g = self._gpu
        if not (g == seqs.get_device() == tok_off.get_device() == (g if parent is None else parent.get_device())):
            _refuse(g, seqs=seqs, tok_off=tok_off, **({} if parent is None else {"parent": parent}))
        handle = _lib._stream_on(g, stream, "the cache is")
        if out is None:
            out = _result(seqs, (n_tokens,), None if stream is None else _other(stream, seqs.device))
        po_out = _ints(out, "out", n_tokens)
        if out.get_device() != g:
            _refuse(g, out=out)
        _lib._check(self._lib.s2moe_kv_positions(self._ref, n, n_tokens, ps, po, pp, po_out,
                                                 handle))
        return out

    def append_rotated(self, layer: int, q, k, v, seqs, tok_off, pos, inv_freq,
                       neighbours: bool = False, out=None, k_out=None, stream=None):
        """append with queries q [n_tokens, n_heads, head_dim] and keys turned by the angles
        pos * inv_freq on the way; returns the turned queries.  inv_freq [rot_dim / 2]
        float32: the first rot_dim coordinates turn, pairs of neighbours or of halves.
        `out` takes the queries (q itself: in place), `k_out` the turned keys of every token
        (k itself: in place), as the prompts' own attention reads them."""
        n, Hkv, D, dt = seqs.shape[0], self.n_kv_heads, self.head_dim, self.dtype
        if q.dim() != 3:
            raise ValueError(f"q: expected [n_tokens, heads, {D}], got {tuple(q.shape)}")
        Hq = q.shape[1]
        qp, ldq, t = _rows(q, "q", Hq, D, dt)
        kp, ldk, tk = _rows(k, "k", Hkv, D, dt)
        vp, ldv, tv = _rows(v, "v", Hkv, D, dt)
        ps, po, pp = _ints(seqs, "seqs", n), _ints(tok_off, "tok_off", n + 1), _ints(pos, "pos", t)
        if inv_freq.dtype is not torch.float32 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
            raise ValueError(f"inv_freq: expected contiguous float32 [rot_dim / 2], got "
                             f"{inv_freq.dtype} {tuple(inv_freq.shape)}")
        g = self._gpu
        if not (g == q.get_device() == k.get_device() == v.get_device() == seqs.get_device()
                == tok_off.get_device() == pos.get_device() == inv_freq.get_device()):
            _refuse(g, q=q, k=k, v=v, seqs=seqs, tok_off=tok_off, pos=pos, inv_freq=inv_freq)
        handle = _lib._stream_on(g, stream, "the cache is")
        if out is None:
            out = _result(q, (t, Hq, D), None if stream is None else _other(stream, q.device))
            op, ldqo, to = out.data_ptr(), Hq * D, t
        else:
            op, ldqo, to = _rows(out, "out", Hq, D, dt)
            if out.get_device() != g:
                _refuse(g, out=out)
        kop, ldko, tko = None, 0, t
        if k_out is not None:
            kop, ldko, tko = _rows(k_out, "k_out", Hkv, D, dt)
            if k_out.get_device() != g:
                _refuse(g, k_out=k_out)
        if not (tk == tv == to == tko == t):
            raise ValueError(f"q, k, v, out, k_out hold {t}, {tk}, {tv}, {to}, {tko} tokens")
        key = (Hq, 2 * inv_freq.shape[0], int(neighbours), ldq, ldk, ldv, ldqo, ldko)
        r = self._rotations.get(key)  # of a model's layers all alike
        if r is None:
            r = ctypes.byref(_lib.Rotation(*key))
            if len(self._rotations) < 64:
                self._rotations[key] = r
        _lib._check(self._lib.s2moe_kv_append_rotated(
            self._ref, layer, r, n, t, ps, po, pp, inv_freq.data_ptr(), qp, kp, vp, op, kop,
            handle))
        return out

    def commit(self, seqs, path, n_accept, stream=None):
        """Keeps nodes path[i, :n_accept[i]] of each drafted tree (ascending);
        path None: the first n_accept[i] tokens as they lie."""
        n = seqs.shape[0]
        most = 0 if path is None else path.shape[1]
        pp = None
        if path is not None:
            _lib._expect(path, "path", _I32, (n, most))
            pp = _lib._ptr(path)
            if path.get_device() != self._gpu:
                _refuse(self._gpu, path=path)
        ps, pa = _ints(seqs, "seqs", n), _ints(n_accept, "n_accept", n)
        if seqs.get_device() != self._gpu or n_accept.get_device() != self._gpu:
            _refuse(self._gpu, seqs=seqs, n_accept=n_accept)
        with self._lock:
            _lib._check(self._lib.s2moe_kv_commit(self._ref, n, most, ps, pp, pa, self._status,
                                                  _lib._stream(stream)))

    def free(self, seqs, stream=None):
        """Empties the sequences."""
        n = seqs.shape[0]
        ps = _ints(seqs, "seqs", n)
        if seqs.get_device() != self._gpu:
            _refuse(self._gpu, seqs=seqs)
        with self._lock:
            _lib._check(self._lib.s2moe_kv_free(self._ref, n, ps, self._status,
                                                _lib._stream(stream)))


class TreeAttention:
    """Attention of drafted trees over `cache`, with the workspaces of calls of
    up to `max_seqs` sequences and `max_nodes` nodes each: one for every stream that
    calls come on, since the second launch of a call reads there what the first has
    left.  A call that a graph captures has memory of that graph's own, as its replay
    runs beside other calls.  Threads may share an object."""

    def __init__(self, cache: KVCache, n_heads: int, max_seqs: int, max_nodes: int,
                 scale: float | None = None):
        self.cache, self.n_heads = cache, n_heads
        self.max_seqs, self.max_nodes = max_seqs, max_nodes
        D = cache.head_dim
        self.scale = D ** -0.5 if scale is None else scale
        self.attn = self._strided(n_heads * D, n_heads * D)
        self._ref = ctypes.byref(self.attn)
        self._lib = _lib.load()
        self.bytes = self._lib.s2moe_tree_attention_workspace_bytes(cache._ref, self._ref,
                                                                    max_seqs, max_nodes)
        if self.bytes == 0:
            raise _lib.S2moeError(_lib.EINVAL, _lib.last_error())
        self.workspace = self._new_space()
        self._spaces = {_lib._stream(None): self.workspace}  # by stream handle
        self._lock = threading.Lock()  # both launches of a call before another's on its stream

    def _new_space(self):
        return torch.empty(self.bytes, dtype=torch.uint8, device=self.cache.k.device)

    def _space(self, handle, other):
        if other is not None:
            with torch.cuda.stream(other):
                return self._space(handle, None)
        if torch.cuda.is_current_stream_capturing():
            return self._new_space()
        space = self._spaces.get(handle)
        if space is None:
            space = self._spaces[handle] = self._new_space()
        return space

    def _strided(self, ldq, ldo):
        c = self.cache
        return _lib.Attn(self.n_heads, c.n_kv_heads, c.head_dim, c.struct.dtype, self.scale, ldq,
                         0, 0, ldo)

    def __call__(self, layer: int, q, seqs, tok_off, parent, out=None, stream=None):
        """q [n_tokens, n_heads, head_dim] -> out of the same shape."""
        c, n = self.cache, seqs.shape[0]
        if n > self.max_seqs:
            raise ValueError(f"{n} sequences, the workspace is for {self.max_seqs}")
        D, Hq = c.head_dim, self.n_heads
        qp, ldq, t = _rows(q, "q", Hq, D, c.dtype)
        ps, po = _ints(seqs, "seqs", n), _ints(tok_off, "tok_off", n + 1)
        pp = _ints(parent, "parent", t)
        g = c._gpu
        if not (g == q.get_device() == seqs.get_device() == tok_off.get_device() == parent.get_device()):
            _refuse(g, q=q, seqs=seqs, tok_off=tok_off, parent=parent)
        other = None if stream is None else _other(stream, q.device)
        if out is None:
            out = _result(q, (t, Hq, D), other)
            op, ldo = out.data_ptr(), Hq * D
        else:
            op, ldo, to = _rows(out, "out", Hq, D, c.dtype)
            if to != t:
                raise ValueError(f"out holds {to} tokens, q {t}")
            if out.get_device() != g:
                _refuse(g, out=out)
        # A struct of its own for other strides than those of whole rows: another thread
        # may be in a call with self.attn.
        ref = self._ref
        if ldq != Hq * D or ldo != Hq * D:
            ref = ctypes.byref(self._strided(ldq, ldo))
        handle = _lib._stream(stream)
        with self._lock:
            space = self._space(handle, other)
            _lib._check(self._lib.s2moe_tree_attention(
                c._ref, layer, ref, n, t, self.max_nodes, qp, ps, po, pp, space.data_ptr(),
                self.bytes, op, handle))
        return out


def prompt_attention(q, k, v, tok_off, out=None, scale: float | None = None, stream=None):
    """Causal attention within packed prompts: q [n_tokens, n_heads, head_dim],
    k and v [n_tokens, n_kv_heads, head_dim], tok_off [n + 1] int32."""
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError("q, k, v: expected [n_tokens, heads, head_dim]")
    Hq, D, Hkv, dt = q.shape[1], q.shape[2], k.shape[1], q.dtype
    code = _code(dt)
    qp, ldq, t = _rows(q, "q", Hq, D, dt)
    kp, ldk, tk = _rows(k, "k", Hkv, D, dt)
    vp, ldv, tv = _rows(v, "v", Hkv, D, dt)
    op, ldo, to = (None, Hq * D, t) if out is None else _rows(out, "out", Hq, D, dt)
    if not (tk == tv == to == t):
        raise ValueError(f"q, k, v, out hold {t}, {tk}, {tv}, {to} tokens")
    if tok_off.dim() != 1 or tok_off.shape[0] < 1:
        raise ValueError("tok_off: expected int32 [n + 1]")
    n = tok_off.shape[0] - 1
    po = _ints(tok_off, "tok_off", n + 1)
    g = q.get_device()
    if g < 0 or not g == k.get_device() == v.get_device() == tok_off.get_device():
        _refuse(g, q=q, k=k, v=v, tok_off=tok_off)
    if out is None:
        out = _result(q, (t, Hq, D), None if stream is None else _other(stream, q.device))
        op = out.data_ptr()
    elif out.get_device() != g:
        _refuse(g, out=out)
    a = _lib.Attn(Hq, Hkv, D, code, D ** -0.5 if scale is None else scale, ldq, ldk, ldv, ldo)
    _lib._check(_lib.load().s2moe_prompt_attention(ctypes.byref(a), n, t, qp, kp, vp, po, op,
                                                   _lib._stream(stream)))
    return out
