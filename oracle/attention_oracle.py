"""Plain definition of the cache and attention operators: fp64 attention by
explicit sets of visible tokens, and a cache whose page operations run one
request after another on host arrays.

Pools are held as the caller lays them out: k [L, page, head, slot, D] and
v [L, page, head, slot / 8, D, slot % 8].
"""

from __future__ import annotations

import numpy as np

NO_PAGES, TOO_LONG, BAD_SEQ, BUSY, BAD_PATH = 1, 2, 4, 8, 16


def attend(q, k, v, visible, scale):
    """One query [D] over the visible rows of k, v [m, D], fp64."""
    idx = np.nonzero(visible)[0]
    if len(idx) == 0:
        return np.zeros(v.shape[1])
    s = scale * (k[idx] @ q)
    p = np.exp(s - s.max())
    return (p @ v[idx]) / p.sum()


def tree_visible(parent):
    """[T, T]: node j is node i or an ancestor of i; a node that hangs, at
    whatever remove, below an invalid parent sees nothing."""
    T = len(parent)
    seen = np.zeros((T, T), dtype=bool)
    valid = np.zeros(T, dtype=bool)
    for i, p in enumerate(parent):
        if p == -1:
            valid[i] = True
        elif 0 <= p < i and valid[p]:
            valid[i] = True
            seen[i] = seen[p]
        if valid[i]:
            seen[i, i] = True
    return seen, valid


def tree_attention(q, k, v, length, parent, scale):
    """q [T, Hq, D] over one sequence's k, v [length + T, Hkv, D]."""
    T, Hq, D = q.shape
    G = Hq // k.shape[1]
    seen, valid = tree_visible(parent)
    out = np.zeros((T, Hq, D))
    for i in range(T):
        if not valid[i]:
            continue
        vis = np.concatenate([np.ones(length, dtype=bool), seen[i]])
        for h in range(Hq):
            out[i, h] = attend(q[i, h], k[:, h // G], v[:, h // G], vis, scale)
    return out


def prompt_attention(q, k, v, tok_off, scale):
    """Packed prompts: q [n, Hq, D], k, v [n, Hkv, D]."""
    out = np.zeros(q.shape)
    G = q.shape[1] // k.shape[1]
    for a, b in zip(tok_off[:-1], tok_off[1:]):
        if b <= a:
            continue
        mask = np.tril(np.ones((b - a, b - a), dtype=bool))
        for h in range(q.shape[1]):
            s = scale * (q[a:b, h] @ k[a:b, h // G].T)
            s = np.where(mask, s, -np.inf)
            p = np.exp(s - s.max(axis=1, keepdims=True))
            out[a:b, h] = (p @ v[a:b, h // G]) / p.sum(axis=1, keepdims=True)
    return out


class Cache:
    """Host copy of a cache; every method returns the requests' status."""

    def __init__(self, k, v, table, length, refs):
        self.k, self.v = k.copy(), v.copy()
        self.table, self.length, self.refs = table.copy(), length.copy(), refs.copy()
        self.P = k.shape[3]

    def _known(self, seqs, i):
        s = int(seqs[i])
        return 0 <= s < len(self.length) and s not in [int(x) for x in seqs[:i]]

    def held(self, s):
        return int((self.table[s] >= 0).sum())

    def _drop(self, s, first):
        for j in range(first, self.table.shape[1]):
            p = self.table[s, j]
            if p >= 0:
                self.refs[p] -= 1
                self.table[s, j] = -1

    def fork(self, src, dst):
        status = []
        targets = {int(x) for x in dst}
        for i in range(len(src)):
            a, b = int(src[i]), int(dst[i])
            if not (0 <= a < len(self.length)) or not self._known(dst, i) or a in targets:
                status.append(BAD_SEQ)
            elif self.length[b] != 0 or self.held(b):
                status.append(BUSY)
            else:
                n = -(-int(self.length[a]) // self.P)
                self.table[b, :n] = self.table[a, :n]
                for p in self.table[a, :n]:
                    self.refs[p] += 1
                self.length[b] = self.length[a]
                status.append(0)
        return status

    def reserve(self, seqs, extra):
        """(status, copied pages)."""
        n, status, want = len(seqs), [], []
        sharers = {}
        for i in range(n):
            s, e = int(seqs[i]), int(extra[i])
            if not self._known(seqs, i):
                status.append(BAD_SEQ)
                want.append(None)
                continue
            length = int(self.length[s])
            if e < 0 or length + e > self.table.shape[1] * self.P:
                status.append(TOO_LONG)
                want.append(None)
                continue
            new = max(0, -(-(length + e) // self.P) - self.held(s))
            shared = copy = None
            if e > 0 and length % self.P:
                p = int(self.table[s, length // self.P])
                if self.refs[p] > 1:
                    shared = p
                    rank = sharers.get(p, 0)
                    sharers[p] = rank + 1
                    copy = p if self.refs[p] - rank > 1 else None
            status.append(0)
            want.append((new, copy, shared))
        free = [p for p in range(len(self.refs)) if self.refs[p] == 0]
        copied = np.full((n, 2), -1, dtype=np.int32)
        used, room = 0, len(free)
        stay = set()  # shared pages whose copy was refused: the sharer holds them still
        for i in range(n):
            if want[i] is None:
                continue
            new, copy, shared = want[i]
            take = new + (copy is not None)
            used += take
            if (take and used > room) or shared in stay:
                status[i] = NO_PAGES
                if copy is not None:
                    stay.add(copy)
                continue
            if take == 0:
                continue
            mine = free[used - take:used]
            s = int(seqs[i])
            length = int(self.length[s])
            if copy is not None:
                to = mine.pop(0)
                n8 = (length % self.P + 7) // 8
                self.k[:, to, :, :8 * n8] = self.k[:, copy, :, :8 * n8]
                self.v[:, to, :, :n8] = self.v[:, copy, :, :n8]
                self.table[s, length // self.P] = to
                self.refs[copy] -= 1
                self.refs[to] = 1
                copied[i] = (copy, to)
            h = self.held(s)
            for j, p in enumerate(mine):
                self.table[s, h + j] = p
                self.refs[p] = 1
        return status, copied

    def own_slot(self, s, pos):
        """slot() where the sequence holds the page alone, else None."""
        at = self.slot(s, pos)
        return at if at is not None and self.refs[at[0]] == 1 else None

    def slot(self, s, pos):
        """(page, slot) of a token, or None where the sequence has no page."""
        if pos // self.P >= self.table.shape[1]:
            return None
        p = int(self.table[s, pos // self.P])
        return None if p < 0 else (p, pos % self.P)

    def append(self, layer, k, v, seqs, tok_off):
        for i, s in enumerate(seqs):
            for j in range(int(tok_off[i + 1]) - int(tok_off[i])):
                at = self.own_slot(s, int(self.length[s]) + j)
                if at is None:
                    continue
                p, x = at
                self.k[layer, p, :, x] = k[tok_off[i] + j]
                self.v[layer, p, :, x // 8, :, x % 8] = v[tok_off[i] + j]

    def commit(self, seqs, path, n_accept):
        status = []
        for i in range(len(seqs)):
            s, acc = int(seqs[i]), int(n_accept[i])
            if not self._known(seqs, i):
                status.append(BAD_SEQ)
                continue
            length = int(self.length[s])
            nodes = list(range(acc)) if path is None else [int(x) for x in path[i][:max(acc, 0)]]
            ok = acc >= 0 and len(nodes) == acc
            ok = ok and all(a < b for a, b in zip([-1] + nodes, nodes))
            ok = ok and all(self.own_slot(s, length + x) is not None
                            for j, p in enumerate(nodes) for x in (p, j))
            if not ok:
                status.append(BAD_PATH)
                continue
            for j, p in enumerate(nodes):
                (pa, xa), (pb, xb) = self.slot(s, length + p), self.slot(s, length + j)
                self.k[:, pb, :, xb] = self.k[:, pa, :, xa]
                self.v[:, pb, :, xb // 8, :, xb % 8] = self.v[:, pa, :, xa // 8, :, xa % 8]
            self.length[s] = length + acc
            self._drop(s, -(-(length + acc) // self.P))
            status.append(0)
        return status

    def free(self, seqs):
        status = []
        for i in range(len(seqs)):
            if not self._known(seqs, i):
                status.append(BAD_SEQ)
                continue
            self._drop(int(seqs[i]), 0)
            self.length[int(seqs[i])] = 0
            status.append(0)
        return status

    def tokens(self, layer, s, n):
        """k, v [n, Hkv, D] of a sequence's first n slots."""
        at = [self.slot(s, j) for j in range(n)]
        if n == 0:
            return np.zeros((0,) + self.k.shape[2:3] + self.k.shape[4:]), \
                np.zeros((0,) + self.k.shape[2:3] + self.k.shape[4:])
        return (np.stack([self.k[layer, p, :, x] for p, x in at]),
                np.stack([self.v[layer, p, :, x // 8, :, x % 8] for p, x in at]))
