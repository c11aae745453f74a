"""The dense half of a layer in 64 bits: the norm, 8-bit rows and weights, their products,
positions and rotation.  numpy only; nothing is shared with the GPU path."""

from __future__ import annotations

import numpy as np

BLOCK, LARGEST, LEAST = 128, 448.0, 2.0 ** -100


def _e4m3_values():
    """The number each code stands for: sign, four exponent bits (bias 7), three mantissa
    bits; exponent 0 without the leading one; all ones NaN."""
    v = np.empty(256)
    for c in range(256):
        e, f = c >> 3 & 15, c & 7
        x = f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7)
        v[c] = np.nan if c & 127 == 127 else (-x if c & 128 else x)
    return v


E4M3 = _e4m3_values()


def half_step(z):
    """Half the distance of e4m3's numbers about z: how far a rounding may be off."""
    e = np.floor(np.log2(np.maximum(np.abs(z), 2.0 ** -6)))
    return 2.0 ** (e - 4)


def blocks_of(n):
    return -(-n // BLOCK)


def row_scales(y):
    """[blocks, rows]: each block's largest magnitude / 448."""
    return np.stack([np.maximum(np.abs(y[:, k:k + BLOCK]).max(1), LEAST) / LARGEST
                     for k in range(0, y.shape[1], BLOCK)])


def spread_rows(scales, cols):
    """Row scales as a factor of each element [rows, cols]."""
    return np.repeat(scales.T, BLOCK, axis=1)[:, :cols]


def weight_scales(w):
    return np.array([[max(np.abs(w[i:i + BLOCK, k:k + BLOCK]).max(), LEAST) / LARGEST
                      for k in range(0, w.shape[1], BLOCK)] for i in range(0, w.shape[0], BLOCK)])


def spread_weight(scales, rows, cols):
    return np.repeat(np.repeat(scales, BLOCK, axis=0)[:rows], BLOCK, axis=1)[:, :cols]


def add_norm(x, residual, weight, eps):
    """(h, y)."""
    h = x if residual is None else x + residual
    return h, h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * weight


def scaled_matmul(x, xs, w, ws):
    """(the product, the sum of its terms' magnitudes), of codes' values and scales."""
    k = x.shape[1]
    a, b = x * spread_rows(xs, k), w * spread_weight(ws, w.shape[0], k)
    return a @ b.T, np.abs(a) @ np.abs(b).T


def cut_off(x, xs, w, ws):
    """How far the 8-bit matrix instruction may be off: it cuts each of eight neighbouring
    products off, towards zero, 13 bits below the largest sum of two exponents among them
    (those of numbers below 2^-6 count as -6)."""
    k = x.shape[1]
    ex, ew = (np.where(t == 0, -100.0, np.floor(np.log2(np.maximum(np.abs(t), 2.0 ** -6)))) for t in (x, w))
    a, b = spread_rows(xs, k), spread_weight(ws, w.shape[0], k)
    off = np.zeros((x.shape[0], w.shape[0]))
    for g in range(0, k, 8):
        top = np.full(off.shape, -200.0)
        for i in range(g, g + 8):
            np.maximum(top, ex[:, i, None] + ew[None, :, i], out=top)
        off += 8 * np.exp2(top - 13) * a[:, g, None] * b[None, :, g]
    return off


def positions(lengths, counts, parent=None):
    """Of packed tokens; parent a packed list, or None for tokens one after another."""
    out, at = [], 0
    for n, c in zip(lengths, counts):
        depth = []
        for i in range(c):
            p = i - 1 if parent is None else parent[at + i]
            depth.append(depth[p] + 1 if 0 <= p < i else 0)
        out += [n + d for d in depth]
        at += c
    return np.array(out, dtype=np.int64)


def rotate(x, pos, freq, neighbours):
    """x [tokens, heads, D] with its first 2 len(freq) coordinates turned, and for each
    element the sum of the magnitudes of the two products it is made of.  Angles in 80
    bits, where the product of an int32 and an fp32 number is exact."""
    x = np.asarray(x, dtype=np.float64)
    half = len(freq)
    angle = np.asarray(pos, dtype=np.longdouble)[:, None] * np.asarray(freq, dtype=np.longdouble)
    c, s = (f(angle).astype(np.float64)[:, None] for f in (np.cos, np.sin))
    a, b = ((slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if neighbours
            else (slice(0, half), slice(half, 2 * half)))
    y, size = x.copy(), np.abs(x)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size
