"""The dense half of a layer: the norm before each half, and projections in 8-bit floating
point with a scale for each block of 128.  Argument marshalling only; every step is a call
into libs2moe.so.

    w = quantize_weight(w_qkv)                                     # once, at load
    x8 = add_norm(y, norm_weight, residual, out_dtype=E4M3)        # residual += y; its norm
    qkv = fp8_matmul(x8, w)
    ...                                                            # rotation, attention
    y = fp8_matmul(quantize(attention_out), w_out)

Calls are made with the tensors' GPU current.  With `stream`, the inputs have to be ready
there, and kept (or recorded on it) until it is done with them; results are allocated on it.
"""

from __future__ import annotations

from typing import NamedTuple

import torch

from . import _lib
from .attention import _other, _refuse

E4M3 = torch.float8_e4m3fn
BLOCK = 128  # elements of a row that share a scale
_CODES = {torch.float32: _lib.F32, torch.bfloat16: _lib.BF16, E4M3: _lib.E4M3}
_F32 = torch.float32


class Fp8Rows(NamedTuple):
    """Rows in 8 bits: element j of row i is codes[i, j] * scales[j // 128, i]."""
    codes: torch.Tensor   # [n, cols] float8_e4m3fn
    scales: torch.Tensor  # [ceil(cols / 128), n] float32


class Fp8Weight(NamedTuple):
    """Weights in 8 bits: element j of row i is codes[i, j] * scales[i // 128, j // 128]."""
    codes: torch.Tensor   # [n, k] float8_e4m3fn
    scales: torch.Tensor  # [ceil(n / 128), ceil(k / 128)] float32


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


# The checks are on every call's path to the GPU, which at the smallest sizes waits for
# them: each property is read once, and results made here are not looked at.
def _matrix(t, name, rows=None, cols=None):
    """(pointer, elements from one row to the next, rows, columns) of a matrix whose
    rows lie together."""
    shape = t.shape
    if len(shape) != 2 or (rows is not None and shape[0] != rows) or (cols is not None and shape[1] != cols):
        want = f"[{'n' if rows is None else rows}, {'columns' if cols is None else cols}]"
        raise ValueError(f"{name}: expected {want}, got {tuple(shape)}")
    s0, s1 = t.stride()
    n, c = shape
    if s1 != 1 and c > 1:
        raise ValueError(f"{name}: the elements of a row must lie together (strides {t.stride()})")
    return t.data_ptr(), s0 if n > 1 else c, n, c


def _float(t, name):
    code = _CODES.get(t.dtype)
    if code is None or code == _lib.E4M3:
        raise TypeError(f"{name}: expected torch.float32 or torch.bfloat16, got {t.dtype}")
    return code


def _of(t, name, dtype):
    if t.dtype is not dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")


def _empty(like, stream, shape, dtype):
    """A tensor for what `stream` writes, from its pool."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    other = _other(stream, like.device)
    if other is None:
        return like.new_empty(shape, dtype=dtype)
    with torch.cuda.stream(other):
        out = like.new_empty(shape, dtype=dtype)
    out.record_stream(torch.cuda.current_stream())
    return out


def _rows_out(out, like, n, cols, gpu, stream):
    """(Fp8Rows, pointer and stride of its codes, of its scales); made if out is None."""
    kb = (cols + BLOCK - 1) // BLOCK
    if out is None:
        codes, scales = _empty(like, stream, (n, cols), E4M3), _empty(like, stream, (kb, n), _F32)
        return Fp8Rows(codes, scales), codes.data_ptr(), cols, scales.data_ptr(), n
    codes, scales = out
    _of(codes, "codes", E4M3)
    _of(scales, "scales", _F32)
    cp, ldc, _, _ = _matrix(codes, "codes", n, cols)
    sp, lds, _, _ = _matrix(scales, "scales", kb, n)
    if not gpu == codes.get_device() == scales.get_device():
        _refuse(gpu, codes=codes, scales=scales)
    return out, cp, ldc, sp, lds


def add_norm(x, weight, residual=None, eps: float = 1e-6, out=None, out_dtype=None, stream=None):
    """h = x + residual, residual <- h (in place), and h * weight / sqrt(mean(h^2) + eps)
    of rows x [n, hidden]; float32 or bfloat16 each by itself.  out_dtype (x's by default):
    float32, bfloat16, or torch.float8_e4m3fn, which gives Fp8Rows.  `out` takes the result
    where it is given: a tensor, or Fp8Rows."""
    xp, ldx, n, H = _matrix(x, "x")
    if out is not None:
        given = E4M3 if isinstance(out, tuple) else out.dtype
        if out_dtype is not None and out_dtype is not given:
            raise TypeError(f"out is {given}, out_dtype {out_dtype}")
        out_dtype = given
    dt = x.dtype if out_dtype is None else out_dtype
    xc, wc, oc = _float(x, "x"), _float(weight, "weight"), _CODES.get(dt)
    if oc is None or (oc == _lib.E4M3 and isinstance(out, torch.Tensor)):
        raise TypeError(f"out: expected float32, bfloat16 or Fp8Rows, got {dt}")
    if weight.dim() != 1 or weight.shape[0] != H or not weight.is_contiguous():
        raise ValueError(f"weight: expected contiguous [{H}], got {tuple(weight.shape)}")
    gpu = x.get_device()
    if gpu < 0 or weight.get_device() != gpu:
        _refuse(gpu, x=x, weight=weight)
    rp, ldr, rc = None, 0, 0
    if residual is not None:
        rc = _float(residual, "residual")
        rp, ldr, _, _ = _matrix(residual, "residual", n, H)
        if residual.get_device() != gpu:
            _refuse(gpu, residual=residual)
    handle = _lib._stream_on(gpu, stream, "the tensors are")
    if oc == _lib.E4M3:
        out, op, ldo, sp, lds = _rows_out(out, x, n, H, gpu, stream)
    elif out is None:
        out, ldo, sp, lds = _empty(x, stream, (n, H), dt), H, None, 0
        op = out.data_ptr()
    else:
        op, ldo, _, _ = _matrix(out, "out", n, H)
        sp, lds = None, 0
        if out.get_device() != gpu:
            _refuse(gpu, out=out)
    _lib._check(_lib.load().s2moe_add_norm(n, H, xp, ldx, xc, rp, ldr, rc, weight.data_ptr(), wc,
                                           eps, op, ldo, oc, sp, lds, handle))
    return out


def quantize(x, out=None, stream=None) -> Fp8Rows:
    """Rows x [n, cols] (float32 or bfloat16) in 8 bits."""
    xc = _float(x, "x")
    xp, ldx, n, K = _matrix(x, "x")
    gpu = x.get_device()
    if gpu < 0:
        _refuse(gpu, x=x)
    handle = _lib._stream_on(gpu, stream, "the tensors are")
    out, cp, ldc, sp, lds = _rows_out(out, x, n, K, gpu, stream)
    _lib._check(_lib.load().s2moe_quantize(n, K, xp, ldx, xc, cp, ldc, sp, lds, handle))
    return out


def quantize_weight(w, stream=None) -> Fp8Weight:
    """Weights w [n, k] (float32 or bfloat16) in 8 bits, once at model load."""
    wc = _float(w, "w")
    wp, ldw, n, K = _matrix(w, "w")
    gpu, nb, kb = w.get_device(), _blocks(n), _blocks(K)
    if gpu < 0:
        _refuse(gpu, w=w)
    handle = _lib._stream_on(gpu, stream, "the tensors are")
    out = Fp8Weight(_empty(w, stream, (n, K), E4M3), _empty(w, stream, (nb, kb), _F32))
    _lib._check(_lib.load().s2moe_quantize_weight(n, K, wp, ldw, wc, out.codes.data_ptr(), K,
                                                  out.scales.data_ptr(), kb, handle))
    return out


def fp8_matmul(x: Fp8Rows, w: Fp8Weight, out=None, out_dtype=None, stream=None):
    """x [m, k] times the transpose of w [n, k]: [m, n] in out_dtype (torch.bfloat16 by
    default, or torch.float32).  Sums that cancel keep their precision in float32 only: for
    bfloat16 results products are cut off 13 bits below the largest of eight neighbours."""
    xc, xs = x
    wc, ws = w
    _of(xc, "x.codes", E4M3)
    _of(wc, "w.codes", E4M3)
    _of(xs, "x.scales", _F32)
    _of(ws, "w.scales", _F32)
    xp, ldx, m, K = _matrix(xc, "x.codes")
    wp, ldw, n, _ = _matrix(wc, "w.codes", None, K)
    kb = (K + BLOCK - 1) // BLOCK
    xsp, ldxs, _, _ = _matrix(xs, "x.scales", kb, m)
    wsp, ldws, _, _ = _matrix(ws, "w.scales", (n + BLOCK - 1) // BLOCK, kb)
    gpu = xc.get_device()
    if gpu < 0 or not gpu == xs.get_device() == wc.get_device() == ws.get_device():
        _refuse(gpu, x=xc, x_scales=xs, w=wc, w_scales=ws)
    handle = _lib._stream_on(gpu, stream, "the tensors are")
    if out is None:
        dt = torch.bfloat16 if out_dtype is None else out_dtype
        oc = _CODES.get(dt)
        if oc is None or oc == _lib.E4M3:
            raise TypeError(f"out_dtype: expected torch.float32 or torch.bfloat16, got {dt}")
        out, ldo = _empty(xc, stream, (m, n), dt), n
        op = out.data_ptr()
    else:
        if out_dtype is not None and out.dtype is not out_dtype:
            raise TypeError(f"out is {out.dtype}, out_dtype {out_dtype}")
        oc = _float(out, "out")
        op, ldo, _, _ = _matrix(out, "out", m, n)
        if out.get_device() != gpu:
            _refuse(gpu, out=out)
    _lib._check(_lib.load().s2moe_scaled_matmul(m, n, K, xp, ldx, xsp, ldxs, wp, ldw, wsp, ldws, op, ldo,
                                                oc, handle))
    return out
