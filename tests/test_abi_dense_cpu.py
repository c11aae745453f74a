"""Host checks of the dense half's entry points, positions and the append with rotation:
malformed arguments are refused before anything is enqueued (no kernel is launched by these
tests)."""

import ctypes

import pytest

import paper_2608_15018_amd as s2
from paper_2608_15018_amd import _lib

# Aligned fake addresses, far apart; every call below fails or does nothing.
A, B, C, D, E = (i << 40 for i in range(1, 6))
F32, BF16, Q4, E4M3 = _lib.F32, _lib.BF16, _lib.Q4G32, _lib.E4M3
INVAL, UNSUP = _lib.EINVAL, _lib.EUNSUPPORTED
BIG = 1 << 22


@pytest.fixture(scope="module")
def lib():
    return s2.load()


def refuse(call, cases):
    for kw, status, needle in cases:
        assert call(**kw) == status, (kw, _lib.last_error())
        assert needle in _lib.last_error(), (kw, _lib.last_error())


def test_add_norm(lib):
    def call(n=4, H=256, x=A, ldx=256, xt=BF16, r=B, ldr=256, rt=F32, w=C, wt=BF16, eps=1e-6, out=D, ldo=256, ot=E4M3, sc=E, lds=4):
        return lib.s2moe_add_norm(n, H, x, ldx, xt, r, ldr, rt, w, wt, eps, out, ldo, ot, sc, lds, None)

    refuse(call, [
        (dict(n=-1), INVAL, "n = "), (dict(n=BIG + 1), UNSUP, "n = "), (dict(H=0), INVAL, "hidden"), (dict(H=-16), INVAL, "hidden"),
        (dict(H=24), INVAL, "hidden"), (dict(H=16400), UNSUP, "hidden"), (dict(xt=E4M3), INVAL, "x_dtype"), (dict(xt=Q4), INVAL, "x_dtype"),
        (dict(wt=7), INVAL, "w_dtype"), (dict(rt=E4M3), INVAL, "r_dtype"), (dict(ot=Q4), INVAL, "out_dtype"), (dict(ot=-1), INVAL, "out_dtype"),
        (dict(eps=0.0), INVAL, "eps"), (dict(eps=-1.0), INVAL, "eps"), (dict(eps=float("nan")), INVAL, "eps"), (dict(eps=float("inf")), INVAL, "eps"),
        (dict(x=None), INVAL, "x is NULL"), (dict(x=A + 8), INVAL, "x is not"), (dict(w=None), INVAL, "weight"), (dict(w=C + 2), INVAL, "weight"),
        (dict(out=None), INVAL, "out is"), (dict(out=D + 4), INVAL, "out is"), (dict(r=B + 8), INVAL, "residual is not"),
        (dict(sc=None), INVAL, "scales"), (dict(sc=E + 2), INVAL, "scales"), (dict(lds=3), INVAL, "lds"), (dict(ldx=255), INVAL, "ldx"),
        (dict(ldx=260), INVAL, "ldx"), (dict(ldx=BIG + 16), UNSUP, "ldx"), (dict(ldr=257), INVAL, "ldr"), (dict(ldo=264), INVAL, "ldo"),
        (dict(ldo=128), INVAL, "ldo"), (dict(out=A), INVAL, "out overlaps x"), (dict(out=A + 3 * 512 + 496), INVAL, "out overlaps x"),
        (dict(out=C), INVAL, "weight"), (dict(sc=A), INVAL, "scales overlap"), (dict(sc=D + 4 * 256 - 4), INVAL, "scales overlap"),
        (dict(sc=C), INVAL, "scales overlap"), (dict(r=A), INVAL, "residual overlaps"), (dict(r=D), INVAL, "residual overlaps"),
        (dict(r=C), INVAL, "residual overlaps"), (dict(r=E), INVAL, "residual overlaps")])
    assert call(n=0) == _lib.OK and call(n=0, x=None, out=None, sc=None) == _lib.OK
    # Without a residual its type and stride do not matter; columns of one array lie side by side.
    assert call(r=None, rt=9, ldr=0, out=None) == INVAL and "out is" in _lib.last_error()
    assert call(ot=BF16, ldo=512, ldx=512, out=A + 512, r=A + 256) == INVAL and "residual overlaps" in _lib.last_error()


def test_quantize(lib):
    def call(n=4, K=256, x=A, ldx=256, xt=F32, c=B, ldc=256, sc=C, lds=4):
        return lib.s2moe_quantize(n, K, x, ldx, xt, c, ldc, sc, lds, None)

    refuse(call, [
        (dict(n=-1), INVAL, "n = "), (dict(n=BIG + 1), UNSUP, "n = "), (dict(K=0), INVAL, "cols"), (dict(K=100), INVAL, "cols"),
        (dict(K=(1 << 18) + 16), UNSUP, "cols"), (dict(xt=E4M3), INVAL, "x_dtype"), (dict(x=None), INVAL, "x is"), (dict(c=None), INVAL, "codes"),
        (dict(c=B + 8), INVAL, "codes"), (dict(sc=None), INVAL, "scales"), (dict(ldx=254), INVAL, "ldx"), (dict(ldc=264), INVAL, "ldc"),
        (dict(lds=3), INVAL, "lds"), (dict(c=A), INVAL, "overlap"), (dict(sc=A + 4 * 1024 - 4), INVAL, "overlap"), (dict(sc=B), INVAL, "overlap")])
    assert call(n=0) == _lib.OK


def test_quantize_weight(lib):
    def call(n=300, K=256, x=A, ldx=256, xt=F32, c=B, ldc=256, sc=C, lds=2):
        return lib.s2moe_quantize_weight(n, K, x, ldx, xt, c, ldc, sc, lds, None)

    refuse(call, [
        (dict(n=0), INVAL, "rows"), (dict(n=BIG + 1), UNSUP, "rows"), (dict(K=8), INVAL, "cols"), (dict(xt=E4M3), INVAL, "w_dtype"),
        (dict(x=None), INVAL, "w is"), (dict(c=B + 1), INVAL, "codes"), (dict(sc=None), INVAL, "scales"), (dict(ldx=252), INVAL, "ldw"),
        (dict(ldc=255), INVAL, "ldc"), (dict(lds=1), INVAL, "lds"), (dict(c=A + 4096), INVAL, "overlap"), (dict(sc=B + 256), INVAL, "overlap")])


def test_scaled_matmul(lib):
    def call(m=4, n=300, k=400, x=A, ldx=400, xs=B, ldxs=4, w=C, ldw=400, ws=D, ldws=4, out=E, ldo=300, ot=BF16):
        return lib.s2moe_scaled_matmul(m, n, k, x, ldx, xs, ldxs, w, ldw, ws, ldws, out, ldo, ot, None)

    refuse(call, [
        (dict(m=-1), INVAL, "m = "), (dict(m=BIG + 1), UNSUP, "m = "), (dict(n=0), INVAL, "n = "), (dict(n=BIG + 1), UNSUP, "n = "),
        (dict(k=0), INVAL, "k = "), (dict(k=40), INVAL, "k = "), (dict(k=(1 << 18) + 16), UNSUP, "k = "),
        (dict(m=BIG, n=BIG), UNSUP, "2^34"), (dict(m=1 << 17, n=(1 << 17) + 1), UNSUP, "2^34"),
        (dict(ot=E4M3), INVAL, "out_dtype"), (dict(x=None), INVAL, "x is"), (dict(x=A + 8), INVAL, "x is"), (dict(w=None), INVAL, "w is"),
        (dict(xs=None), INVAL, "x_scales"), (dict(xs=B + 2), INVAL, "x_scales"), (dict(ws=None), INVAL, "w_scales"), (dict(out=None), INVAL, "out is"),
        (dict(out=E + 2), INVAL, "out is"), (dict(ldx=392), INVAL, "ldx"), (dict(ldx=408), INVAL, "ldx"), (dict(ldxs=3), INVAL, "ldxs"),
        (dict(ldw=399), INVAL, "ldw"), (dict(ldws=3), INVAL, "ldws"), (dict(ldo=299), INVAL, "ldo"), (dict(ldo=BIG + 1), UNSUP, "ldo"),
        (dict(out=A), INVAL, "overlaps"), (dict(out=B), INVAL, "overlaps"), (dict(out=C + 299 * 400), INVAL, "overlaps"), (dict(out=D), INVAL, "overlaps")])
    assert call(m=0) == _lib.OK and call(m=0, x=None) == _lib.OK


def cache(**kw):
    d = dict(n_layers=2, n_kv_heads=2, head_dim=64, n_pages=8, page_size=16, max_seqs=4, max_pages=4, dtype=BF16, k=A, v=A, table=A,
             length=A, refs=A)
    d.update(kw)
    return _lib.KvCacheStruct(**d)


def test_positions(lib):
    c = cache()

    def call(c=c, n=2, t=9, seqs=A, off=B, par=C, pos=D):
        return lib.s2moe_kv_positions(ctypes.byref(c) if c else None, n, t, seqs, off, par, pos, None)

    refuse(call, [
        (dict(c=None), INVAL, "cache is NULL"), (dict(c=cache(head_dim=96)), UNSUP, "head_dim"), (dict(n=-1), INVAL, "n = "),
        (dict(n=1025), UNSUP, "n = "), (dict(t=-1), INVAL, "n_tokens"), (dict(t=(1 << 28) + 1), UNSUP, "n_tokens"),
        (dict(seqs=None), INVAL, "seqs"), (dict(off=B + 2), INVAL, "tok_off"), (dict(par=C + 1), INVAL, "parent"), (dict(pos=None), INVAL, "pos"),
        (dict(pos=D + 2), INVAL, "pos"), (dict(pos=C), INVAL, "overlaps"), (dict(pos=C + 32), INVAL, "overlaps"), (dict(pos=A + 4), INVAL, "overlaps"),
        (dict(pos=B + 8), INVAL, "overlaps")])
    assert call(n=0) == _lib.OK and call(t=0) == _lib.OK


def test_append_rotated(lib):
    c = cache()
    rot = lambda **kw: _lib.Rotation(**dict(dict(n_heads=4, rot_dim=64, neighbours=0, ldq=512, ldk=512, ldv=512, ldqo=256, ldko=128), **kw))  # noqa: E731
    # A fused projection's output: 4 query heads, 2 key heads, 2 value heads of 64 in rows of 512.
    Q, K, V = A, A + 512, A + 768

    def call(c=c, layer=0, r=None, n=2, t=9, seqs=B, off=B, pos=B, f=B, q=Q, k=K, v=V, qo=C, ko=D, null=False):
        r = r or rot()
        return lib.s2moe_kv_append_rotated(ctypes.byref(c), layer, None if null else ctypes.byref(r), n, t, seqs, off, pos, f, q, k, v, qo, ko, None)

    refuse(call, [
        (dict(c=cache(dtype=2)), INVAL, "dtype"), (dict(layer=2), INVAL, "layer"), (dict(layer=-1), INVAL, "layer"), (dict(n=-1), INVAL, "n = "),
        (dict(n=1025), UNSUP, "n = "), (dict(t=-1), INVAL, "n_tokens"), (dict(t=(1 << 28) + 1), UNSUP, "n_tokens"), (dict(null=True), INVAL, "rotation"),
        (dict(r=rot(n_heads=0)), INVAL, "n_heads"), (dict(r=rot(n_heads=1025)), UNSUP, "n_heads"), (dict(r=rot(rot_dim=0)), INVAL, "rot_dim"),
        (dict(r=rot(rot_dim=40)), INVAL, "rot_dim"), (dict(r=rot(rot_dim=80)), INVAL, "rot_dim"), (dict(r=rot(neighbours=2)), INVAL, "neighbours"),
        (dict(seqs=None), INVAL, "seqs"), (dict(off=None), INVAL, "tok_off"), (dict(pos=B + 1), INVAL, "pos"), (dict(f=None), INVAL, "inv_freq"),
        (dict(q=None), INVAL, "q is"), (dict(k=K + 8), INVAL, "k is"), (dict(v=None), INVAL, "v is"), (dict(qo=None), INVAL, "q_out"),
        (dict(ko=D + 8), INVAL, "k_out"), (dict(r=rot(ldq=255)), INVAL, "ldq"), (dict(r=rot(ldk=132)), INVAL, "ldk"), (dict(r=rot(ldv=64)), INVAL, "ldv"),
        (dict(r=rot(ldqo=260)), INVAL, "ldqo"), (dict(r=rot(ldko=127)), INVAL, "ldko"),
        # Overlaps: in place with another stride, shifted, over k or v, over each other.
        (dict(qo=Q), INVAL, "q_out overlaps"), (dict(qo=Q + 16, r=rot(ldqo=512)), INVAL, "q_out overlaps"), (dict(qo=K, r=rot(ldqo=512)), INVAL, "q_out overlaps"),
        (dict(ko=K), INVAL, "k_out overlaps"), (dict(ko=V, r=rot(ldko=512)), INVAL, "k_out overlaps"), (dict(ko=Q + 256, r=rot(ldko=512)), INVAL, "k_out overlaps"),
        (dict(ko=C + 512 * 8), INVAL, "k_out overlaps"),
        # Over what both sides read, and more tokens than a launch has threads for.
        (dict(pos=C + 8 * 512 + 508), INVAL, "overlaps pos"), (dict(f=D), INVAL, "overlaps pos"), (dict(seqs=D + 256), INVAL, "overlaps pos"),
        (dict(off=C - 8), INVAL, "overlaps pos"), (dict(t=1 << 26), UNSUP, "n_tokens (n_kv_heads + 40)")])
    assert call(n=0) == _lib.OK and call(t=0) == _lib.OK


def test_under_host_sanitizers():
    """These checks again with the C-ABI sources built by g++ with both sanitizers, in a child process."""
    import os
    import subprocess
    import sys

    if os.environ.get("S2MOE_LIBRARY"):
        return  # the child
    from paper_2608_15018_amd import build

    build.build_host_sanitized(verbose=False)
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", os.path.abspath(__file__)],
                       cwd=build.ROOT, env=build.host_sanitizer_env(), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
