"""Host checks of the cache and attention entry points: malformed arguments are
refused before anything is enqueued (no kernel is launched by these tests)."""

import ctypes

import pytest

import paper_2608_15018_amd as s2
from paper_2608_15018_amd import _lib

P = ctypes.c_void_p
A, B = 0x10000000, 0x20000000  # aligned fake addresses; every call below fails or does nothing


@pytest.fixture(scope="module")
def lib():
    return s2.load()


def cache(**kw):
    d = dict(n_layers=2, n_kv_heads=2, head_dim=64, n_pages=8, page_size=16, max_seqs=4, max_pages=4,
             dtype=_lib.BF16, k=A, v=A, table=A, length=A, refs=A)
    d.update(kw)
    return _lib.KvCacheStruct(**d)


def attn(**kw):
    d = dict(n_heads=4, n_kv_heads=2, head_dim=64, dtype=_lib.BF16, scale=0.125, ldq=256, ldk=128, ldv=128, ldo=256)
    d.update(kw)
    return _lib.Attn(**d)


CACHE_FAULTS = [
    (dict(dtype=2), _lib.EINVAL, "dtype"), (dict(head_dim=96), _lib.EUNSUPPORTED, "head_dim"),
    (dict(head_dim=0), _lib.EINVAL, "head_dim"), (dict(n_kv_heads=0), _lib.EINVAL, "n_kv_heads"),
    (dict(n_kv_heads=257), _lib.EUNSUPPORTED, "n_kv_heads"), (dict(n_layers=0), _lib.EINVAL, "n_layers"),
    (dict(n_layers=1025), _lib.EUNSUPPORTED, "n_layers"), (dict(page_size=8), _lib.EINVAL, "page_size"),
    (dict(page_size=48), _lib.EINVAL, "page_size"), (dict(n_pages=0), _lib.EINVAL, "n_pages"),
    (dict(n_pages=(1 << 24) + 1), _lib.EINVAL, "n_pages"), (dict(max_seqs=0), _lib.EINVAL, "max_seqs"),
    (dict(max_pages=0), _lib.EINVAL, "max_pages"), (dict(max_pages=1 << 27), _lib.EINVAL, "max_pages"),
    (dict(k=None), _lib.EINVAL, "c.k"), (dict(v=A + 8), _lib.EINVAL, "c.v"), (dict(table=A + 2), _lib.EINVAL, "c.table"),
    (dict(length=None), _lib.EINVAL, "c.length"), (dict(refs=A + 1), _lib.EINVAL, "c.refs"),
]


def calls(lib, c, n=1):
    """Every entry point that takes a cache, on plausible arguments."""
    r, a = ctypes.byref(c) if c is not None else None, ctypes.byref(attn())
    return {
        "kv_init": lambda: lib.s2moe_kv_init(r, None),
        "kv_fork": lambda: lib.s2moe_kv_fork(r, n, A, A, A, None),
        "kv_reserve": lambda: lib.s2moe_kv_reserve(r, n, A, A, A, A, None),
        "kv_append": lambda: lib.s2moe_kv_append(r, 0, n, 1, A, A, A, 128, A, 128, None),
        "kv_commit": lambda: lib.s2moe_kv_commit(r, n, 1, A, A, A, A, None),
        "kv_free": lambda: lib.s2moe_kv_free(r, n, A, A, None),
        "tree_attention": lambda: lib.s2moe_tree_attention(r, 0, a, n, 1, 1, A, A, A, A, A, 1 << 40, B, None),
    }


@pytest.mark.parametrize("kw,status,needle", CACHE_FAULTS)
def test_malformed_caches(lib, kw, status, needle):
    for name, call in calls(lib, cache(**kw)).items():
        assert call() == status, name
        assert needle in _lib.last_error() and "s2moe_" + name in _lib.last_error()
    assert lib.s2moe_tree_attention_workspace_bytes(ctypes.byref(cache(**kw)), ctypes.byref(attn()), 1, 1) == 0


def test_null_cache_and_request_counts(lib):
    for name, call in calls(lib, None).items():
        assert call() == _lib.EINVAL and "cache is NULL" in _lib.last_error(), name
    for n, status in ((-1, _lib.EINVAL), (1025, _lib.EUNSUPPORTED)):
        for name, call in calls(lib, cache(), n).items():
            if name != "kv_init":
                assert call() == status and "n = " in _lib.last_error(), name
    for name, call in calls(lib, cache(), 0).items():
        if name != "kv_init":
            assert call() == _lib.OK and _lib.last_error() == "", name


def test_page_operations_need_their_arrays(lib):
    c = ctypes.byref(cache())
    for i in range(3):
        p = [A, A, A]
        for bad, word in ((None, "NULL"), (A + 2, "aligned")):
            p[i] = bad
            assert lib.s2moe_kv_fork(c, 1, *p, None) == _lib.EINVAL and word in _lib.last_error()
            assert lib.s2moe_kv_reserve(c, 1, *p, A, None) == _lib.EINVAL and word in _lib.last_error()
    assert lib.s2moe_kv_reserve(c, 1, A, A, A, None, None) == _lib.EINVAL and "status" in _lib.last_error()
    assert lib.s2moe_kv_free(c, 1, None, A, None) == _lib.EINVAL and "seqs" in _lib.last_error()
    assert lib.s2moe_kv_free(c, 1, A, None, None) == _lib.EINVAL and "status" in _lib.last_error()
    assert lib.s2moe_kv_commit(c, 1, -1, A, A, A, A, None) == _lib.EINVAL and "max_path" in _lib.last_error()
    assert lib.s2moe_kv_commit(c, 1, 257, A, A, A, A, None) == _lib.EUNSUPPORTED and "max_path" in _lib.last_error()
    assert lib.s2moe_kv_commit(c, 1, 4, A, A + 1, A, A, None) == _lib.EINVAL and "path" in _lib.last_error()
    assert lib.s2moe_kv_commit(c, 1, 4, A, A, None, A, None) == _lib.EINVAL and "n_accept" in _lib.last_error()


@pytest.mark.parametrize("args,needle", [
    ((-1, 1, 1, A, A, A, 128, A, 128), "layer"), ((2, 1, 1, A, A, A, 128, A, 128), "layer"),
    ((0, 1, -1, A, A, A, 128, A, 128), "n_tokens"), ((0, 1, 1, None, A, A, 128, A, 128), "seqs"),
    ((0, 1, 1, A, A + 2, A, 128, A, 128), "tok_off"), ((0, 1, 1, A, A, None, 128, A, 128), "k is NULL"),
    ((0, 1, 1, A, A, A, 128, A + 4, 128), "v is not"), ((0, 1, 1, A, A, A, 127, A, 128), "ldk"),
    ((0, 1, 1, A, A, A, 128, A, 132), "ldv"), ((0, 1, 1, A, A, A, 128, A, -128), "ldv")])
def test_append_arguments(lib, args, needle):
    assert lib.s2moe_kv_append(ctypes.byref(cache()), *args, None) == _lib.EINVAL
    assert needle in _lib.last_error()


@pytest.mark.parametrize("kw,status,needle", [
    (dict(dtype=2), _lib.EINVAL, "dtype"), (dict(head_dim=80), _lib.EUNSUPPORTED, "head_dim"),
    (dict(head_dim=-1), _lib.EINVAL, "head_dim"), (dict(n_heads=3), _lib.EINVAL, "n_heads"),
    (dict(n_heads=0), _lib.EINVAL, "n_heads"), (dict(n_kv_heads=0), _lib.EINVAL, "n_kv_heads"),
    (dict(n_heads=1026), _lib.EUNSUPPORTED, "n_heads"), (dict(scale=0.0), _lib.EINVAL, "scale"),
    (dict(scale=float("nan")), _lib.EINVAL, "scale"), (dict(scale=float("inf")), _lib.EINVAL, "scale"),
    (dict(ldq=255), _lib.EINVAL, "ldq"), (dict(ldq=260), _lib.EINVAL, "ldq"), (dict(ldo=0), _lib.EINVAL, "ldo")])
def test_malformed_attention(lib, kw, status, needle):
    a, c = attn(**kw), cache()
    assert lib.s2moe_prompt_attention(ctypes.byref(a), 1, 1, A, A, A, A, B, None) == status
    assert needle in _lib.last_error()
    assert lib.s2moe_tree_attention(ctypes.byref(c), 0, ctypes.byref(a), 1, 1, 1, A, A, A, A, A, 1 << 40, B, None) == status
    assert needle in _lib.last_error()


def test_tree_arguments(lib):
    c, a = ctypes.byref(cache()), ctypes.byref(attn())
    need = lib.s2moe_tree_attention_workspace_bytes(c, a, 3, 7)
    assert need > 0

    def call(layer=0, at=a, n=3, t=9, nodes=7, q=A, seqs=A, off=A, par=A, ws=A, size=need, out=B):
        return lib.s2moe_tree_attention(c, layer, at, n, t, nodes, q, seqs, off, par, ws, size, out, None)

    for kw, status, needle in (
            (dict(layer=2), _lib.EINVAL, "layer"), (dict(at=None), _lib.EINVAL, "attn"), (dict(t=-1), _lib.EINVAL, "n_tokens"),
            (dict(nodes=0), _lib.EINVAL, "max_nodes"), (dict(nodes=257), _lib.EUNSUPPORTED, "max_nodes"),
            (dict(q=None), _lib.EINVAL, "q is"), (dict(q=A + 8), _lib.EINVAL, "q is"), (dict(seqs=None), _lib.EINVAL, "seqs"),
            (dict(off=A + 1), _lib.EINVAL, "tok_off"), (dict(par=None), _lib.EINVAL, "parent"),
            (dict(ws=None), _lib.EWORKSPACE, str(need)), (dict(size=need - 1), _lib.EWORKSPACE, str(need)),
            (dict(ws=A + 4), _lib.EINVAL, "workspace"), (dict(out=None), _lib.EINVAL, "out"),
            (dict(out=A + 512 * 8), _lib.EINVAL, "overlaps"),
            (dict(at=ctypes.byref(attn(n_heads=6, n_kv_heads=3, ldq=384, ldo=384))), _lib.EINVAL, "differ"),
            (dict(at=ctypes.byref(attn(head_dim=128, ldq=512, ldo=512))), _lib.EINVAL, "differ"),
            (dict(at=ctypes.byref(attn(dtype=_lib.F32))), _lib.EINVAL, "differ")):
        assert call(**kw) == status, kw
        assert needle in _lib.last_error(), (kw, _lib.last_error())
    assert call(t=0) == _lib.OK
    assert lib.s2moe_tree_attention_workspace_bytes(c, None, 3, 7) == 0


def test_prompt_arguments(lib):
    def call(at=None, n=2, t=9, q=A, k=B, v=B, off=A, out=0x30000000):
        at = at or attn()
        return lib.s2moe_prompt_attention(ctypes.byref(at), n, t, q, k, v, off, out, None)

    for kw, status, needle in (
            (dict(n=-1), _lib.EINVAL, "n = "), (dict(n=1025), _lib.EUNSUPPORTED, "n = "), (dict(t=-1), _lib.EINVAL, "n_tokens"),
            (dict(q=None), _lib.EINVAL, "q is"), (dict(k=B + 8), _lib.EINVAL, "k is"), (dict(v=None), _lib.EINVAL, "v is"),
            (dict(off=A + 2), _lib.EINVAL, "tok_off"), (dict(out=None), _lib.EINVAL, "out"), (dict(out=A), _lib.EINVAL, "overlaps"),
            (dict(out=B + 256 * 8), _lib.EINVAL, "overlaps"), (dict(at=attn(ldk=127)), _lib.EINVAL, "ldk"),
            (dict(at=attn(ldv=136 + 4)), _lib.EINVAL, "ldv")):
        assert call(**kw) == status, kw
        assert needle in _lib.last_error(), (kw, _lib.last_error())
    assert call(t=0) == _lib.OK and call(n=0) == _lib.OK
    assert lib.s2moe_prompt_attention(None, 1, 1, A, A, A, A, B, None) == _lib.EINVAL


def test_rows_of_one_array_side_by_side_do_not_overlap(lib):
    """out may be columns of the array that q is columns of; one element in common is refused."""
    ok = attn(ldq=640, ldk=640, ldv=640, ldo=640)  # fails later, at the last pointer checked before the launch
    call = lambda at, out, off: lib.s2moe_prompt_attention(ctypes.byref(at), 1, 9, A, A + 512, A + 768, off, out, None)  # noqa: E731
    for col, want in ((0, "overlaps"), (496, "overlaps"), (512, "overlaps"), (1008, "overlaps"), (784, "overlaps")):
        assert call(ok, A + col, A) == _lib.EINVAL and want in _lib.last_error(), col


def test_binding_checks():
    import torch

    with pytest.raises(TypeError):
        s2.KVCache(1, 1, 64, 1, 16, 1, 1, dtype=torch.float16, device="cpu")
    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    off = torch.tensor([0, 4], dtype=torch.int32)
    for q, kk in ((k[:, :, :32], k), (k.float(), k), (k, k.transpose(0, 1)), (k[0], k), (k[::2], k)):
        with pytest.raises(ValueError):
            s2.prompt_attention(q, kk, k, off)
    with pytest.raises(ValueError):
        s2.prompt_attention(k, k, k, off.long())
    with pytest.raises(s2.S2moeError) as e:
        s2.prompt_attention(torch.zeros((4, 3, 64), dtype=torch.bfloat16), k, k, off, stream=0)
    assert e.value.status == _lib.EINVAL


def test_under_host_sanitizers():
    """These checks again with api.cpp and api_cache.cpp built by g++ with both sanitizers, in a child process."""
    import os
    import subprocess
    import sys

    if os.environ.get("S2MOE_LIBRARY"):
        return  # the child
    from paper_2608_15018_amd import build

    lib = build.build_host_sanitized(verbose=False)
    assert "__asan_" in subprocess.run(["nm", "-D", lib], capture_output=True, text=True, check=True).stdout
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", os.path.abspath(__file__)],
                       cwd=build.ROOT, env=build.host_sanitizer_env(), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
