"""The Python side of the dense half, positions and the append with rotation, without a GPU:
the library is replaced by a recorder, and tensors on the host that say they are on a GPU
stand for tensors there."""

import pytest

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402
from paper_2608_15018_amd import _lib, dense  # noqa: E402

E4M3, BF16, F32 = s2.E4M3, torch.bfloat16, torch.float32


class OnGpu(torch.Tensor):
    """A host tensor that says it is on GPU 0."""

    def get_device(self):
        return 0


def gpu(t):
    return t.as_subclass(OnGpu)


def zeros(*shape, dtype=F32):
    return gpu(torch.zeros(shape, dtype=dtype))


def ints(x):
    return gpu(torch.tensor(x, dtype=torch.int32))


class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return _lib.OK
        return call


@pytest.fixture
def lib(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(_lib, "load", lambda: r)
    monkeypatch.setattr(_lib, "_stream", lambda s: 11 if s is None else int(s))
    monkeypatch.setattr(_lib, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return r


def rows(n, k):
    return s2.Fp8Rows(zeros(n, k, dtype=E4M3), zeros(-(-k // 128), n))


def weight(n, k):
    return s2.Fp8Weight(zeros(n, k, dtype=E4M3), zeros(-(-n // 128), -(-k // 128)))


def cache(lib):
    i32 = torch.int32
    return s2.KVCache(1, 2, 64, 6, 16, 4, 3, k=zeros(1, 6, 2, 16, 64, dtype=BF16), v=zeros(1, 6, 2, 2, 64, 8, dtype=BF16),
                      table=zeros(4, 3, dtype=i32), length=zeros(4, dtype=i32), refs=zeros(6, dtype=i32))


def calls(c):
    """(name, function, its tensors) of every call that takes tensors."""
    seqs, off, pos = ints([0, 1]), ints([0, 3, 5]), ints([0] * 5)
    q, kv, f = zeros(5, 4, 64, dtype=BF16), zeros(5, 2, 64, dtype=BF16), zeros(16)
    return [
        ("add_norm", lambda a: s2.add_norm(a["x"], a["weight"], a["residual"], out=s2.Fp8Rows(a["codes"], a["scales"])),
         dict(x=zeros(3, 272), weight=zeros(272), residual=zeros(3, 272), codes=zeros(3, 272, dtype=E4M3), scales=zeros(3, 3))),
        ("add_norm", lambda a: s2.add_norm(a["x"], a["weight"], out=a["out"]), dict(x=zeros(3, 272), weight=zeros(272), out=zeros(3, 272))),
        ("quantize", lambda a: s2.quantize(a["x"], s2.Fp8Rows(a["codes"], a["scales"])),
         dict(x=zeros(3, 272), codes=zeros(3, 272, dtype=E4M3), scales=zeros(3, 3))),
        ("quantize_weight", lambda a: s2.quantize_weight(a["w"]), dict(w=zeros(130, 272))),
        ("scaled_matmul", lambda a: s2.fp8_matmul(s2.Fp8Rows(a["x"], a["x_scales"]), s2.Fp8Weight(a["w"], a["w_scales"]), out=a["out"]),
         dict(x=zeros(3, 272, dtype=E4M3), x_scales=zeros(3, 3), w=zeros(130, 272, dtype=E4M3), w_scales=zeros(2, 3), out=zeros(3, 130))),
        ("kv_positions", lambda a: c.positions(a["seqs"], a["tok_off"], 5, a["parent"], out=a["out"]),
         dict(seqs=seqs, tok_off=off, parent=pos, out=pos)),
        ("kv_append_rotated", lambda a: c.append_rotated(0, a["q"], a["k"], a["v"], a["seqs"], a["tok_off"], a["pos"], a["inv_freq"],
                                                         out=a["out"], k_out=a["k_out"]),
         dict(q=q, k=kv, v=kv, seqs=seqs, tok_off=off, pos=pos, inv_freq=f, out=q, k_out=kv)),
    ]


def test_every_tensor_has_to_be_on_the_gpu(lib):
    c = cache(lib)
    for name, f, tensors in calls(c):
        lib.calls.clear()
        f(tensors)
        assert [n for n, _ in lib.calls] == ["s2moe_" + name]
        for one in tensors:
            lib.calls.clear()
            away = dict(tensors, **{one: torch.zeros_like(tensors[one].as_subclass(torch.Tensor))})
            with pytest.raises(s2.S2moeError, match="not on") as e:
                f(away)
            assert e.value.status == _lib.EINVAL and not lib.calls, (name, one)


def test_the_gpu_has_to_be_the_current_one(lib, monkeypatch):
    c = cache(lib)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    lib.calls.clear()
    for name, f, tensors in calls(c):
        with pytest.raises(s2.S2moeError, match="current"):
            f(tensors)
        assert not lib.calls, name


def test_shapes_and_types(lib):
    x, w = zeros(3, 272), zeros(272)
    for bad in (lambda: s2.add_norm(zeros(272), w), lambda: s2.add_norm(x, zeros(256)), lambda: s2.add_norm(x, w, zeros(3, 256)),
                lambda: s2.add_norm(x, w, zeros(2, 272)), lambda: s2.add_norm(gpu(torch.zeros(272, 3).t()), w),
                lambda: s2.add_norm(x, w, out=zeros(4, 272)), lambda: s2.add_norm(x, zeros(272, 2)[:, 0]),
                lambda: s2.add_norm(x, w, out=rows(4, 272)), lambda: s2.quantize(zeros(2, 3, 4)), lambda: s2.quantize(x, rows(3, 256)),
                lambda: s2.quantize(x, s2.Fp8Rows(zeros(3, 272, dtype=E4M3), zeros(3, 4))), lambda: s2.quantize_weight(zeros(3)),
                lambda: s2.fp8_matmul(rows(3, 272), weight(130, 256)), lambda: s2.fp8_matmul(rows(3, 272), weight(130, 272), out=zeros(3, 131)),
                lambda: s2.fp8_matmul(s2.Fp8Rows(rows(3, 272).codes, zeros(3, 4)), weight(130, 272)),
                lambda: s2.fp8_matmul(rows(3, 272), s2.Fp8Weight(weight(130, 272).codes, zeros(1, 3)))):
        with pytest.raises(ValueError):
            bad()
    half = zeros(3, 272, dtype=torch.float16)
    for bad in (lambda: s2.add_norm(half, w), lambda: s2.add_norm(x, w.half()), lambda: s2.add_norm(x, w, half),
                lambda: s2.add_norm(x, w, out_dtype=torch.float16), lambda: s2.add_norm(x, w, out=half), lambda: s2.add_norm(x, w, out=x, out_dtype=BF16),
                lambda: s2.add_norm(x, w, out=rows(3, 272).codes), lambda: s2.quantize(rows(3, 272).codes), lambda: s2.quantize_weight(half),
                lambda: s2.quantize(x, s2.Fp8Rows(zeros(3, 272, dtype=torch.uint8), zeros(3, 3))),
                lambda: s2.fp8_matmul(s2.Fp8Rows(x, zeros(3, 3)), weight(130, 272)), lambda: s2.fp8_matmul(rows(3, 272), weight(130, 272), out_dtype=E4M3),
                lambda: s2.fp8_matmul(rows(3, 272), weight(130, 272), out=zeros(3, 130, dtype=torch.float16)),
                lambda: s2.fp8_matmul(rows(3, 272), weight(130, 272), out=zeros(3, 130), out_dtype=BF16)):
        with pytest.raises(TypeError):
            bad()
    assert not lib.calls


def test_strides_go_through(lib):
    wide = zeros(10, 320)
    out = s2.Fp8Rows(zeros(10, 400, dtype=E4M3)[2:5, :272], zeros(3, 20)[:, 4:7])
    s2.add_norm(wide[1:4, :272], zeros(272, dtype=BF16), wide[5:8, :272], 1e-5, out=out)
    name, a = lib.calls.pop()
    assert name == "s2moe_add_norm" and a[:2] == (3, 272) and a[3:5] == (320, _lib.F32) and a[6:8] == (320, _lib.F32)
    assert a[9:11] == (_lib.BF16, 1e-5) and a[12:14] == (400, _lib.E4M3) and a[15] == 20 and a[16] == 11
    y = s2.fp8_matmul(s2.Fp8Rows(zeros(9, 400, dtype=E4M3)[:3, :272], zeros(3, 20)[:, :3]), weight(130, 272), out=zeros(3, 200)[:, :130])
    name, a = lib.calls.pop()
    assert name == "s2moe_scaled_matmul" and a[:3] == (3, 130, 272) and a[4] == 400 and a[6] == 20 and a[8] == 272 and a[10] == 3
    assert a[12:14] == (200, _lib.F32) and y.shape == (3, 130)
    # One row, or one block: the stride of a size-one dimension says nothing.
    s2.fp8_matmul(s2.Fp8Rows(zeros(1, 64, dtype=E4M3), zeros(1, 1)), weight(5, 64))
    name, a = lib.calls.pop()
    assert a[4] == 64 and a[6] >= 1 and a[10] >= 1


def test_results_are_made(lib):
    x = zeros(3, 272, dtype=BF16)
    assert s2.add_norm(x, zeros(272)).dtype == BF16 and s2.add_norm(x, zeros(272), out_dtype=F32).dtype == F32
    y = s2.add_norm(x, zeros(272), out_dtype=E4M3)
    assert isinstance(y, s2.Fp8Rows) and y.codes.shape == (3, 272) and y.scales.shape == (3, 3) and y.codes.dtype == E4M3
    assert s2.quantize(x).scales.shape == (3, 3) and s2.quantize_weight(zeros(130, 272)).scales.shape == (2, 3)
    assert s2.fp8_matmul(y, weight(130, 272)).dtype == BF16


def test_rotation_arguments(lib):
    c = cache(lib)
    seqs, off, pos, f = ints([0, 1]), ints([0, 3, 5]), ints([0] * 5), zeros(16)
    big = zeros(5, 8, 64, dtype=BF16)
    q, k, v = big[:, :4], big[:, 4:6], big[:, 6:]
    lib.calls.clear()
    got = c.append_rotated(0, q, k, v, seqs, off, pos, f, True, out=q, k_out=k)
    name, a = lib.calls.pop()
    r = a[2]._obj
    assert got is q and (r.n_heads, r.rot_dim, r.neighbours, r.ldq, r.ldk, r.ldv, r.ldqo, r.ldko) == (4, 32, 1, 512, 512, 512, 512, 512)
    assert c.append_rotated(0, q, k, v, seqs, off, pos, f).shape == (5, 4, 64)
    name, a = lib.calls.pop()
    assert (a[2]._obj.ldqo, a[2]._obj.neighbours, a[13]) == (256, 0, None)
    for bad in (lambda: c.append_rotated(0, q[:, :, :32], k, v, seqs, off, pos, f), lambda: c.append_rotated(0, q, k[:4], v, seqs, off, pos, f),
                lambda: c.append_rotated(0, q, k, v, seqs, off, pos[:4], f), lambda: c.append_rotated(0, q, k, v, seqs, off, pos, f.double()),
                lambda: c.append_rotated(0, q, k, v, seqs, off[:2], pos, f), lambda: c.append_rotated(0, q[0], k, v, seqs, off, pos, f),
                lambda: c.append_rotated(0, q, k, v, seqs, off, pos, f, out=q[:4]), lambda: c.append_rotated(0, q.float(), k, v, seqs, off, pos, f),
                lambda: c.append_rotated(0, q, k, v, seqs, off, pos, f, k_out=k[:4]), lambda: c.positions(seqs, off, 5, pos[:4]),
                lambda: c.positions(seqs, off, 5, out=pos[:4]), lambda: c.positions(seqs, off.long(), 5)):
        with pytest.raises(ValueError):
            bad()
    assert not lib.calls


def test_blocks():
    assert dense.BLOCK == 128 and [dense._blocks(n) for n in (1, 128, 129, 2880)] == [1, 1, 2, 23]
