"""The Python side of the cache and attention operators, without a GPU: the library is
replaced by a recorder, and tensors on the host that say they are on a GPU stand for
tensors there."""

import pytest

torch = pytest.importorskip("torch")

import paper_2608_15018_amd as s2  # noqa: E402
from paper_2608_15018_amd import _lib, attention  # noqa: E402


class OnGpu(torch.Tensor):
    """A host tensor that says it is on GPU 0."""

    def get_device(self):
        return 0


def gpu(t):
    return t.as_subclass(OnGpu)


def ints(x):
    return torch.tensor(x, dtype=torch.int32)


class Recorder:
    """Every entry point: notes its name and arguments and reports success."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 64 if name.endswith("workspace_bytes") else _lib.OK
        return call


@pytest.fixture
def lib(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(_lib, "load", lambda: r)
    monkeypatch.setattr(_lib, "_stream", lambda s: 11 if s is None else int(s))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return r


L, HKV, D, PAGES, P, S, MAXP, HQ, BF16 = 2, 2, 64, 6, 16, 4, 3, 4, torch.bfloat16


def arrays():
    return dict(k=torch.zeros((L, PAGES, HKV, P, D), dtype=BF16), v=torch.zeros((L, PAGES, HKV, P // 8, D, 8), dtype=BF16),
                table=torch.full((S, MAXP), -1, dtype=torch.int32), length=torch.zeros(S, dtype=torch.int32),
                refs=torch.zeros(PAGES, dtype=torch.int32))


def make_cache(**kw):
    return s2.KVCache(L, HKV, D, PAGES, P, S, MAXP, **dict({n: gpu(t) for n, t in arrays().items()}, **kw))


def calls(cache, att):
    """(name, function, its tensors) of every call that takes tensors."""
    t = 5
    kv = torch.zeros((t, HKV, D), dtype=BF16)
    q = torch.zeros((t, HQ, D), dtype=BF16)
    seqs, off = ints([0, 1]), ints([0, 3, 5])
    return [
        ("fork", lambda a: cache.fork(a["src"], a["dst"], stream=11), dict(src=seqs, dst=seqs + 2)),
        ("reserve", lambda a: cache.reserve(a["seqs"], a["extra"], stream=11), dict(seqs=seqs, extra=seqs)),
        ("append", lambda a: cache.append(0, a["k"], a["v"], a["seqs"], a["tok_off"], stream=11),
         dict(k=kv, v=kv, seqs=seqs, tok_off=off)),
        ("commit", lambda a: cache.commit(a["seqs"], a["path"], a["n_accept"], stream=11),
         dict(seqs=seqs, path=ints([[0], [0]]), n_accept=seqs)),
        ("free", lambda a: cache.free(a["seqs"], stream=11), dict(seqs=seqs)),
        ("tree", lambda a: att(0, a["q"], a["seqs"], a["tok_off"], a["parent"], out=a["out"], stream=11),
         dict(q=q, seqs=seqs, tok_off=off, parent=ints([-1] * t), out=torch.zeros_like(q))),
        ("prompt", lambda a: s2.prompt_attention(a["q"], a["k"], a["v"], a["tok_off"], out=a["out"], stream=11),
         dict(q=q, k=kv, v=kv, tok_off=off, out=torch.zeros_like(q))),
    ]


@pytest.mark.parametrize("which", range(7))
def test_a_tensor_on_the_host_is_refused_before_the_library(lib, which):
    cache = make_cache()
    name, call, args = calls(cache, s2.TreeAttention(cache, HQ, 2, 4))[which]
    lib.calls.clear()
    call({n: gpu(t) for n, t in args.items()})
    assert [c[0] for c in lib.calls] == [{"tree": "s2moe_tree_attention", "prompt": "s2moe_prompt_attention"}.get(name, "s2moe_kv_" + name)]
    lib.calls.clear()
    for host in args:
        with pytest.raises(s2.S2moeError) as e:
            call({n: t if n == host else gpu(t) for n, t in args.items()})
        assert e.value.status == _lib.EINVAL and "cpu" in str(e.value), (name, host)
    with pytest.raises(s2.S2moeError):
        call(args)
    assert not lib.calls


def test_a_cache_on_the_host_is_refused(lib):
    with pytest.raises(s2.S2moeError):
        s2.KVCache(L, HKV, D, PAGES, P, S, MAXP, device="cpu")
    for name, t in arrays().items():
        with pytest.raises(s2.S2moeError) as e:
            make_cache(**{name: t})
        assert "cpu" in str(e.value)
    assert not lib.calls


class Streams:
    """Which stream is current, and which one each tensor was allocated on and recorded on."""

    def __init__(self, monkeypatch):
        self.current, self.made, self.recorded = 11, [], []
        monkeypatch.setattr(_lib, "_stream", lambda s: self.current if s is None else int(s))
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
        monkeypatch.setattr(torch.cuda, "stream", self.under)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: self.current)
        monkeypatch.setattr(OnGpu, "new_empty", self.new_empty, raising=False)
        monkeypatch.setattr(OnGpu, "record_stream", lambda t, s: self.recorded.append(s), raising=False)

    def new_empty(self, shape, **kw):
        self.made.append(self.current)
        return gpu(torch.zeros(shape, dtype=kw.get("dtype", BF16)))

    def under(self, s):
        import contextlib

        @contextlib.contextmanager
        def manager():
            before, self.current = self.current, s
            yield
            self.current = before
        return manager()


@pytest.mark.parametrize("which", ["tree", "prompt"])
def test_a_result_is_allocated_on_the_stream_that_writes_it(lib, monkeypatch, which):
    """Memory of the current stream's may still be in use there when another stream writes it; and what
    another stream's allocator gets back may still be in use here."""
    streams = Streams(monkeypatch)
    cache = make_cache()
    att = s2.TreeAttention(cache, HQ, 2, 4)
    q, kv = gpu(torch.zeros((5, HQ, D), dtype=BF16)), gpu(torch.zeros((5, HKV, D), dtype=BF16))
    seqs, off, parent = (gpu(ints(x)) for x in ([0, 1], [0, 3, 5], [-1] * 5))
    for stream, made, recorded in ((None, [11], []), (11, [11], []), (22, [22], [11])):
        streams.made, streams.recorded = [], []
        if which == "tree":
            out = att(0, q, seqs, off, parent, stream=stream)
        else:
            out = s2.prompt_attention(q, kv, kv, off, stream=stream)
        assert out.shape == (5, HQ, D) and streams.current == 11
        assert streams.made == made and streams.recorded == recorded, stream
        assert lib.calls[-1][1][-1] == (stream or 11)


def tree_call(cache, att, rows=HQ, **kw):
    """A call whose q is HQ of `rows` heads of a wider array."""
    q = gpu(torch.zeros((5, rows, D), dtype=BF16))[:, :HQ]
    return att(0, q, *(gpu(ints(x)) for x in ([0, 1], [0, 3, 5], [-1] * 5)), **kw)


def test_a_call_does_not_change_the_strides_of_another(lib, monkeypatch):
    """The library reads the struct while other threads may be in the same object."""
    Streams(monkeypatch)
    cache = make_cache()
    att = s2.TreeAttention(cache, HQ, 2, 4)
    lib.calls.clear()
    wide = gpu(torch.zeros((5, 3 * HQ, D), dtype=BF16))
    for rows, out in ((HQ, None), (2 * HQ, None), (HQ, wide[:, HQ:2 * HQ]), (HQ, None)):
        tree_call(cache, att, rows, out=out)
    got = [args[2]._obj for _, args in lib.calls]
    assert [(a.ldq, a.ldo) for a in got] == [(HQ * D, HQ * D), (2 * HQ * D, HQ * D), (HQ * D, 3 * HQ * D), (HQ * D, HQ * D)]
    assert {(a.n_heads, a.n_kv_heads, a.head_dim, a.dtype, a.scale) for a in got} == {(HQ, HKV, D, _lib.BF16, 0.125)}


def test_calls_on_different_streams_have_workspaces_of_their_own(lib, monkeypatch):
    """The second launch of a call reads there what the first has left."""
    streams = Streams(monkeypatch)
    cache = make_cache()
    att = s2.TreeAttention(cache, HQ, 2, 4)
    capturing = []
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: streams.current in capturing)
    space = lambda **kw: (lib.calls.clear(), tree_call(cache, att, **kw), lib.calls[-1][1][10])[2]  # noqa: E731
    here, there = space(), space(stream=22)
    assert here == att.workspace.data_ptr() and there != here
    assert [space(), space(stream=22), space(stream=11), space(stream=33)][:3] == [here, there, here]
    assert space(stream=33) not in (here, there)
    with torch.cuda.stream(22):
        assert [space(), space(stream=11)] == [there, here]
    # A graph is replayed beside other calls, so it has memory of its own.
    capturing[:] = [11, 22]
    assert space() not in (here, there) and space(stream=22) not in (here, there)
    capturing.clear()
    assert [space(), space(stream=22)] == [here, there]


def run_threads(*functions):
    import threading

    threads = [threading.Thread(target=f) for f in functions]
    for t in threads:
        t.start()
    for t in threads:
        t.join()


class Slow(Recorder):
    """Calls take a while, and note when two are under way at once."""

    def __init__(self, names):
        super().__init__()
        self.names, self.inside, self.met = names, 0, []

    def __getattr__(self, name):
        import time

        call = super().__getattr__(name)
        if name not in self.names:
            return call

        def slow(*args):
            self.inside += 1
            if self.inside > 1:
                self.met.append(name)
            time.sleep(0.02)
            self.inside -= 1
            return call(*args)
        return slow


def test_the_launches_of_two_threads_calls_do_not_mix(lib, monkeypatch):
    Streams(monkeypatch)
    slow = Slow(["s2moe_tree_attention"])
    monkeypatch.setattr(_lib, "load", lambda: slow)
    cache = make_cache()
    att = s2.TreeAttention(cache, HQ, 2, 4)
    run_threads(*[lambda: [tree_call(cache, att) for _ in range(3)]] * 3)
    assert len([c for c in slow.calls if c[0] == "s2moe_tree_attention"]) == 9 and not slow.met


PAGE_CALLS = ["s2moe_kv_init", "s2moe_kv_fork", "s2moe_kv_reserve", "s2moe_kv_commit", "s2moe_kv_free"]


def test_the_launches_of_two_threads_page_operations_do_not_mix(lib, monkeypatch):
    """reserve's second launch reads `copied`, commit's what the first has checked."""
    slow = Slow(PAGE_CALLS)
    monkeypatch.setattr(_lib, "load", lambda: slow)
    cache = make_cache()
    seqs = gpu(ints([0, 1]))
    run_threads(cache.clear, lambda: cache.fork(seqs, seqs), lambda: cache.reserve(seqs, seqs), lambda: cache.reserve(seqs, seqs),
                lambda: cache.commit(seqs, None, seqs), lambda: cache.free(seqs))
    assert sorted(c[0] for c in slow.calls) == sorted(PAGE_CALLS + ["s2moe_kv_reserve"]) and not slow.met
