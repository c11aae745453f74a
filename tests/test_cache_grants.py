"""Grants of the cache when pages run out: a request whose status is 0 can write every slot
that it asked for, and one that is refused changes nothing.  The host model by that
invariant, and the device against the model."""

import numpy as np
import pytest

from oracle import attention_oracle as ao


def model(pages, seqs=8, maxp=6, P=16):
    return ao.Cache(np.zeros((1, pages, 1, P, 2)), np.zeros((1, pages, 1, P // 8, 2, 8)),
                    np.full((seqs, maxp), -1, dtype=np.int32), np.zeros(seqs, dtype=np.int32), np.zeros(pages, dtype=np.int32))


def held_writable(c, seqs, extra, status):
    """Every slot that a granted request asked for is in a page of the sequence's own."""
    return all(c.own_slot(s, int(c.length[s]) + j) is not None
               for s, e, st in zip(seqs, extra, status) if st == 0 for j in range(e))


def start(c, forks, length=20):
    """Sequence 0 with `length` tokens, and forks of it."""
    assert c.reserve([0], [length])[0] == [0]
    assert c.commit([0], None, [length]) == [0]
    assert c.fork([0] * forks, list(range(1, forks + 1))) == [0] * forks


# (pages, forks, requested sequences, extra tokens, wanted status): a sharer that was refused its copy still
# holds the page, so nobody else may keep it.
SHARED = [
    (2, 1, [1, 0], [1, 1], [1, 1]),
    (3, 1, [1, 0], [1, 1], [0, 0]),
    (3, 2, [1, 2, 0], [1, 1, 1], [0, 1, 1]),
    (4, 2, [1, 2, 0], [1, 1, 1], [0, 0, 0]),
    (3, 1, [1, 0], [13, 1], [1, 1]),
    (2, 1, [1, 0], [1, 0], [1, 0]),
    (2, 1, [1, 7, 0], [1, 0, 1], [1, 0, 1]),
    (2, 1, [1, 0, 0], [1, 1, 1], [1, 1, 4]),
    (2, 1, [1, 0], [77, 1], [2, 1]),
    (2, 1, [7, 1], [1, 0], [1, 0]),
    (3, 0, [1, 0, 2], [17, 1, 1], [1, 0, 1]),
]


@pytest.mark.parametrize("pages,forks,seqs,extra,want", SHARED)
def test_model_sharers_of_a_page_that_was_not_copied(pages, forks, seqs, extra, want):
    c = model(pages)
    start(c, forks)
    before = c.table.copy(), c.refs.copy()
    assert c.reserve(seqs, extra)[0] == want
    assert held_writable(c, seqs, extra, want)
    if not any(st == 0 and e for st, e in zip(want, extra)):
        assert np.array_equal(c.table, before[0]) and np.array_equal(c.refs, before[1])


@pytest.mark.parametrize("seed", range(20))
def test_model_grants_are_writable(seed):
    r = np.random.default_rng(seed)
    c = model(int(r.integers(4, 16)))
    refused = 0
    for _ in range(200):
        n = int(r.integers(1, 7))
        seqs = r.permutation(8)[:n].tolist()
        op = r.integers(0, 4)
        if op == 0:
            c.fork(r.integers(0, 8, n).tolist(), seqs)
        elif op == 1:
            c.free(seqs[:1])
        else:
            extra = r.integers(0, 20, n).tolist()
            status, _ = c.reserve(seqs, extra)
            refused += ao.NO_PAGES in status
            assert held_writable(c, seqs, extra, status)
            acc = [int(r.integers(0, e + 1)) if st == 0 else 0 for e, st in zip(extra, status)]
            assert c.commit(seqs, None, acc) == [0] * n
    assert refused


@pytest.mark.gpu
@pytest.mark.parametrize("pages,forks,seqs,extra,want", SHARED)
def test_sharers_of_a_page_that_was_not_copied(pages, forks, seqs, extra, want):
    from tests.test_gpu_kv_cache import Pair

    c = Pair(pages=pages, seqs=8, maxp=6)
    c.reserve([0], [20]), c.commit([0], None, [20]), c.fork([0] * forks, list(range(1, forks + 1)))
    assert c.reserve(seqs, extra) == want
    # What was granted is written, and kept.
    had = [(s, e) for s, e, st in zip(seqs, extra, want) if st == 0 and e]
    if had:
        c.append(0, [s for s, _ in had], [e for _, e in had])
        assert c.commit([s for s, _ in had], None, [e for _, e in had]) == [0] * len(had)


@pytest.mark.gpu
def test_a_refused_sharer_that_leaves_frees_the_page_for_the_other():
    from tests.test_gpu_kv_cache import Pair

    c = Pair(pages=2)
    c.reserve([0], [20]), c.commit([0], None, [20]), c.fork([0], [1])
    assert c.reserve([1, 0], [1, 1]) == [ao.NO_PAGES, ao.NO_PAGES]
    c.free([1])
    assert c.reserve([0], [1]) == [0]
    c.append(0, [0], [1])
    assert c.commit([0], None, [1]) == [0]


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(4))
def test_random_programs_short_of_pages(seed):
    from tests.test_gpu_kv_cache import Pair

    r = np.random.default_rng(100 + seed)
    c = Pair(pages=int(r.integers(5, 14)), seqs=8, maxp=6, seed=seed)
    refused = 0
    for _ in range(60):
        n = int(r.integers(1, 7))
        seqs = r.permutation(8)[:n].tolist()
        op = r.integers(0, 4)
        if op == 0:
            c.fork(r.integers(0, 8, n).tolist(), seqs)
        elif op == 1:
            c.free(seqs[:1])
        else:
            extra = r.integers(0, 20, n).tolist()
            status = c.reserve(seqs, extra)
            refused += ao.NO_PAGES in status
            assert held_writable(c.host, seqs, extra, status)
            c.append(1, seqs, extra)
            assert c.commit(seqs, None, [e if st == 0 else 0 for e, st in zip(extra, status)]) == [0] * n
    assert refused


@pytest.mark.gpu
def test_many_sharers_of_one_page():
    """1000 branches of one page, as many copies as there are pages."""
    from tests.test_gpu_kv_cache import Pair

    c = Pair(layers=1, Hkv=1, pages=602, seqs=1024, maxp=4)
    c.reserve([0], [20]), c.commit([0], None, [20])
    c.fork([0] * 999, list(range(1, 1000)))
    order = np.random.default_rng(2).permutation(1000).tolist()
    assert c.reserve(order, [1] * 1000) == [0] * 600 + [ao.NO_PAGES] * 400
    c.free(order[600:999])
    assert c.reserve([order[999]], [1]) == [0]


@pytest.mark.gpu
def test_wants_that_add_up_to_more_than_32_bits():
    """40 requests of 2^27 - 1 pages each: none fits, and the sums of what they want do not wrap."""
    import paper_2608_15018_amd as s2
    import torch

    maxp, n = (1 << 27) - 1, 40
    c = s2.KVCache(1, 1, 64, 12, 16, n + 2, maxp)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    order = [n] + list(range(n)) + [n + 1]
    c.reserve(ints(order), ints([40] + [16 * maxp] * n + [0]))
    assert c.status[:n + 2].tolist() == [0] + [ao.NO_PAGES] * n + [0]
    assert c.refs.tolist() == [1, 1, 1] + [0] * 9 and c.table[n, :4].tolist() == [0, 1, 2, -1]
    assert int((c.table[:n] >= 0).sum()) == 0
