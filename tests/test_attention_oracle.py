"""Pins of the attention and cache oracle: closed forms and invariants."""

import numpy as np
import pytest

from oracle import attention_oracle as ao


def _rng(seed):
    return np.random.default_rng(seed)


def test_equal_scores_give_the_mean_and_one_large_score_its_row():
    v = _rng(0).normal(size=(5, 8))
    vis = np.array([True, False, True, True, False])
    np.testing.assert_allclose(ao.attend(np.zeros(8), np.ones((5, 8)), v, vis, 1.0),
                               v[[0, 2, 3]].mean(0), rtol=1e-14)
    k = np.zeros((5, 8))
    k[3, 0] = 1.0
    q = np.zeros(8)
    q[0] = 800.0
    np.testing.assert_allclose(ao.attend(q, k, v, vis, 1.0), v[3], rtol=1e-14)
    assert not ao.attend(q, k, v, np.zeros(5, dtype=bool), 1.0).any()


def test_two_rows_are_a_logistic_mix():
    q, k, v = np.array([2.0, 0.0]), np.array([[0.3, 5.0], [-0.4, 7.0]]), np.array([[1.0, 0], [0, 1.0]])
    p = 1 / (1 + np.exp(-0.5 * 2 * 0.7))
    np.testing.assert_allclose(ao.attend(q, k, v, np.ones(2, dtype=bool), 0.5), [p, 1 - p], rtol=1e-14)


def test_visibility_of_a_hand_made_tree():
    seen, valid = ao.tree_visible([-1, 0, 0, 2, -1, 3, 7, 3, 5, -2, 9])
    assert valid.tolist() == [True] * 6 + [False, True, True, False, False]
    rows = {i: np.nonzero(seen[i])[0].tolist() for i in range(11)}
    assert rows == {0: [0], 1: [0, 1], 2: [0, 2], 3: [0, 2, 3], 4: [4], 5: [0, 2, 3, 5], 6: [],
                    7: [0, 2, 3, 7], 8: [0, 2, 3, 5, 8], 9: [], 10: []}


def test_a_chain_over_an_empty_cache_is_a_prompt():
    r = _rng(1)
    q, k, v = r.normal(size=(7, 4, 8)), r.normal(size=(7, 2, 8)), r.normal(size=(7, 2, 8))
    a = ao.tree_attention(q, k, v, 0, list(range(-1, 6)), 0.4)
    np.testing.assert_allclose(a, ao.prompt_attention(q, k, v, [0, 7], 0.4), rtol=1e-12)
    b = ao.prompt_attention(q, k, v, [0, 3, 3, 7], 0.4)
    np.testing.assert_allclose(b[:3], a[:3], rtol=1e-12)
    np.testing.assert_allclose(b[3:], ao.prompt_attention(q[3:], k[3:], v[3:], [0, 4], 0.4), rtol=1e-12)


def _cache(P=16, pages=9, seqs=4, maxp=3):
    r = _rng(2)
    return ao.Cache(r.normal(size=(2, pages, 2, P, 4)), r.normal(size=(2, pages, 2, P // 8, 4, 8)),
                    np.full((seqs, maxp), -1, dtype=np.int32), np.zeros(seqs, dtype=np.int32),
                    np.zeros(pages, dtype=np.int32))


def test_a_sequence_reads_back_what_was_appended_and_kept():
    c, r = _cache(), _rng(3)
    k, v = r.normal(size=(20, 2, 4)), r.normal(size=(20, 2, 4))
    assert c.reserve([1], [20])[0] == [0]
    assert c.table[1].tolist() == [0, 1, -1] and c.refs.tolist() == [1, 1] + [0] * 7
    c.append(1, k, v, [1], [0, 20])
    assert c.commit([1], None, [12]) == [0]
    assert c.length[1] == 12 and c.table[1].tolist() == [0, -1, -1]
    assert c.reserve([1], [8])[0] == [0]  # the drafted tokens' page comes back, with what it held
    assert c.commit([1], [[1, 4, 5, 7]], [4]) == [0]
    gk, gv = c.tokens(1, 1, 16)
    keep = list(range(12)) + [13, 16, 17, 19]
    np.testing.assert_array_equal(gk, k[keep])
    np.testing.assert_array_equal(gv, v[keep])


def test_forks_share_until_they_write():
    c = _cache()
    c.reserve([0], [20])
    c.commit([0], None, [20])
    assert c.fork([0, 0, 1], [1, 2, 3]) == [0, 0, ao.BAD_SEQ]
    assert c.refs.tolist()[:2] == [3, 3]
    status, copied = c.reserve([1, 2, 0], [1, 1, 1])
    assert status == [0, 0, 0] and copied.tolist() == [[1, 2], [1, 3], [-1, -1]]
    assert c.refs.tolist() == [3, 1, 1, 1] + [0] * 5
    np.testing.assert_array_equal(c.k[:, 2, :, :8], c.k[:, 1, :, :8])
    assert c.free([0, 1, 2]) == [0, 0, 0] and not c.refs.any() and (c.table == -1).all()


@pytest.mark.parametrize("extra,want", [([48, 48, 48, 1], [0, 0, 0, ao.NO_PAGES]),
                                        ([48, 40, 49, 33], [0, 0, ao.TOO_LONG, 0]),
                                        ([48, 48, 0, 49], [0, 0, 0, ao.TOO_LONG])])
def test_grants_in_order(extra, want):
    c = _cache()
    assert c.reserve([2, 0, 1, 3], extra)[0] == want
