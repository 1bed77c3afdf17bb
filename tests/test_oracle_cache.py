"""Pins of the cache oracle: closed forms, agreement with the masked attention oracle, evictions worked by hand."""

import numpy as np

from oracle import attention as oa
from oracle import cache as oc


def test_zero_queries_average_what_they_see():
    rng = np.random.default_rng(1)
    k, v, pk, pv = rng.normal(size=(2, 1, 6, 4)), rng.normal(size=(2, 1, 6, 4)), rng.normal(size=(1, 3, 4)), rng.normal(size=(1, 3, 4))
    q = np.zeros((2, 2, 2, 4))
    O, LSE, A, W = oc.cache_attention(q, [5, 1], k, v, pk, pv, causal=True)
    # sequence 0, five keys, two new ones: query 0 sees four own keys, query 1 five; sequence 1's first query none of its one key
    for b, t, n in ((0, 0, 4), (0, 1, 5), (1, 0, 0), (1, 1, 1)):
        np.testing.assert_allclose(LSE[b, :, t], np.log(3 + n))
        seen = np.concatenate([pv[0], v[b, 0, :n]])
        np.testing.assert_allclose(O[b, 0, t], seen.mean(0))
        np.testing.assert_allclose(A[b, 0, t], np.abs(seen).mean(0))
    np.testing.assert_allclose(W[0, 0], [2 * (1 / 7 + 1 / 8)] * 4 + [2 / 8, 0])      # two heads of the group
    np.testing.assert_allclose(W[1, 0], [2 / 4] + [0] * 5)


def test_without_causality_it_is_dense_attention_over_prefix_and_own_keys():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(1, 2, 8, 4)), rng.normal(size=(1, 2, 8, 4)), rng.normal(size=(1, 2, 8, 4))
    O, LSE, _, W = oc.cache_attention(q, [5], k[:, :, 3:], v[:, :, 3:], k[0, :, :3], v[0, :, :3], causal=False)
    Od, Ld = oa.masked_attention(q, k, v, np.ones((2, 2, 2), np.uint8), 4)
    np.testing.assert_allclose(O, Od, atol=1e-12)
    np.testing.assert_allclose(LSE, Ld, atol=1e-12)
    assert (W.sum(-1) < 8).all()


def test_weights_sum_to_the_queries_without_a_prefix():
    rng = np.random.default_rng(3)
    q, k, v = rng.normal(size=(2, 6, 5, 4)), rng.normal(size=(2, 3, 9, 4)), rng.normal(size=(2, 3, 9, 4))
    O, LSE, _, W = oc.cache_attention(q, [9, 0], k, v, q_lens=[3, 5])
    np.testing.assert_allclose(W[0].sum(-1), 2 * 3)
    assert (W[1] == 0).all() and (O[1] == 0).all() and (LSE[1] == -np.inf).all()
    assert np.isnan(O[0, :, 3:]).all()


def _evict(weights, positions, n, budget, **kw):
    cap = len(weights)
    k = np.arange(cap, dtype=float).reshape(1, 1, cap, 1)
    out = oc.cache_evict(k, k + 100, np.array(weights, float)[None, None], np.array(positions)[None, None], [n], budget, **kw)
    return [x.ravel().tolist() for x in out]


def test_evictions_by_hand():
    # slots 1 and 3 go (the lightest); the kept ones behind the budget, 4 and 5, take their places
    k, v, w, pos, lens = _evict([5, 1, 4, 0, 3, 2, 9], range(7), 6, 4)
    assert k == [0, 4, 2, 5, 4, 5, 6] and v == [100, 104, 102, 105, 104, 105, 106] and lens == [4]
    assert w == [5, 3, 4, 2, 0, 0, 9] and pos == [0, 4, 2, 5, 4, 5, 6]
    # equal weights: the lowest slots stay
    assert _evict([1, 1, 1, 1], range(4), 4, 2)[0] == [0, 1, 2, 3]
    # sinks and recent positions stay whatever their weight; NaN is the lightest
    k, _, _, pos, _ = _evict([0, 9, np.nan, 8, 7, 0], [0, 1, 2, 3, 4, 5], 6, 3, sinks=1, keep_from=[5])
    assert sorted(pos[:3]) == [0, 1, 5] and k[:3] == [0, 1, 5]
    # nothing over the budget
    assert _evict([1, 2, 3], range(3), 2, 2)[4] == [2]
