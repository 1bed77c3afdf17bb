"""The oracle of norms, rotations and the paged cache, held to hand-worked values, to differences, and to the oracle of the contiguous cache."""

import numpy as np
import pytest

from oracle import cache as oc
from oracle import rows as orows


def test_rotation_by_hand():
    x = np.array([1.0, 2.0, 3.0, 4.0, 5.0, 6.0])
    a = np.array([np.pi / 2, np.pi])
    np.testing.assert_allclose(orows.rotate(x, a, halves=False), [-2, 1, -3, -4, 5, 6], atol=1e-12)
    np.testing.assert_allclose(orows.rotate(x, a, halves=True), [-3, -2, 1, -4, 5, 6], atol=1e-12)
    np.testing.assert_allclose(orows.rotate(orows.rotate(x, a, True), -a, True), x, atol=1e-12)
    # two axes: the first has one pair, the second two
    np.testing.assert_allclose(orows.angles([[2, 10]], (1, 2), (0.5, 1.0, 0.1)), [[1.0, 10.0, 1.0]])


def test_norms_by_hand():
    x = np.array([3.0, -4.0, 0.0, 0.0])
    hat, r = orows.normed(x, "rms", 0.0)
    np.testing.assert_allclose(hat, x / 2.5)
    assert r == pytest.approx(0.4)
    hat, r = orows.normed(x + 7, "layer", 0.0)
    np.testing.assert_allclose(hat.mean(), 0, atol=1e-12)
    np.testing.assert_allclose((hat * hat).mean(), 1)
    np.testing.assert_allclose(orows.rows_fwd(x, "rms", 2.0, 1.0, 0.0, None, False), x / 2.5 * 2 + 1)


def test_rotation_turns_scores_into_ones_of_distances():
    rng = np.random.default_rng(0)
    q, k = rng.normal(size=(2, 16))
    freqs = rng.random(8)

    def score(i, j):
        return orows.rotate(q, orows.angles([i], (8,), freqs), True) @ orows.rotate(k, orows.angles([j], (8,), freqs), True)
    assert score(5, 3) == pytest.approx(score(105, 103))


@pytest.mark.parametrize("kind", ["none", "rms", "layer"])
@pytest.mark.parametrize("halves", [False, True])
def test_gradients_are_those_of_differences(kind, halves):
    rng = np.random.default_rng(1)
    x, dy, gain, bias = rng.normal(size=(3, 12)), rng.normal(size=(3, 12)), rng.normal(size=12), rng.normal(size=12)
    a = orows.angles(rng.integers(0, 50, size=(3, 2)), (1, 3), rng.random(4))
    dx, dgain, dbias = orows.rows_bwd(x, dy, kind, gain, 1e-3, a, halves)

    def loss(x, gain, bias):
        return (orows.rows_fwd(x, kind, gain, bias, 1e-3, a, halves) * dy).sum()
    step = 1e-5

    def slope(which, i):
        args = [x, gain, bias]
        both = []
        for sign in (1, -1):
            moved = args[which].copy()
            moved.flat[i] += sign * step
            both.append(loss(*(moved if j == which else y for j, y in enumerate(args))))
        return (both[0] - both[1]) / (2 * step)
    for which, found in ((0, dx), (1, dgain), (2, dbias)):
        if found is not None:
            np.testing.assert_allclose([slope(which, i) for i in range(found.size)], found.ravel(), rtol=1e-6, atol=1e-7)


def test_pages_hold_what_a_contiguous_cache_holds():
    rng = np.random.default_rng(2)
    B, H, Hk, Nq, d, page, per = 3, 4, 2, 3, 8, 5, 4
    k, v, q = rng.normal(size=(B, Hk, per * page, d)), rng.normal(size=(B, Hk, per * page, d)), rng.normal(size=(B, H, Nq, d))
    lens, q_lens = [20, 7, 2], [3, 1, 2]
    table = rng.permutation(B * per + 2)[:B * per].reshape(B, per)
    pool_k, pool_v = rng.normal(size=(2, B * per + 2, Hk, page, d))
    want_k, want_v = pool_k.copy(), pool_v.copy()
    for b in range(B):
        for slot in range(lens[b]):
            want_k[table[b, slot // page], :, slot % page], want_v[table[b, slot // page], :, slot % page] = k[b, :, slot], v[b, :, slot]
    got = orows.paged_append(pool_k, pool_v, table, lens, k, v, lens)
    assert (got[0] == want_k).all() and (got[1] == want_v).all()
    for causal in (False, True):
        O, LSE, A, seen = orows.paged_attention(q, *got, table, lens, q_lens, causal, 0.3)
        O2, LSE2, A2, _ = oc.cache_attention(q, lens, k, v, q_lens=q_lens, causal=causal, scale=0.3)
        np.testing.assert_allclose(O, O2)
        np.testing.assert_allclose(LSE, LSE2)
        np.testing.assert_allclose(A, A2)
        assert seen[0, 0].tolist() == ([18, 19, 20] if causal else [20, 20, 20])
    # a page that is not there takes its slots out, and nothing is written for them
    table[0, 1], table[1, 0] = -1, B * per + 2
    got = orows.paged_append(pool_k, pool_v, table, lens, k, v, lens)
    seen = orows.paged_attention(q, *got, table, lens, q_lens, False, 0.3)[3]
    assert seen[:, 0, 0].tolist() == [15, 2, 2]
