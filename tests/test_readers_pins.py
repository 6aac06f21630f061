"""Pins of the oracle for many readers (``oracle/readers.py``) against facts fixed
outside it: the attention oracle, closed forms, invariants and hand-made selections.
"""
import numpy as np
import pytest

from oracle import readers as O
from oracle import ref


def rnd(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


def test_shared_is_a_continuation_of_prefix_and_own_rows():
    n, S, Hq, Hkv, d, L, tcap = 3, 4, 6, 2, 8, 11, 9
    q, k, v = rnd(1, n, S, Hq, d), rnd(2, n, S, Hkv, d), rnd(3, n, S, Hkv, d)
    kc, vc, kt, vt = rnd(4, Hkv, L + 2, d), rnd(5, Hkv, L + 2, d), rnd(6, n, Hkv, tcap, d), rnd(7, n, Hkv, tcap, d)
    lens = [0, 5, -1]
    out, mass = O.shared(q, k, v, kc, vc, L, kt, vt, lens)
    assert np.isnan(out[2]).all()
    for r in (0, 1):
        kk = np.concatenate((kc[:, :L], kt[r, :, :lens[r]]), 1)
        vv = np.concatenate((vc[:, :L], vt[r, :, :lens[r]]), 1)
        want, _ = ref.continue_(q[r], k[r], v[r], kk, vv, L + lens[r])
        np.testing.assert_allclose(out[r], want, rtol=0, atol=1e-12)
        assert (np.abs(out[r]) <= mass[r] + 1e-12).all()


def test_shared_without_scores_is_a_mean():
    q, k = np.zeros((1, 2, 2, 4)), rnd(1, 1, 2, 1, 4)
    v, vc, vt = rnd(2, 1, 2, 1, 4), rnd(3, 1, 3, 4), rnd(4, 1, 1, 5, 4)
    out, _ = O.shared(q, k, v, rnd(5, 1, 3, 4), vc, 3, rnd(6, 1, 1, 5, 4), vt, [2])
    seen = np.concatenate((vc[0], vt[0, 0, :2]))
    np.testing.assert_allclose(out[0, 0, 0], np.concatenate((seen, v[0, :1, 0])).mean(0), atol=1e-14)
    np.testing.assert_allclose(out[0, 1, 1], np.concatenate((seen, v[0, :, 0])).mean(0), atol=1e-14)


def test_weigh_gives_each_row_one():
    S, Hq, Hkv, d, L = 5, 6, 3, 8, 7
    w = O.weigh(rnd(1, S, Hq, d), rnd(2, S, Hkv, d), rnd(3, Hkv, L + 4, d), L, np.zeros((Hkv, L + 8)))
    np.testing.assert_allclose(w.sum(1), S * Hq / Hkv, rtol=1e-13)
    assert not w[:, L + S:].any()


def test_weigh_without_scores():
    """Q = 0: token i gives each of its L + i + 1 keys the same."""
    S, L = 3, 4
    w = O.weigh(np.zeros((S, 2, 8)), rnd(2, S, 1, 8), rnd(3, 1, 9, 8), L, np.full((1, 9), 0.5))
    give = [2.0 / (L + i + 1) for i in range(S)]
    want = [0.5 + sum(give)] * (L + 1) + [0.5 + give[1] + give[2], 0.5 + give[2]] + [0.5] * 2
    np.testing.assert_allclose(w[0], want, rtol=1e-14)


def test_weigh_two_keys():
    """Scores (0, 1) on the cached key and the token's own: weights 1 - s, s of the logistic of 1."""
    q = np.array([[[1.0, 0, 0, 0]]])
    w = O.weigh(q, np.array([[[1.0, 0, 0, 0]]]), np.zeros((1, 2, 4)), 1, np.zeros((1, 2)), scale=1.0)
    s = 1 / (1 + np.exp(-1.0))
    np.testing.assert_allclose(w[0], [1 - s, s], rtol=1e-15)


@pytest.mark.parametrize("w,keep,first,last,want", [
    ([3, 1, 2, 5, 4], 2, 0, 0, [3, 4]),
    ([3, 1, 2, 5, 4], 3, 1, 0, [0, 3, 4]),
    ([3, 1, 2, 5, 4], 3, 0, 1, [0, 3, 4]),
    ([9, 1, 2, 2, 2, 0], 3, 1, 1, [0, 2, 5]),             # the lower of equal weights
    ([1, 1, 1, 1], 2, 0, 0, [0, 1]),
    ([0.0, -0.0, -0.0, 0.0], 2, 0, 0, [0, 1]),            # zeros are equal
    ([1, float("nan"), float("inf"), 2], 2, 0, 0, [1, 2]),
    ([1, 2, 3], 3, 0, 0, [0, 1, 2]),
    ([1, 2, 3], 0, 0, 0, []),
])
def test_evict(w, keep, first, last, want):
    assert O.evict(np.array([w], dtype=float), len(w), keep, first, last).tolist() == [want]
