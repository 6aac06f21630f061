"""Pins of the oracle of the paged cache (``oracle/paged.py``) against facts fixed outside it:
the attention and rotation oracles, closed forms and hand-made page tables."""
import numpy as np

from oracle import paged as P
from oracle import ref
from oracle import rope


def rnd(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


def test_decode_is_a_continuation_of_one_token():
    n, Hq, Hkv, d, ps, reach = 3, 6, 2, 8, 4, 5
    q, kp, vp = rnd(1, n, Hq, d), rnd(2, 12, Hkv, ps, d), rnd(3, 12, Hkv, ps, d)
    table = np.array([[7, 2, 9, 0, 1], [3, 3, 3, 3, 3], [5, 11, -1, -1, -1]])
    rows = [17, -1, 6]
    out, mass = P.decode(q, kp, vp, table, rows)
    assert np.isnan(out[1]).all()
    for r in (0, 2):
        pages = table[r][:-(-rows[r] // ps)]
        k = np.concatenate(list(kp[pages]), 1)[:, :rows[r]]
        v = np.concatenate(list(vp[pages]), 1)[:, :rows[r]]
        # the last row is the token's own
        m = rows[r] - 1
        want, _ = ref.continue_(q[r:r + 1], k[:, m][None], v[:, m][None], k, v, m)
        np.testing.assert_allclose(out[r], want[0], rtol=0, atol=1e-12)
        assert (np.abs(out[r]) <= mass[r] + 1e-12).all()


def test_decode_leaves_out_pages_that_are_not_in_the_pool():
    q, kp, vp = rnd(1, 2, 2, 4), rnd(2, 3, 1, 4, 4), rnd(3, 3, 1, 4, 4)
    table = np.array([[1, -1, 0], [9, 3, -5]])
    out, _ = P.decode(q, kp, vp, table, [10, 12])
    both, _ = P.decode(q, kp, vp, np.array([[1, 0, 0], [0, 0, 0]]), [6, 0])
    np.testing.assert_allclose(out[0], both[0], atol=1e-14)
    assert (out[1] == 0).all() and (both[1] == 0).all()


def test_decode_without_scores_is_a_mean():
    kp, vp = rnd(2, 3, 1, 4, 4), rnd(3, 3, 1, 4, 4)
    out, _ = P.decode(np.zeros((1, 2, 4)), kp, vp, np.array([[2, 0]]), [7])
    seen = np.concatenate((vp[2, 0], vp[0, 0, :3]))
    np.testing.assert_allclose(out[0, 1], seen.mean(0), atol=1e-14)


def test_places():
    table = np.array([[4, 5], [6, -1], [0, 1]])
    at = P.places([3, 2, -1], [0, 2, 7, 8], table, 4, 7, 10)
    assert at[0] == (0, 3, 4, 3) and at[1] == (0, 4, 5, 0)
    assert at[2] == (1, 2, 6, 2) and at[3] == (1, 3, 6, 3)
    assert at[4:] == [None] * 6            # no page, an empty slot, padding
    assert P.places([7, 8, 1], None, table, 4, 7, 3) == [(0, 7, 5, 3), None, (2, 1, 0, 1)]


def test_turned():
    x, w = rnd(1, 5, 3, 8), rnd(2, 8)
    y = P.turned(x, w, 0.0, None, None)
    np.testing.assert_allclose((y / w * 1.0).__pow__(2).mean(-1), np.ones((5, 3)), atol=1e-12)
    pos = [4, 0, 9, 1, 1]
    np.testing.assert_allclose(P.turned(x, None, 0.0, pos, 1e4), rope.rotate(x, pos, 1e4), atol=0)
    z = P.turned(x, np.ones(8), 0.0, pos, 1e4)
    np.testing.assert_allclose(z[1], P.turned(x, np.ones(8), 0.0, None, None)[1], atol=1e-12)      # position 0
    np.testing.assert_allclose((z ** 2).sum(-1), np.full((5, 3), 8.0), atol=1e-11)                 # a rotation
