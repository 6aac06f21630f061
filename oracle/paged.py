"""Oracle of the paged cache: head norms with rotation, new tokens into pages, and
attention of one token of each sequence over its pages.  Plain fp64 numpy, straight
from the definitions.

TEST INFRASTRUCTURE ONLY, as the rest of this package: the product path never
imports it.
"""
import numpy as np

from oracle import layer
from oracle import rope
from oracle.readers import _f64, softmax


def turned(x, w, eps, pos, base):
    """x [T, heads, d], normalized with weights w (None: not), rotated at positions pos
    (base None: not)."""
    y = _f64(x) if w is None else layer.rmsnorm(_f64(x), _f64(w), eps)
    return y if base is None else rope.rotate(y, pos, base)


def places(lens, cu, table, ps, n_pages, T):
    """(sequence, row, page, slot) of each token, None where it has no place."""
    n, reach = table.shape
    out = [None] * T
    for r in range(n):
        a, b = (r, r + 1) if cu is None else (int(cu[r]), int(cu[r + 1]))
        for t in range(a, min(b, T)):
            row = int(lens[r]) + t - a
            if lens[r] < 0 or row >= reach * ps:
                continue
            page = int(table[r, row // ps])
            if 0 <= page < n_pages:
                out[t] = (r, row, page, row % ps)
    return out


def decode(q, kp, vp, table, rows, scale=None):
    """q [n, Hq, d], kp / vp [n_pages, Hkv, ps, d], table [n, max_pages], rows [n]: rows that
    each sequence's token sees (negative: no part).

    Returns (out, mass): out [n, Hq, d], NaN where a sequence takes no part, zeros where it
    has no row in any page; mass = sum_j p_j |v_j|.
    """
    q, kp, vp, table = _f64(q), _f64(kp), _f64(vp), np.asarray(table)
    n, Hq, d = q.shape
    n_pages, Hkv, ps, _ = kp.shape
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, mass = np.full(q.shape, np.nan), np.zeros(q.shape)
    for r in range(n):
        m = int(rows[r])
        if m < 0:
            continue
        keys, vals = np.zeros((Hkv, 0, d)), np.zeros((Hkv, 0, d))
        for j in range(-(-m // ps)):
            if 0 <= table[r, j] < n_pages:
                take = min(ps, m - j * ps)
                keys = np.concatenate((keys, kp[table[r, j], :, :take]), 1)
                vals = np.concatenate((vals, vp[table[r, j], :, :take]), 1)
        if keys.shape[1] == 0:
            out[r] = 0.0
            continue
        p = softmax(np.matmul(q[r].reshape(Hkv, G, d), keys.transpose(0, 2, 1)) * scale)
        out[r] = np.matmul(p, vals).reshape(Hq, d)
        mass[r] = np.matmul(p, np.abs(vals)).reshape(Hq, d)
    return out, mass
