"""Oracle of the operators for many readers of one cached document: attention over
a shared prefix and each reader's own rows, accumulated attention weight, and
eviction by it.  Plain fp64 numpy, straight from the definitions.

TEST INFRASTRUCTURE ONLY, as the rest of this package: the product path never
imports it.
"""
import numpy as np


def _f64(x):
    import torch
    if isinstance(x, torch.Tensor):
        return x.detach().cpu().double().numpy()
    return np.asarray(x, dtype=np.float64)


def softmax(s):
    with np.errstate(invalid="ignore"):
        e = np.exp(s - s.max(axis=-1, keepdims=True))
        return e / e.sum(axis=-1, keepdims=True)


def shared(q, k, v, kc, vc, L, kt, vt, lens, scale=None):
    """q [n, S, Hq, d], k / v [n, S, Hkv, d] (rotated where the caller wants it),
    kc / vc [Hkv, cap, d], kt / vt [n, Hkv, tcap, d] or None, lens [n].

    Returns (out, mass): out [n, S, Hq, d], NaN for a reader with a negative length;
    mass = sum_j p_j |v_j|, what a relative error of the weights may move an output by.
    """
    q, k, v = _f64(q), _f64(k), _f64(v)
    n, S, Hq, d = q.shape
    Hkv = k.shape[2]
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    out, mass = np.full(q.shape, np.nan), np.zeros(q.shape)
    for r in range(n):
        ln = int(lens[r])
        if ln < 0:
            continue
        for g in range(Hkv):
            ks, vs = [], []
            if L:
                ks.append(_f64(kc[g, :L]))
                vs.append(_f64(vc[g, :L]))
            if ln:
                ks.append(_f64(kt[r, g, :ln]))
                vs.append(_f64(vt[r, g, :ln]))
            for i in range(S):
                keys = np.concatenate(ks + [k[r, :i + 1, g]])
                vals = np.concatenate(vs + [v[r, :i + 1, g]])
                p = softmax(q[r, i, g * G:(g + 1) * G] @ keys.T * scale)
                out[r, i, g * G:(g + 1) * G] = p @ vals
                mass[r, i, g * G:(g + 1) * G] = p @ np.abs(vals)
    return out, mass


def weigh(q, k, kc, L, weight, scale=None):
    """q [S, Hq, d], k [S, Hkv, d], kc [Hkv, cap, d]; weight [Hkv, cap] before the
    call.  Returns weight after it, fp64."""
    q, k, kc, w = _f64(q), _f64(k), _f64(kc), _f64(weight).copy()
    S, Hq, d = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    for g in range(Hkv):
        keys = np.concatenate([kc[g, :L], k[:, g]])
        for i in range(S):
            p = softmax(q[i, g * G:(g + 1) * G] @ keys[:L + i + 1].T * scale)
            w[g, :L + i + 1] += p.sum(axis=0)
    return w


def evict(weight, L, n_keep, n_first, n_last):
    """The kept rows of each kv head, ascending: [Hkv, n_keep]."""
    w = _f64(weight)
    rows = []
    for g in range(w.shape[0]):
        between = range(n_first, L - n_last)
        # a weight that is no number counts as the largest
        order = sorted(between, key=lambda j: (0 if np.isnan(w[g, j]) else 1, -w[g, j] if not np.isnan(w[g, j]) else 0.0, j))
        rows.append(sorted(list(range(n_first)) + list(range(L - n_last, L)) + order[:n_keep - n_first - n_last]))
    return np.asarray(rows, dtype=np.int64).reshape(w.shape[0], n_keep)
