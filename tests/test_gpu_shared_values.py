"""kvr_continue_shared where scores are far apart and values large, against the fp64 oracle.

The descriptor's scale is ln 2, so that q . k is a score in log2 units: component 0 of a
key says how far its weight is raised for a query whose component 0 is 1.

Tolerance, derived: that of test_gpu_shared.py (each 16-bit weight and each output rounded
once, fp32 scores, exponentials and sums), which counts the raised scores in sum |q k|.
"""
import math

import numpy as np
import pytest
import torch

from harness import workloads as W
from oracle import readers as O
from paper_2606_13361_amd import kvr

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
DEV = "cuda"
LN2 = math.log(2.0)
Q = (32, 8, 128)

# heads, readers, new tokens, prefix, longest own rows, room for own rows: calls of each way
WAYS16 = {
    "one_launch": (Q, 2, 1, 470, 60, 64),
    "by_keys": (Q, 2, 1, 12000, 60, 700),
    "by_rows": ((8, 2, 128), 17, 1, 3001, 650, 1400),
    "by_rows_2": ((4, 1, 128), 64, 1, 6301, 40, 70),
    "own_by_rows": ((8, 2, 128), 9, 8, 1003, 645, 1300),
    "one_launch_64": ((16, 2, 64), 2, 2, 470, 60, 64),
    "by_rows_64": ((16, 2, 64), 9, 2, 3001, 650, 1400),
    "by_rows_2_64": ((8, 2, 64), 40, 1, 10001, 40, 50),
}
WAYS32 = {
    "one_launch": (Q, 2, 1, 90, 60, 64),
    "by_keys": (Q, 2, 1, 6000, 60, 700),
    "by_keys_2": ((8, 1, 64), 11, 3, 2100, 640, 1300),
}
WAYS = [(dt, w) for dt in (BF16, F16) for w in WAYS16] + [(F32, w) for w in WAYS32]
EACH_WAY = pytest.mark.parametrize("dt,way", WAYS, ids=lambda x: str(x).replace("torch.", ""))


class Call:
    """One call: q, k, v [n, S, heads, d], prefix kc, vc, own rows kt, vt of lens[r] rows; scores' noise has a
    standard deviation of 1.4 (d = 128) and 1 (64) log2 units."""

    def __init__(self, dt, way, seed=0):
        self.heads, n, S, L, most, tcap = (WAYS32 if dt == F32 else WAYS16)[way]
        Hq, Hkv, d = self.heads
        self.dt, self.n, self.S, self.L, self.tcap = dt, n, S, L, tcap
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g)
        self.lens = [most * i // max(1, n - 1) for i in range(n)]
        self.q, self.k, self.v = r(n, S, Hq, d) / 8, r(n, S, Hkv, d), r(n, S, Hkv, d)
        self.kc, self.vc = r(Hkv, L, d), r(Hkv, L, d)
        self.kt, self.vt = r(n, Hkv, tcap, d), r(n, Hkv, tcap, d)
        for x in (self.q, self.k, self.kc, self.kt):
            x[..., 0] = 0.0
        self.g = g

    def run(self):
        """The outputs, on the CPU; every tensor of the call as its type holds it."""
        for x in ("q", "k", "v", "kc", "vc", "kt", "vt"):
            setattr(self, x, getattr(self, x).to(self.dt))
        desc = kvr.make_desc(*self.heads, self.dt, self.L, scale=LN2)
        out = torch.zeros(self.q.shape, dtype=self.dt, device=DEV)
        lens = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        ws = kvr.workspace_for_shared(desc, self.L, self.n, self.S, self.tcap)
        t = [getattr(self, x).to(DEV).contiguous() for x in ("q", "k", "v", "kc", "vc", "kt", "vt")]
        kvr.kvr_continue_shared(desc, *t[:5], self.L, t[5], t[6], lens, out, ws)
        torch.cuda.synchronize()
        return out.cpu()

    def exact(self):
        """(out, what each may be off by)"""
        scale = float(np.float32(LN2))
        q, k, v, kc, vc, kt, vt = (O._f64(getattr(self, x)) for x in ("q", "k", "v", "kc", "vc", "kt", "vt"))
        out, mass = O.shared(q, k, v, kc, vc, self.L, kt, vt, self.lens, scale=scale)
        Hq, Hkv, d = self.heads
        top = np.maximum(np.maximum(np.abs(kc).max(1), np.abs(kt).max((0, 2))), np.abs(k).max((0, 1)))
        dots = (np.abs(q) * np.repeat(top, Hq // Hkv, 0)).sum(-1) * scale
        n_keys = self.L + max(self.lens) + self.S
        half = torch.finfo(self.dt).eps / 2
        rel = 2 * (d + 2) * 2.0 ** -24 * dots + 2.0 ** -22 + 2 * n_keys * 2.0 ** -24
        return out, 1.1 * (half * np.abs(out) + mass * ((0.0 if self.dt == F32 else half) + rel[..., None]))

    def check(self):
        got = O._f64(self.run())
        want, far = self.exact()
        err = np.abs(got - want)
        worst = np.unravel_index(int(np.argmax(np.nan_to_num(err / far, nan=np.inf))), err.shape)
        assert (err <= far).all(), "at %s: %.6g, exact %.6g, allowed %.3g" % (worst, got[worst], want[worst], far[worst])


# ------------------------------------------------------------ a key far above all others
@pytest.mark.parametrize("below", [18, 24.5, 25.5])
@EACH_WAY
def test_weights_far_below_one_that_adds_nothing(dt, way, below):
    """The first key is `below` log2 units above the others and its value is zero: the output is the others',
    a small one.  Then the same with that key among a reader's own rows, and among the new ones."""
    for place in ("prefix", "own", "new"):
        c = Call(dt, way)
        c.q[...], c.q[..., 0] = 0.0, 1.0
        c.v[...], c.vc[...], c.vt[...] = 512.0, 512.0, 512.0
        c.v[..., 1::2], c.vc[..., 1::2], c.vt[..., 1::2] = -1536.0, -1536.0, -1536.0
        k, v = {"prefix": (c.kc[:, 0], c.vc[:, 0]), "own": (c.kt[:, :, 0], c.vt[:, :, 0]), "new": (c.k[:, 0], c.v[:, 0])}[place]
        k[..., 0], v[...] = below, 0.0
        c.check()


# ------------------------------------------------------------ large values
@pytest.mark.parametrize("dt,way", [x for x in WAYS if x[0] != F16], ids=lambda x: str(x).replace("torch.", ""))
def test_large_values_stay_finite(dt, way):
    """Values of 2^110 and keys that raise their weights by up to 2^55, over which a sum of weights above 1
    times such values would pass the largest fp32 number."""
    c = Call(dt, way, seed=1)
    c.q[..., 0] = 1.0
    for k in (c.kc, c.kt, c.k.transpose(1, 2)):
        at = torch.randint(0, 40, k.shape[:-1], generator=c.g) == 0
        k[..., 0] = torch.where(at, torch.randint(0, 56, k.shape[:-1], generator=c.g).float(), torch.zeros(()))
    for v in (c.v, c.vc, c.vt):
        v *= 2.0 ** 110
    c.check()


# ------------------------------------------------------------ the bar between two GPU results
@pytest.mark.parametrize("kind", ["scaled", "sink", "tile_end", "rising"])
@pytest.mark.parametrize("n", [1, 12])
def test_peaky_rows_agree_with_a_prefill(kind, n):
    """The rows of a prefill of prefix and new tokens, at 2e-3 and one output ulp, the bar that a
    continuation is held to on these inputs; n readers with the same tokens (12: two row tiles a wave)."""
    L, S, sh = 1500, 24, W.QWEN
    q, k, v = (x.to(DEV) for x in W.stress(kind, L + S, sh, seed=3))
    full = torch.empty_like(q)
    desc = kvr.make_desc(sh.n_q_heads, sh.n_kv_heads, sh.head_dim, sh.dtype, L + S)
    kc, vc = (torch.zeros((sh.n_kv_heads, L + S, sh.head_dim), dtype=sh.dtype, device=DEV) for _ in range(2))
    kvr.kvr_prefill(desc, q, k, v, L + S, full, kc, vc)
    new = [x[L:].expand(n, *x[L:].shape).contiguous() for x in (q, k, v)]
    out = torch.empty_like(new[0])
    kvr.kvr_continue_shared(desc, *new, kc, vc, L, None, None, torch.zeros(n, dtype=torch.int32, device=DEV), out,
                            kvr.workspace_for_shared(desc, L, n, S, 0))
    want = full[L:].double().cpu()
    far = 2e-3 + 2.0 ** -7 * want.abs()
    assert float(((out.double().cpu() - want).abs() - far).max()) <= 0.0


# ------------------------------------------------------------ references that move
@EACH_WAY
@pytest.mark.parametrize("seed", [2, 3])
def test_weights_that_rise_in_late_stages(dt, way, seed):
    """One key in 32 is 0 to 140 log2 units above the others, in every range, among own and new rows: references move
    while sums are not zero, partials of very different ones are joined.  Rows of a tile see them at full
    height, in part, not at all and upside down."""
    c = Call(dt, way, seed=seed)
    heights = torch.tensor([0.0, 10.0, 18.0, 40.0, 70.0, 90.0, 139.0, 140.0])
    for k in (c.kc, c.kt, c.k.transpose(1, 2)):
        at = torch.randint(0, 32, k.shape[:-1], generator=c.g) == 0
        k[..., 0] = torch.where(at, heights[torch.randint(0, 8, k.shape[:-1], generator=c.g)], torch.zeros(()))
    part = torch.tensor([0.0, 0.125, 0.25, 0.5, 1.0, -0.5])
    c.q[..., 0] = part[torch.randint(0, 6, c.q.shape[:-1], generator=c.g)]
    c.check()


# ------------------------------------------------------------ infinities that are seen
@EACH_WAY
def test_an_infinite_value_in_the_last_row(dt, way):
    """Infinite values in the last row of the prefix and of each reader's own rows, where a range ends inside a
    stage: infinite outputs, of that sign, in those components, and the others as without them."""
    c = Call(dt, way, seed=4)
    want = c.run().float()
    c.vc[:, c.L - 1, 3] = float("inf")
    c.vc[:, c.L - 1, 33] = -float("inf")
    for i, ln in enumerate(c.lens):
        if ln:
            c.vt[i, :, ln - 1, 7] = -float("inf")
            want[i, ..., 7] = -float("inf")
    want[..., 3], want[..., 33] = float("inf"), -float("inf")
    assert torch.equal(c.run().float(), want)
