"""kvr_continue_shared against the fp64 oracle: every output of every reader, the
readers' caches bit for bit, and what must stay as it was.

Tolerance, derived: an output is sum p v / sum p.  In the 16-bit types each weight is
rounded once (half a step, h = eps / 2) and the output once: h (|out| + mass), mass =
sum p |v|.  fp32 arithmetic adds, relative to mass: a score of d products differs by at
most (d + 2) 2^-24 sum |q k| scale, twice (numerator and denominator), 2^x by 2^-22, and
sums of n terms by n 2^-24 each, twice.  Second-order terms: a tenth more.
"""
import numpy as np
import pytest
import torch

from oracle import readers as O
from paper_2606_13361_amd import kvr

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
DEV = "cuda"
SENTINEL = 7.0


def bound(dt, out, mass, q, keys_abs, n_keys):
    """keys_abs: the largest |k| of each head-dim index, [Hkv, d]."""
    h = torch.finfo(dt).eps / 2 if dt != F32 else 0.0
    G = q.shape[2] // keys_abs.shape[0]
    d = q.shape[3]
    dots = (np.abs(q) * np.repeat(keys_abs, G, 0)).sum(-1) / np.sqrt(d)           # [n, S, Hq]
    rel = 2 * (d + 2) * 2.0 ** -24 * dots + 2.0 ** -22 + 2 * n_keys * 2.0 ** -24
    last = torch.finfo(dt).eps / 2 * np.abs(out)
    return 1.1 * (last + mass * (h + rel[..., None]))


class Batch:
    """Inputs of one call; rows behind every valid one hold NaN."""

    def __init__(self, dt, heads, n, S, L, lens, tcap, cap=None, seed=0, rope_base=None, pos0=None):
        Hq, Hkv, d = heads
        g = torch.Generator().manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g).to(dt)
        cap = L + 5 if cap is None else cap
        self.dt, self.heads, self.n, self.S, self.L, self.lens, self.tcap = dt, heads, n, S, L, list(lens), tcap
        self.q, self.k, self.v = r(n, S, Hq, d), r(n, S, Hkv, d), r(n, S, Hkv, d)
        nan = lambda *s: torch.full(s, float("nan"), dtype=dt)
        self.kc, self.vc, self.kt, self.vt = nan(Hkv, cap, d), nan(Hkv, cap, d), nan(n, Hkv, tcap, d), nan(n, Hkv, tcap, d)
        self.kc[:, :L], self.vc[:, :L] = r(Hkv, L, d), r(Hkv, L, d)
        for i, ln in enumerate(self.lens):
            m = min(max(ln, 0), tcap)
            self.kt[i, :, :m], self.vt[i, :, :m] = r(Hkv, m, d), r(Hkv, m, d)
        self.pos0 = L if pos0 is None else pos0
        self.base = rope_base
        self.desc = kvr.make_desc(Hq, Hkv, d, dt, cap)

    def active(self, append):
        return [0 <= ln <= self.tcap - (self.S if append else 0) for ln in self.lens]

    def gpu(self):
        t = {x: getattr(self, x).to(DEV) for x in ("q", "k", "v", "kc", "vc", "kt", "vt")}
        t["len"] = torch.tensor(self.lens, dtype=torch.int32, device=DEV)
        t["out"] = torch.full(self.q.shape, SENTINEL, dtype=self.dt, device=DEV)
        t["ws"] = kvr.workspace_for_shared(self.desc, self.L, self.n, self.S, self.tcap)
        t["ws"].fill_(255)      # NaN everywhere
        t["rope"] = (kvr.RopeTable(self.heads[2], self.pos0 + self.tcap + self.S, base=self.base)
                     if self.base else None)
        return t

    def call(self, t, append=True, **kw):
        kvr.kvr_continue_shared(self.desc, t["q"], t["k"], t["v"], t["kc"], t["vc"], self.L, t["kt"], t["vt"], t["len"],
                                t["out"], t["ws"], rope=t["rope"], pos0=self.pos0, append=append, **kw)

    def rotated(self, t):
        """q and k as the library rotates rows at these positions."""
        if not self.base:
            return self.q, self.k
        q, k = self.q.to(DEV), self.k.to(DEV)
        for i, ln in enumerate(self.lens):
            if ln >= 0:
                kvr.kvr_rope_apply(self.desc, t["rope"], q[i], self.pos0 + ln)
                kvr.kvr_rope_apply(self.desc, t["rope"], k[i], self.pos0 + ln)
        return q.cpu(), k.cpu()

    def check(self, t, append=True):
        torch.cuda.synchronize()
        on = self.active(append)
        q, k = self.rotated(t)
        lens = [ln if a else -1 for ln, a in zip(self.lens, on)]
        out, mass = O.shared(q, k, self.v, self.kc, self.vc, self.L, self.kt, self.vt, lens)
        keys = np.nan_to_num(np.abs(O._f64(self.kc))).max(1, initial=0.0)
        keys = np.maximum(keys, np.nan_to_num(np.abs(O._f64(self.kt))).max((0, 2), initial=0.0))
        keys = np.maximum(keys, np.nan_to_num(np.abs(O._f64(k))).max((0, 1)))
        b = bound(self.dt, out, mass, np.abs(O._f64(q)), keys, self.L + max(max(lens), 0) + self.S)
        got = t["out"].cpu()
        for i, a in enumerate(on):
            if not a:
                assert torch.equal(got[i], torch.full_like(got[i], SENTINEL)), "row of reader %d written" % i
                continue
            err = np.abs(O._f64(got[i]) - out[i])
            assert (err <= b[i]).all(), "reader %d: %.3g, allowed %.3g there" % (
                i, np.nan_to_num(err, nan=np.inf).max(), b[i].flat[int(np.argmax(np.nan_to_num(err - b[i], nan=np.inf)))])
        # the readers' caches, bit for bit
        bits = {F32: torch.int32}.get(self.dt, torch.int16)
        for name, new in (("kt", k), ("vt", self.v)):
            want = getattr(self, name).clone()
            for i, a in enumerate(on):
                if a and append:
                    want[i, :, self.lens[i]:self.lens[i] + self.S] = new[i].transpose(0, 1)
            assert torch.equal(t[name].cpu().view(bits), want.view(bits)), name
        return got


def run(b, append=True):
    t = b.gpu()
    b.call(t, append)
    return b.check(t, append)


Q = (32, 8, 128)
PARITY = [
    # dt, heads, n, S, L, lens, tcap
    (BF16, Q, 1, 1, 0, [0], 1),                                   # one token, nothing cached
    (BF16, Q, 1, 1, 1, [0], 4),
    (BF16, Q, 2, 1, 255, [1, 13], 64),
    (BF16, Q, 9, 1, 300, [-1, 0, 31, 32, 33, 64, 127, 128, 129], 140),
    (F16, Q, 5, 4, 129, [0, 5, 28, 60, 61], 64),                  # one full tail
    (BF16, Q, 3, 33, 31, [0, 7, 40], 80),                         # new rows over a stage, rows over a tile
    (BF16, Q, 2, 70, 33, [3, 90], 200),
    (BF16, Q, 64, 1, 513, list(range(0, 128, 2)), 129),           # four row tiles
    (BF16, (8, 8, 128), 33, 1, 127, list(range(33)), 40),         # G = 1
    (F16, (12, 3, 128), 7, 3, 200, [0, 1, 2, 50, -1, 33, 17], 60),   # 3 kv heads
    (BF16, (64, 8, 128), 3, 5, 96, [9, 100, 0], 110),             # G = 8
    (BF16, (128, 2, 128), 2, 2, 65, [3, 4], 8),                   # G = 64
    (BF16, (16, 2, 64), 6, 2, 1000, [300, 5, 0, 64, 33, 99], 310),
    (F16, (8, 2, 64), 40, 1, 333, list(range(40)), 50),
    (F32, (16, 2, 64), 3, 5, 245, [0, 40, 77], 96),
    (F32, Q, 2, 1, 100, [0, 21], 40),
    (F32, (6, 3, 128), 5, 17, 49, [0, 1, 15, 16, 17], 40),
    (BF16, (5, 5, 64), 2, 1, 0, [700, 3], 701),                   # no prefix, split own rows
    # one launch up to 20 stages (fp32: 10) of 32 (16) prefix and own rows, up to 16 rows a reader and kv head
    (BF16, Q, 3, 4, 320, [320, 0, 314], 320), (BF16, Q, 3, 4, 321, [320, 0, 314], 320), (F16, Q, 3, 5, 320, [315, 0, 9], 320),
    (F32, Q, 3, 4, 80, [80, 0, 70], 80), (F32, Q, 3, 4, 81, [80, 0, 70], 80), (BF16, (8, 8, 64), 2, 16, 30, [0, 9], 40),
    (F16, (8, 8, 64), 2, 17, 30, [0, 9], 40), (BF16, Q, 1, 1, 0, [639], 640), (BF16, Q, 300, 1, 40, list(range(300)), 301),
    # the same readers as before, in items
    (BF16, Q, 1, 1, 0, [0], 700), (BF16, Q, 1, 1, 1, [0], 700), (BF16, Q, 9, 1, 300, [-1, 0, 31, 32, 33, 64, 127, 128, 129], 800),
    (F16, Q, 5, 4, 129, [0, 5, 28, 60, 61], 700), (BF16, (8, 8, 128), 33, 1, 127, list(range(33)), 700),
    (F16, (12, 3, 128), 7, 3, 200, [0, 1, 2, 50, -1, 33, 17], 700), (F32, Q, 2, 1, 100, [0, 21], 400),
    # rows of a kv head where a prefix item has 16, 64 and 128 of them, and one more
    (BF16, Q, 4, 1, 700, [1, 2, 3, 4], 30), (BF16, Q, 16, 1, 700, list(range(16)), 30), (BF16, Q, 17, 1, 700, list(range(17)), 30),
    (BF16, Q, 32, 1, 700, list(range(32)), 40), (BF16, Q, 33, 1, 700, list(range(33)), 40),
    (F32, (8, 8, 64), 16, 1, 300, list(range(16)), 30), (F32, (8, 8, 64), 33, 1, 300, list(range(33)), 40),
    # as many rows and keys as two row tiles at a time need: 16-bit, own rows by keys and by rows; fp32
    (BF16, (4, 1, 128), 64, 1, 6300, list(range(64)), 70), (BF16, (4, 1, 128), 32, 1, 12321, [7] * 32, 9),
    (BF16, (4, 1, 128), 33, 1, 12000, [7] * 33, 9), (F16, (4, 1, 64), 40, 1, 9999, list(range(40)), 50),
    (BF16, (4, 1, 128), 9, 8, 5600, [0, 1, 600, 31, 32, 33, -1, 64, 100], 700),
    (F32, (8, 1, 64), 16, 2, 2100, list(range(16)), 20), (F32, (8, 1, 64), 11, 3, 2000, [5 * i for i in range(11)], 60),
    (F32, (4, 1, 128), 35, 1, 3800, [3] * 35, 9),
    (BF16, (4096, 4096, 64), 1, 1, 5, [3], 8), (F16, (4096, 1, 64), 1, 1, 5, [3], 8),      # the most heads
]


@pytest.mark.parametrize("append", [True, False], ids=["append", "keep"])
@pytest.mark.parametrize("rope", [None, 1e4], ids=["plain", "rope"])
@pytest.mark.parametrize("case", PARITY, ids=lambda c: "%s-%s-n%d-S%d-L%d" % (str(c[0])[6:], "x".join(map(str, c[1])), *c[2:5]))
def test_parity(case, rope, append):
    run(Batch(*case, rope_base=rope, seed=len(case[5])), append)


# prefixes of a call in one launch and of one in items and a merge
BOTH = pytest.mark.parametrize("L", [64, 700])


@BOTH
def test_no_tails(L):
    """First tokens of readers that have no rows yet and keep none: no tail tensors."""
    b = Batch(BF16, Q, 3, 4, L, [0, 0, 0], 0)
    t = b.gpu()
    t["kt"] = t["vt"] = None
    b.call(t, append=False)
    t["kt"], t["vt"] = b.kt, b.vt
    b.check(t, append=False)


@BOTH
def test_positions_go_on_from_pos0(L):
    """A prefix that rows were evicted from: positions are not row numbers."""
    run(Batch(BF16, Q, 2, 2, L, [5, 40], 64, rope_base=1e6, pos0=4000))


@BOTH
def test_readers_that_do_not_fit_take_no_part(L):
    b = Batch(BF16, Q, 6, 3, L, [-1, 30, 29, 32, 33, -2 ** 31], 32)
    assert b.active(True) == [False, False, True, False, False, False]
    assert b.active(False) == [False, True, True, True, False, False]
    run(b, True)
    run(b, False)


@BOTH
@pytest.mark.parametrize("dt", [BF16, F16, F32], ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_later_tokens_do_not_reach_earlier_ones(dt, bad, L):
    """Token 2 of reader 1 holds no numbers: the tokens before it, and other readers, are as without it."""
    b = Batch(dt, (16, 4, 64), 3, 4 if L < 700 else 5, L, [0, 9, 40], 64, rope_base=1e4)
    good = run(b)
    b.k[1, 2], b.v[1, 2] = bad, bad
    t = b.gpu()
    b.call(t)
    torch.cuda.synchronize()
    got = t["out"].cpu()
    assert torch.equal(got[0], good[0]) and torch.equal(got[2], good[2])
    assert torch.equal(got[1, :2], good[1, :2])
    assert not torch.isfinite(got[1, 2:].float()).any()


@BOTH
def test_far_rows(L):
    """Offsets past 2^32 bytes: the last kv head's prefix, the last reader's rows."""
    Hq, Hkv, d = 16, 8, 128
    cap = 2_400_000                       # 8 x 2.4M x 256 bytes = 4.9 GB
    b = Batch(BF16, (Hq, Hkv, d), 3, 1, L, [3, 0, 20], 24)
    t = b.gpu()
    big = torch.zeros((Hkv, cap, d), dtype=BF16, device=DEV)
    big[:, :L] = t["kc"][:, :L]
    t["kc"] = big
    big = torch.zeros((Hkv, cap, d), dtype=BF16, device=DEV)
    big[:, :L] = t["vc"][:, :L]
    t["vc"] = big
    b.desc = kvr.make_desc(Hq, Hkv, d, BF16, cap)
    b.call(t)
    b.check(t)
    del t, big
    b = Batch(BF16, (Hq, Hkv, d), 3, 1, L, [3, -1, 20], 24)
    t = b.gpu()
    tcap = 900_000                        # 3 readers x 8 heads x 0.9M x 256 bytes = 5.5 GB
    kt, vt = (torch.zeros((3, Hkv, tcap, d), dtype=BF16, device=DEV) for _ in range(2))
    kt[:, :, :24], vt[:, :, :24] = t["kt"], t["vt"]
    small = t["kt"], t["vt"]
    t["kt"], t["vt"] = kt, vt
    t["ws"] = kvr.workspace_for_shared(b.desc, b.L, b.n, b.S, tcap)
    b.call(t)
    t["kt"], t["vt"] = kt[:, :, :24], vt[:, :, :24]
    b.check(t)


@BOTH
def test_same_bits_twice_and_on_another_stream(L):
    b = Batch(BF16, Q, 20, 2, L, list(range(0, 200, 10)), 210, rope_base=1e6)
    one = run(b)
    s = torch.cuda.Stream()
    t = b.gpu()
    torch.cuda.synchronize()
    b.call(t, stream=s)
    s.synchronize()
    assert torch.equal(t["out"].cpu(), one)
    with torch.cuda.stream(s):
        b.call(t)
    s.synchronize()
    assert torch.equal(t["out"].cpu(), one)


@BOTH
def test_one_graph_serves_a_decode(L):
    """Lengths, rows and outputs of a captured step follow the tensors: eager steps give the same bits,
    with the program's own work between the replays."""
    b = Batch(BF16, Q, 7, 1, L, [0, 3, 30, 31, -1, 60, 5], 70, rope_base=1e6)
    t, e = b.gpu(), b.gpu()
    t["step"] = (t["len"] >= 0).int()
    b.call(t)                                   # warm up
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        b.call(t)
    gen = torch.Generator().manual_seed(9)
    for step in range(6):
        for x in ("q", "k", "v"):
            new = torch.randn(t[x].shape, generator=gen).to(BF16)
            t[x].copy_(new)
            e[x].copy_(new)
        g.replay()
        b.call(e)
        t["len"] += t["step"]
        e["len"] += t["step"]
        float(t["out"].float().nan_to_num().sum())      # work of the program's own, and a wait
        for x in ("out", "kt", "vt"):
            assert torch.equal(t[x].view(torch.int16), e[x].view(torch.int16)), (step, x)


@BOTH
def test_two_streams_with_a_workspace_each(L):
    b, c = (Batch(BF16, Q, 16, 1, L, [10 * i for i in range(16)], 160, seed=s) for s in (1, 2))
    t, u = b.gpu(), c.gpu()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(4):
        b.call(t, append=False, stream=s1)
        c.call(u, append=False, stream=s2)
    torch.cuda.synchronize()
    b.check(t, append=False)
    c.check(u, append=False)


@BOTH
def test_agrees_with_single_continuations(L):
    """Each reader alone, over its own copy of prefix and rows, through kvr_continue: within both calls' bounds."""
    b = Batch(BF16, Q, 4, 3, L, [0, 17, 64, 100], 128)
    got = run(b)
    Hq, Hkv, d = b.heads
    for i, ln in enumerate(b.lens):
        n = b.L + ln
        kc = torch.cat((b.kc[:, :b.L], b.kt[i, :, :ln]), 1).to(DEV).contiguous()
        vc = torch.cat((b.vc[:, :b.L], b.vt[i, :, :ln]), 1).to(DEV).contiguous()
        desc = kvr.make_desc(Hq, Hkv, d, BF16, n)
        out = torch.empty((b.S, Hq, d), dtype=BF16, device=DEV)
        kvr.kvr_continue(desc, b.q[i].to(DEV), b.k[i].to(DEV), b.v[i].to(DEV), kc, vc, n, b.S, out,
                         kvr.workspace_for(desc, n, b.S))
        want, mass = O.shared(b.q[i:i + 1], b.k[i:i + 1], b.v[i:i + 1], kc.cpu(), vc.cpu(), n, None, None, [0])
        # each result is within h (|x| + mass) of the exact one, and a little for fp32
        far = 2 * 1.2 * 2.0 ** -8 * (np.abs(want[0]) + mass[0])
        assert (np.abs(O._f64(out) - O._f64(got[i])) <= far).all()


@BOTH
def test_a_scale_of_its_own(L):
    b = Batch(BF16, Q, 2, 2, L, [4, 9], 32)
    b.desc = kvr.make_desc(*Q, BF16, b.kc.shape[1], scale=0.03)
    t = b.gpu()
    b.call(t)
    torch.cuda.synchronize()
    out, mass = O.shared(b.q, b.k, b.v, b.kc, b.vc, b.L, b.kt, b.vt, b.lens, scale=0.03)
    far = 1.2 * 2.0 ** -8 * (np.abs(out) + mass)
    assert (np.abs(O._f64(t["out"]) - out) <= far).all()
