"""kvr_paged_decode against the fp64 oracle, and what must stay as it was.

Rows behind a sequence's length, pages of nobody and the workspace hold NaN; the page
table holds numbers that are no page wherever a sequence has no rows.

Tolerance, derived: an output is sum p v / sum p, rounded once to its type: h |out|, h = eps / 2.
Relative to mass = sum p |v|: a weight of 16 bits is a value cut off, which leaves 2 h of it
at most, and a little, and that rest rounded: off by 2 h^2 and a tenth (fp16 numbers end at
2^-25, 2^-37 of the largest weight, for each of n keys); a score of d products in fp32 by (d + 2) 2^-24 sum |q k| scale, twice (numerator and
denominator), 2^x by 2^-22, in the weight and in up to three joins; sums of n terms by
n 2^-24 each, twice.  Second-order terms: a tenth more.
"""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2606_13361_amd import kvr

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
DEV = "cuda"
SENTINEL = 7.0
NOWHERE = [-1, 1 << 30, -(1 << 31), (1 << 31) - 1]


def bound(dt, out, mass, q, keys_abs, n_keys):
    """keys_abs: the largest |k| of each head-dim index, [Hkv, d]; n_keys [n]."""
    h = torch.finfo(dt).eps / 2
    d = q.shape[2]
    dots = (np.abs(q) * np.repeat(keys_abs, q.shape[1] // keys_abs.shape[0], 0)).sum(-1) / np.sqrt(d)      # [n, Hq]
    n_keys = np.asarray(n_keys, dtype=np.float64)[:, None]
    rel = 2 * (d + 2) * 2.0 ** -24 * dots + 4 * 2.0 ** -22 + 2 * n_keys * 2.0 ** -24
    rel = rel + (0 if dt == F32 else 2.2 * h * h) + (n_keys * 2.0 ** -37 if dt == F16 else 0)
    return 1.1 * (h * np.abs(out) + mass * rel[..., None])


class Batch:
    """One call.  rows: what each sequence's token sees (n_new of them not in `length`)."""

    def __init__(self, dt, heads, ps, rows, seed=0, n_new=0, spare=2, max_pages=None, apart=0, lost=()):
        Hq, Hkv, d = heads
        g = torch.Generator().manual_seed(seed)
        self.dt, self.heads, self.ps, self.rows, self.n_new = dt, heads, ps, list(rows), n_new
        n = len(rows)
        need = [-(-max(m, 0) // ps) for m in rows]
        total = sum(need) + spare
        order = torch.randperm(total, generator=g).tolist()
        cols = max(need + [1]) if max_pages is None else max_pages
        self.table = torch.tensor([[NOWHERE[(r + j) % 4] for j in range(cols)] for r in range(n)], dtype=torch.int32)
        self.q = torch.randn((n, Hq, d), generator=g).to(dt)
        self.pool = torch.full((total, 2, Hkv * ps * d + apart), float("nan"), dtype=dt)
        self.kp, self.vp = (self.pool[:, i, :Hkv * ps * d].unflatten(1, (Hkv, ps, d)) for i in (0, 1))
        at = 0
        for r, m in enumerate(rows):
            for j in range(min(need[r], cols)):
                page, took = order[at], min(ps, m - j * ps)
                at += 1
                self.kp[page, :, :took] = torch.randn((Hkv, took, d), generator=g).to(dt)
                self.vp[page, :, :took] = torch.randn((Hkv, took, d), generator=g).to(dt)
                self.table[r, j] = page
        for r, j, entry in lost:
            self.table[r, j] = entry
        self.desc = kvr.make_desc(Hq, Hkv, d, dt, 0)

    def gpu(self, max_len=None):
        t = {"q": self.q.to(DEV), "pool": self.pool.to(DEV), "table": self.table.to(DEV)}
        Hq, Hkv, d = self.heads
        t["kp"], t["vp"] = (t["pool"][:, i, :Hkv * self.ps * d].unflatten(1, (Hkv, self.ps, d)) for i in (0, 1))
        t["cache"] = kvr.PagedCache(self.desc, t["kp"], t["vp"], t["table"])
        t["len"] = torch.tensor([m - self.n_new if m >= 0 else -5 for m in self.rows], dtype=torch.int32, device=DEV)
        t["out"] = torch.full(self.q.shape, SENTINEL, dtype=self.dt, device=DEV)
        t["max_len"] = t["cache"].reach if max_len is None else max_len
        t["ws"] = kvr.workspace_for_paged(self.desc, len(self.rows), t["max_len"])
        t["ws"].fill_(255)      # NaN everywhere
        return t

    def call(self, t, **kw):
        kvr.kvr_paged_decode(self.desc, t["cache"], t["q"], t["len"], t["out"], t["ws"], n_new=self.n_new,
                             max_len=t["max_len"], **kw)

    def check(self, t, got=None):
        torch.cuda.synchronize()
        rows = [m if m <= t["max_len"] else -1 for m in self.rows]
        out, mass = P.decode(self.q, self.kp, self.vp, self.table.numpy(), rows)
        keys = np.nan_to_num(np.abs(P._f64(self.kp))).max((0, 2), initial=0.0)
        b = bound(self.dt, out, mass, P._f64(self.q), keys, np.maximum(rows, 0))
        got = (t["out"] if got is None else got).cpu()
        for r, m in enumerate(rows):
            if m < 0:
                assert torch.equal(got[r], torch.full_like(got[r], SENTINEL)), "row of sequence %d written" % r
                continue
            err = np.abs(P._f64(got[r]) - out[r])
            assert (err <= b[r]).all(), "sequence %d (%d rows): %.3g off, %.3g allowed there" % (
                r, m, np.nan_to_num(err, nan=np.inf).max(), b[r].flat[int(np.argmax(np.nan_to_num(err - b[r], nan=np.inf)))])
        return got


Q = (32, 8, 128)
DTYPES = pytest.mark.parametrize("dt", [BF16, F16, F32], ids=["bf16", "fp16", "f32"])


@DTYPES
@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 31, 33, 63, 65, 127, 128, 129, 255, 300, 512])
def test_one_sequence_one_launch(dt, m):
    b = Batch(dt, Q, 16, [m], seed=m)
    t = b.gpu()
    b.call(t)
    b.check(t)


@DTYPES
@pytest.mark.parametrize("m", [1, 64, 513, 1024, 1025, 3774, 4097, 9001])
def test_one_sequence_shared_out(dt, m):
    b = Batch(dt, Q, 64, [m], seed=m, max_pages=9100 // 64 + 1)
    t = b.gpu()
    b.call(t)
    b.check(t)


HEADS = [(8, 8, 128), (12, 3, 128), (64, 8, 128), (32, 1, 128), (17, 1, 64), (48, 1, 128), (40, 1, 64), (130, 2, 64), (16, 2, 64),
         (1, 1, 64), (7, 7, 64)]


@DTYPES
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d_%d_%d" % h)
@pytest.mark.parametrize("reach", [384, 4096], ids=["one_launch", "shared_out"])
def test_heads(dt, heads, reach):
    b = Batch(dt, heads, 32, [77, 300, 1, 0, -1, 203], seed=heads[0], max_pages=reach // 32)
    t = b.gpu()
    b.call(t)
    b.check(t)


@DTYPES
@pytest.mark.parametrize("ps", [16, 32, 48, 80, 112, 256, 1008])
@pytest.mark.parametrize("apart", [0, 64])
def test_page_sizes(dt, ps, apart):
    b = Batch(dt, (16, 2, 64), ps, [1500, ps, ps + 1, ps - 1, 2 * ps, 700], seed=ps, apart=apart)
    t = b.gpu()
    b.call(t)
    b.check(t)


@DTYPES
@pytest.mark.parametrize("n", [2, 63, 64, 65, 130, 200])
def test_ragged_batches(dt, n):
    """Lengths of all kinds, empty slots and empty sequences among them, first and last too."""
    g = torch.Generator().manual_seed(n)
    rows = torch.randint(0, 700, (n,), generator=g).tolist()
    for r in range(0, n, 7):
        rows[r] = -1
    for r in range(3, n, 11):
        rows[r] = 0
    rows[n // 2] = 2600
    for first, last in ((rows[0], -1), (0, rows[-1])):
        b = Batch(dt, (8, 2, 64), 16, [first] + rows[1:-1] + [last], seed=n)
        t = b.gpu()
        b.call(t)
        b.check(t)


@pytest.mark.parametrize("max_pages", [None, 400], ids=["one_launch", "shared_out"])
def test_many_sequences(max_pages):
    """More sequences than two rounds of the search take one by one."""
    n = 4500
    rows = [(37 * r) % 29 - 3 for r in range(n)]
    rows[4200] = 1100
    b = Batch(BF16, (4, 1, 64), 16, rows, seed=1, max_pages=max_pages)
    t = b.gpu()
    assert (t["ws"].numel() > 0) == (max_pages is not None)
    b.call(t)
    b.check(t)


# max_len of the ways of a call of 6 sequences of at most 150 rows or so, by the bytes of a sequence and head: one
# launch of four waves each, ranges of one wave, ranges of four
WAYS = {"one_launch": 160, "ranges_of_a_wave": 1024, "ranges_of_four": 3200}
EACH = [(w, h) for w in WAYS for h in ((8, 2, 128), (8, 2, 64), (20, 1, 128), (40, 1, 64)) if w != "ranges_of_a_wave" or h[2] == 128]


@DTYPES
@pytest.mark.parametrize("way,heads", EACH, ids=lambda x: x if isinstance(x, str) else "%d_%d_%d" % x)
def test_each_way(dt, heads, way):
    reach = WAYS[way] // (2 if dt == F32 else 1)
    rows = [reach // (7 if way == "one_launch" else 3), 150, 0, -1, 33, 64]
    if way != "one_launch":
        rows[4] = reach
    b = Batch(dt, heads, 16, [min(m, reach) for m in rows], seed=reach, max_pages=reach // 16)
    t = b.gpu()
    assert (t["ws"].numel() > 0) == (way != "one_launch")
    b.call(t)
    b.check(t)


@DTYPES
def test_keys_and_values_around_the_caches(dt):
    """53 MB of 16-bit keys and values (f32: 105), which are loaded with the non-temporal hint; with a page that
    is not there and rows behind the lengths."""
    b = Batch(dt, (8, 2, 128), 64, [30001, 0, 12345, -1, 9000], seed=8, lost=[(0, 17, -1)])
    t = b.gpu()
    b.call(t)
    b.check(t)


@DTYPES
@pytest.mark.parametrize("heads", [(8, 8, 64), (8, 4, 128), (68, 2, 64)], ids=lambda h: "%d_%d_%d" % h)
def test_a_wave_for_each_of_many_short_ones(dt, heads):
    n = 1024 // heads[1] + 3
    b = Batch(dt, heads, 16, [(r * 13) % 61 - 1 for r in range(n)], seed=2)
    t = b.gpu()
    assert t["ws"].numel() == 0
    b.call(t)
    b.check(t)


@DTYPES
def test_nothing_to_do(dt):
    for rows in ([-1], [-1] * 70, [0], [0, -1] * 50):
        b = Batch(dt, Q, 16, rows, max_pages=100)
        t = b.gpu()
        b.call(t)
        b.check(t)


@DTYPES
@pytest.mark.parametrize("reach", [384, 8192], ids=["one_launch", "shared_out"])
def test_pages_that_are_not_there(dt, reach):
    """Entries out of the pool's range, at the front, inside and at the end; one sequence has no page at all."""
    rows = [370, 300, 100, 64, 380]
    lost = [(0, 0, -1), (0, 5, 1 << 30), (1, 9, -7), (2, 3, 10 ** 6)] + [(3, j, -1) for j in range(4)]
    lost += [(4, j, -1) for j in range(8)]      # nothing until the ninth page
    b = Batch(dt, Q, 32, rows, seed=3, max_pages=reach // 32, lost=lost)
    b.table[0, 6] = b.kp.shape[0]               # one behind the last
    t = b.gpu()
    b.call(t)
    got = b.check(t)
    assert bool((got[3] == 0).all())


@DTYPES
def test_sequences_share_pages(dt):
    b = Batch(dt, Q, 32, [200, 200, 130], seed=5)
    b.table[1, :4] = b.table[0, :4]
    b.table[2] = b.table[0]
    t = b.gpu()
    b.call(t)
    got = b.check(t)
    assert not torch.equal(got[0], got[1])


@DTYPES
def test_longer_than_max_len_takes_no_part(dt):
    b = Batch(dt, Q, 16, [40, 41, 64, 12], n_new=1)
    t = b.gpu(max_len=40)
    b.call(t)
    b.check(t)
    t = b.gpu()
    t["len"][1] = (1 << 31) - 1      # with n_new beyond 32 bits
    b.rows[1] = 1 << 31
    b.call(t)
    b.check(t)


@DTYPES
def test_max_len_and_batch_do_not_change_much(dt):
    """One launch and shared out: both within the bound, and each the same bits again."""
    b = Batch(dt, Q, 16, [300, 12, 511, 77], seed=9, max_pages=200)
    outs = []
    for most in (512, 512, 3200, 3200):
        t = b.gpu(max_len=most)
        b.call(t)
        outs.append(b.check(t))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[2], outs[3])


@DTYPES
@pytest.mark.parametrize("reach", [512, 8192], ids=["one_launch", "shared_out"])
def test_scores_far_apart(dt, reach):
    """Score ranges of hundreds of log2 units, rising, falling and with one key far above; values of many sizes."""
    rows = [500, 500, 500, 500]
    b = Batch(dt, (8, 2, 128), 16, rows, seed=4, max_pages=reach // 16)
    b.q.mul_(0.25)
    b.q[:, :, 0] = 8.0
    g = torch.Generator().manual_seed(1)
    ramp = torch.linspace(-40.0, 40.0, 500)
    for r, a in enumerate((ramp, -ramp, torch.where(torch.arange(500) == 333, 60.0, 0.0), torch.zeros(500))):
        for j in range(32):
            page, took = b.table[r, j], min(16, 500 - 16 * j)
            b.kp[page, :, :took, 0] = a[16 * j:16 * j + took].to(dt)
            b.vp[page, :, :took] *= torch.exp2(torch.randint(-6, 7, (took, 1), generator=g)).to(dt)
    t = b.gpu()
    b.call(t)
    b.check(t)


def test_scores_as_large_as_numbers_go():
    """All scores are -2^120 or so: the largest of them has all the weight."""
    b = Batch(F32, (2, 1, 64), 16, [40, 700])
    b.q.zero_()
    b.q[:, :, 0] = -2.0 ** 60
    for r, m in enumerate(b.rows):
        for j in range(-(-m // 16)):
            b.kp[b.table[r, j], 0, :, 0] = 2.0 ** 62
        b.kp[b.table[r, 1], 0, 5, 0] = 2.0 ** 61
    t = b.gpu()
    b.call(t)
    torch.cuda.synchronize()
    for r in range(2):
        assert torch.equal(t["out"][r].cpu(), b.vp[b.table[r, 1], 0, 5].expand(2, 64))


@pytest.mark.parametrize("reach", [208, 8192], ids=["one_launch", "shared_out"])
def test_largest_numbers(reach):
    """A mean of the largest values is finite; an infinity where it has weight shows."""
    for dt, big in ((BF16, 3.3e38), (F16, 65504.0), (F32, 3.4e38)):
        m = reach - 8
        b = Batch(dt, (4, 1, 64), 16, [m, m], max_pages=reach // 16)
        b.q.zero_()
        for j in range(reach // 16):
            b.vp[b.table[0, j], :, :min(16, m - 16 * j)] = big
        b.vp[b.table[1, 7], 0, 3, 5] = float("inf")
        t = b.gpu()
        b.call(t)
        torch.cuda.synchronize()
        got = t["out"].float().cpu()
        want = torch.tensor(big, dtype=dt).float()
        assert torch.allclose(got[0], want.expand_as(got[0]), rtol=2.0 ** -7, atol=0)
        assert bool((got[1, :, 5] == float("inf")).all())
        assert bool(torch.isfinite(got[1, :, torch.arange(64) != 5]).all())


def test_a_score_that_is_no_number_shows():
    b = Batch(F32, (4, 2, 64), 16, [100, 100])
    b.kp[b.table[0, 2], 0, 3, 5] = float("nan")
    t = b.gpu()
    b.call(t)
    torch.cuda.synchronize()
    got = t["out"].cpu()
    assert bool(torch.isnan(got[0, :2]).all()) and bool(torch.isfinite(got[0, 2:]).all()) and bool(torch.isfinite(got[1]).all())


def test_offsets_beyond_32_bits():
    """Pages 5 GB into a pool, and page strides of that size."""
    Hkv, ps, d = 2, 16, 64
    pool = torch.empty(3 << 30, dtype=torch.bfloat16, device=DEV)      # 6 GB
    stride = (5 << 28)                                                  # elements: 2.5 GB
    kp = torch.as_strided(pool, (3, Hkv, ps, d), (stride, ps * d, d, 1))
    vp = torch.as_strided(pool[1 << 20:], (3, Hkv, ps, d), (stride, ps * d, d, 1))
    b = Batch(BF16, (8, 2, 64), ps, [45], spare=0)
    for x, y in ((kp, b.kp), (vp, b.vp)):
        x.copy_(y)
    t = b.gpu()
    t["cache"] = kvr.PagedCache(b.desc, kp, vp, t["table"])
    b.call(t)
    b.check(t)


def test_a_long_sequence():
    """2^25 rows and some: one page over and over, so that every row counts alike and the mean is the page's.
    A range has at most 2^25 / 1024 rows, 32 of which are one product: 1024 sums each off by 2^-24, twice,
    and as many ranges joined; a row more or less is 2^-25."""
    b = Batch(BF16, (4, 1, 64), 4096, [4096], spare=0)
    page = int(b.table[0, 0])
    b.table = torch.full((1, 8193), page, dtype=torch.int32)
    t = b.gpu()
    t["len"].fill_(8192 * 4096 + 5)
    b.call(t)
    torch.cuda.synchronize()
    want, mass = P.decode(b.q, b.kp, b.vp, b.table.numpy(), [4096])
    err = np.abs(P._f64(t["out"]) - want)
    assert (err <= 1.1 * (2.0 ** -8 * np.abs(want) + mass * 2.0 ** -11)).all()


def test_dense_cache_is_a_pool_of_one_page():
    b = Batch(BF16, Q, 320, [300], spare=0)
    t = b.gpu()
    kc, vc = t["kp"][0].contiguous(), t["vp"][0].contiguous()
    t["cache"] = kvr.PagedCache(b.desc, kc[None], vc[None], torch.zeros((1, 1), dtype=torch.int32, device=DEV))
    b.call(t)
    b.check(t)
