"""kvr_paged_decode with scores and values of every size.

Queries have one element that is not zero, so that a score is one product: exact in 16-bit types, rounded once in
fp32.  What each test allows is derived in its docstring."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2606_13361_amd import kvr
from test_gpu_paged_decode import Batch

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
DTYPES = pytest.mark.parametrize("dt", [BF16, F16, F32], ids=["bf16", "fp16", "f32"])
# table's rows of 16-bit types (f32: half): one launch, ranges of a wave, ranges of four
REACH = pytest.mark.parametrize("reach", [320, 1024, 6144], ids=["one_launch", "ranges_of_a_wave", "ranges_of_four"])
HEADS = pytest.mark.parametrize("heads", [(4, 1, 128), (40, 1, 128)], ids=lambda h: "%d_%d_%d" % h)


def column(b, pool, r, d, values):
    """Element d of the rows of sequence r, in every kv head."""
    for j in range(-(-len(values) // b.ps)):
        x = values[b.ps * j:b.ps * (j + 1)]
        pool[b.table[r, j], :, :len(x), d] = x.to(b.dt)


def batch(dt, heads, reach, rows, q0, seed=0, **kw):
    b = Batch(dt, heads, 16, rows, seed=seed, max_pages=reach // 16, **kw)
    b.q.zero_()
    b.q[:, :, 0] = q0
    return b


def run(b):
    t = b.gpu()
    b.call(t)
    torch.cuda.synchronize()
    return t["out"].cpu()


def oracle(b):
    with np.errstate(invalid="ignore", over="ignore"):
        return P.decode(b.q, b.kp, b.vp, b.table.numpy(), b.rows)


# queries' and keys' sizes: scores of 1e7 and more, all finite in fp32
LARGE = [(F16, 2999.0, 3001.0), (F16, 59000.0, 61000.0), (BF16, 3.3e4, 5.1e4), (BF16, 1.3e9, 7.7e9), (BF16, 1.1e19, 0.9e19),
         (F32, 5.0e4, 4.9e4), (F32, 3.1e5, 2.9e5), (F32, 7.3e11, 1.9e12), (F32, 3.0 * 2.0 ** 60, 5.0 * 2.0 ** 59)]


@pytest.mark.parametrize("dt,q,k", LARGE, ids=lambda x: str(x).replace("torch.", ""))
@REACH
@HEADS
def test_large_finite_scores(dt, q, k, heads, reach):
    """Scores are apart by 500 units of log2 and more, or the same number: the keys of the largest one have one weight, the
    others none (2^-500 in 64 bits).  The result is the mean of w values: off by its rounding, and by w + 8 steps of
    fp32 (two sums, a quotient, products).  Scores rise and fall; queries of odd heads are negative."""
    reach //= 2 if dt == F32 else 1
    rows = [reach, reach - 7, 40, 1, 0, -1, reach // 2]
    b = batch(dt, heads, reach, rows, q, seed=3)
    b.q[:, 1::2, 0] *= -1.0
    g = torch.Generator().manual_seed(reach)
    keys = {}
    for r, m in enumerate(rows):
        if m <= 0:
            continue
        low = torch.randint(1, 33, (m,), generator=g) / 64.0 if r % 3 else torch.arange(m, 0, -1) / (2.0 * m) + 1.0 / 64.0
        x = (k * (1.0 - low.double())).to(dt)
        x[torch.randperm(m, generator=g)[:1 + r % 3]] = k
        keys[r] = -x if r % 2 else x
        column(b, b.kp, r, 0, keys[r])
    got, (out, mass) = P._f64(run(b)), oracle(b)
    for r, m in enumerate(rows):
        if m < 0:
            continue
        for p in (0, 1):
            best = 0 if m == 0 else int((keys[r] == (keys[r].min() if p else keys[r].max())).sum())
            allowed = 1.1 * (torch.finfo(dt).eps / 2 * np.abs(out[r, p::2]) + (best + 8) * 2.0 ** -24 * mass[r, p::2])
            err = np.nan_to_num(np.abs(got[r, p::2] - out[r, p::2]), nan=np.inf)
            assert (err <= allowed).all(), "sequence %d: %.3g off, a mean of %d values" % (r, err.max(), best)


def test_weights_of_fp32_keep_their_bits():
    """Two keys, the values 1 and 0: out = w / (1 + w) for one, 1 / (1 + w) for the other order, w = 2^-x, 0 <= x < 0.19.
    Steps of 2^-24: x has the rounding of the scores' difference, of the scale (two) and of the product, 3 x: 0.6, of w 0.4;
    2^x of one place, 1 (its steps are half as large below 1); out changes by at most 0.53 of w's; the sum 1,
    the quotient 1, the product 1.  In all 3.8, a tenth more."""
    n = 400
    b = batch(F32, (4, 2, 64), 16, [2] * n, 8.0)
    g = torch.Generator().manual_seed(5)
    for r in range(n):
        column(b, b.kp, r, 0, torch.rand(2, generator=g) * 0.125)
        b.vp[b.table[r, 0], :, 0] = 1.0
        b.vp[b.table[r, 0], :, 1] = 0.0
    got, (out, _) = P._f64(run(b)), oracle(b)
    rel = np.abs(got - out) / out
    assert (rel <= 1.1 * 3.8 * 2.0 ** -24).all(), "%.3g steps" % (rel.max() * 2.0 ** 24)


@DTYPES
def test_weights_keep_their_bits_where_values_cancel(dt):
    """Two keys, the values 1 and -1: out = (1 - w) / (1 + w), w = 2^-x, 0 <= x < 0.003, up to 0.001: the weights' errors are not
    hidden by its rounding.  Steps of 2^-24: a weight's 1.2 (x has three roundings, 2^x is off by one place), the sum 1, the quotient 1,
    the products 1, twice; and what a weight loses as operands: nothing (fp32), a third cut's rest of 2^-14, rounded: 2
    (bf16), a rest of 2^-10 2^-11: 8 and a little (fp16)."""
    n = 400
    b = batch(dt, (4, 2, 64), 16, [2] * n, 0.125)
    g = torch.Generator().manual_seed(6)
    for r in range(n):
        column(b, b.kp, r, 0, torch.rand(2, generator=g) * 0.125)
        b.vp[b.table[r, 0], :, 0] = 1.0
        b.vp[b.table[r, 0], :, 1] = -1.0
    got, (out, _) = P._f64(run(b)), oracle(b)
    steps = 8.4 + {F32: 0, BF16: 2, F16: 8.8}[dt]
    err, allowed = np.abs(got - out), 1.1 * (torch.finfo(dt).eps / 2 * np.abs(out) + steps * 2.0 ** -24)
    assert (err <= allowed).all(), "%.3g of what is allowed" % (err / allowed).max()


# weights that an infinite value is seen with, in log2 below the largest
SEEN = {F16: 36.0, BF16: 60.0, F32: 100.0}


@DTYPES
@REACH
def test_an_infinite_value_shows_at_small_weights(dt, reach):
    """One key of each sequence has some weight down to 2^-36 (fp16), 2^-60, 2^-100 of the largest, and infinities among its values; the other
    keys' are finite."""
    reach //= 2 if dt == F32 else 1
    n = 48
    rows = [reach] + [min(17 + 5 * r, reach) for r in range(1, n)]
    b = batch(dt, (4, 2, 128), reach, rows, 1.0, seed=7)
    g = torch.Generator().manual_seed(9)
    unit = np.sqrt(128.0) * np.log(2.0)                    # of a score: a factor of 2
    for r, m in enumerate(rows):
        x = torch.zeros(m)
        j = int(torch.randint(0, m, (1,), generator=g))
        x[j] = -unit * SEEN[dt] * (r + torch.rand(1, generator=g).item()) / n * 0.98
        column(b, b.kp, r, 0, x)
        page = b.table[r, j // 16]
        b.vp[page, :, j % 16, 5] = float("inf")
        b.vp[page, :, j % 16, 100] = -float("inf")
    got = run(b).float()
    assert bool((got[:, :, 5] == float("inf")).all()), (got[:, 0, 5] != float("inf")).nonzero().flatten().tolist()
    assert bool((got[:, :, 100] == -float("inf")).all())
    rest = [i for i in range(128) if i not in (5, 100)]
    assert bool(torch.isfinite(got[:, :, rest]).all())


@DTYPES
@REACH
def test_scores_that_are_all_minus_infinity(dt, reach):
    """Their softmax is no number, as in 64 bits; a sequence without rows in pages has zeros, and one finite score all
    the weight."""
    reach //= 2 if dt == F32 else 1
    rows = [reach, 1, 40, 0, 40, reach, reach, 33]
    lost = [(4, j, -1) for j in range(3)] + [(5, j, -1) for j in range(0, reach // 16, 2)]
    b = batch(dt, (4, 2, 64) if reach != 1024 else (4, 2, 128), reach, rows, 1.0, seed=11, lost=lost)
    for r, m in enumerate(rows):
        if r not in (3, 4):
            at = {j: int(b.table[r, j]) for j in range(-(-m // 16))}
            for j, page in at.items():
                if page >= 0:
                    b.kp[page, :, :min(16, m - 16 * j), 0] = -float("inf")
    last = rows[6] - 1
    b.kp[b.table[6, last // 16], :, last % 16, 0] = -3.0
    b.kp[b.table[7, 0], :, 2, 0] = 0.0
    got = run(b)
    for r in (0, 1, 2, 5):
        assert bool(torch.isnan(got[r]).all()), r
    for r in (3, 4):
        assert bool((got[r] == 0).all()), r
    for r, j in ((6, last), (7, 2)):
        want = b.vp[b.table[r, j // 16], :, j % 16].repeat_interleave(2, 0)
        assert torch.equal(got[r], want), r


@pytest.mark.parametrize("dt,big", [(BF16, 3.3e38), (F32, 3.3e38), (F16, 65504.0)], ids=["bf16", "f32", "fp16"])
def test_a_mean_of_many_of_the_largest_values_is_finite(dt, big):
    """2^25 rows, one page over and over, all of one value and one weight: 2^14 rows to each of 2048 waves, 2^12 products at
    most, each off by 2^-24 of the sum, and up to 2^9 records joined: 2^-11 in all."""
    b = Batch(dt, (4, 1, 64), 4096, [4096], spare=0)
    b.q.zero_()
    page = int(b.table[0, 0])
    b.vp[page] = big
    b.table = torch.full((1, 8192), page, dtype=torch.int32)
    t = b.gpu()
    t["len"].fill_(8192 * 4096)
    b.call(t)
    torch.cuda.synchronize()
    want = float(torch.tensor(big, dtype=dt))
    err = (t["out"].double().cpu() - want).abs().max().item()
    assert err <= 1.1 * want * (2.0 ** -11 + torch.finfo(dt).eps / 2), err


def test_small_values_of_short_sequences():
    """Weights are lifted by 1 / max_len (32 rows: 2^-6) and no more: values of 3e-36 stay normal numbers.  32 sums and a
    few more steps."""
    b = Batch(F32, (4, 1, 64), 16, [32, 32, 16])
    b.q.zero_()
    g = torch.Generator().manual_seed(2)
    want = (2.9e-36 * (1.0 + torch.rand(64, generator=g))).float()
    for r in range(3):
        for j in range(b.rows[r] // 16):
            b.vp[b.table[r, j]] = want
    err = (run(b).double() / want.double() - 1.0).abs().max().item()
    assert err <= 1.1 * 38 * 2.0 ** -24, err
