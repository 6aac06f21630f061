"""Offsets of packed tokens that are not in order: kvr_paged_append leaves the pages and the queries' rows alone."""
import pytest
import torch

from paper_2606_13361_amd import kvr
from test_gpu_paged_rows import BF16, DEV, SENTINEL, Append, bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,cu", [([3, 3], [5, 4, 3]), ([3, 3], [-7, -7, 900]), ([3, 3], [9, 9, 9]), ([3, 3], [0, 0, 0]),
                                     ([3, 3], [8, 0, -1]), ([3, 3], [-(1 << 31), -1, (1 << 31) - 1]), ([(1 << 31) - 1] * 2, [0, 4, 8]),
                                     ([-(1 << 31), -1], [0, 4, 8])], ids=str)
def test_nothing_is_written(lens, cu):
    """No token t of the 8 has a sequence r with cu[r] <= t < cu[r + 1], cu[r] >= 0 and rows."""
    assert not any(0 <= cu[r] <= t < cu[r + 1] and 0 <= lens[r] < 1000 for t in range(8) for r in range(2))
    c = Append(BF16, (4, 2, 64), 16, [3, 3], [4, 4])
    t = c.gpu()
    before = t["pool"].clone()
    t["len"].copy_(torch.tensor(lens))
    t["cu"].copy_(torch.tensor(cu))
    c.call(t)
    torch.cuda.synchronize()
    assert torch.equal(bits(t["pool"]), bits(before))
    assert bool((t["q_out"] == SENTINEL).all())


def test_only_the_tokens_between_a_sequences_ends_are_written():
    """200 sequences, the offsets of half of them out of order: a row of a page changes only where a token t with
    cu[r] <= t is row len[r] + t - cu[r] of sequence r."""
    n = 200
    c = Append(BF16, (4, 2, 64), 16, [3] * n, [4] * n)
    g = torch.Generator().manual_seed(1)
    cu = torch.tensor(c.cu, dtype=torch.int32)
    cu[1:n:2] = torch.randint(-9, 4 * n + 9, (n // 2,), generator=g, dtype=torch.int32)
    t = c.gpu()
    before = t["pool"].clone()
    t["cu"].copy_(cu)
    c.call(t)
    torch.cuda.synchronize()
    changed = (bits(t["pool"]) != bits(before)).any(dim=-1).any(dim=2).any(dim=0).cpu()      # [pages, rows of a page]
    may = torch.zeros_like(changed)
    for r in range(n):
        for tok in range(max(int(cu[r]), 0), c.T):
            row = 3 + tok - int(cu[r])
            if int(cu[r]) >= 0 and row < 16 * c.table.shape[1]:
                may[int(c.table[r, row // 16]), row % 16] = True
    assert not bool((changed & ~may).any())
    assert bool((changed.sum() <= c.T).all())
