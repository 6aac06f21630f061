"""Sizes of kvr_paged_decode's workspace, and integers of the paged calls' binding, without a GPU."""
import pytest
import torch

from paper_2606_13361_amd import kvr


@pytest.mark.parametrize("heads,n", [((32, 8, 128), 64), ((32, 8, 128), 32), ((16, 2, 64), 64), ((16, 2, 64), 1), ((40, 1, 64), 5)],
                         ids=str)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_workspace_has_the_records_that_a_call_can_use(dt, heads, n):
    """Where every max_len up to 32 stages is one launch (head_dim 64, or 256 heads of the batch), ranges are of four
    waves: 256 workgroups (512 where a stage is 8 KB) at most, two records of each."""
    Hq, Hkv, d = heads
    G = Hq // Hkv
    tiles, rows = -(-G // 32), min(G, 32)
    stage = (16 if dt == torch.float32 else 32) * d * (4 if dt == torch.float32 else 2) * 2
    groups = (64 << 10) // stage * 256 // 4
    need = kvr.kvr_workspace_bytes_paged(kvr.make_desc(Hq, Hkv, d, dt, 0), n, 1 << 17)
    assert need == 2 * groups * rows * (d + 2) * 4 + n * Hkv * tiles * 8


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "fp16", "f32"])
def test_workspace_serves_every_shorter_max_len(dt):
    for heads in ((32, 8, 128), (16, 2, 64), (40, 1, 128), (4, 1, 64)):
        desc = kvr.make_desc(*heads, dt, 0)
        for n in (1, 3, 20, 30, 31, 32, 33, 70, 300):
            sizes = [kvr.kvr_workspace_bytes_paged(desc, n, 16 * i) for i in range(400)]
            assert sizes == sorted(sizes), (heads, n)


def test_integers_that_the_c_types_do_not_hold():
    """Not cut to their lower bits: 2^32 + 1 sequences are not one."""
    desc = kvr.make_desc(32, 8, 128, torch.bfloat16, 0)
    for n, most in ((1 << 32, 1 << 17), ((1 << 32) + 1, 1 << 17), (-(1 << 32) + 1, 1 << 17), (1, 1 << 64), (1, (1 << 64) + 5000)):
        with pytest.raises(ValueError):
            kvr.kvr_workspace_bytes_paged(desc, n, most)
        with pytest.raises(ValueError):
            kvr.workspace_for_paged(desc, n, most, device="cpu")


@pytest.mark.gpu
def test_integers_of_calls_that_the_c_types_do_not_hold():
    desc = kvr.make_desc(4, 2, 64, torch.bfloat16, 0)
    pool = torch.zeros((3, 2, 2, 16, 64), dtype=torch.bfloat16, device="cuda")
    table = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    cache = kvr.PagedCache(desc, pool[:, 0], pool[:, 1], table)
    q = torch.ones((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    out, length = torch.full_like(q, 7.0), torch.full((2,), 5, dtype=torch.int32, device="cuda")
    for kw in (dict(n_new=1 << 32), dict(n_new=(1 << 32) + 1), dict(max_len=1 << 64), dict(max_len=(1 << 64) + 16)):
        with pytest.raises(ValueError):
            kvr.kvr_paged_decode(desc, cache, q, length, out, **kw)
    with pytest.raises(ValueError):
        kvr.kvr_qk_norm_rope(desc, q, None, rope=kvr.RopeTable(64, 32), pos0=1 << 64)
    for shape in ((0, 1 << 32), ((1 << 32) + 1, 0)):
        with pytest.raises(ValueError):
            kvr.PagedCache(desc, pool[:, 0], pool[:, 1], torch.empty(shape, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert bool((out == 7.0).all()) and bool((q == 1.0).all())
