"""kvr_continue_shared on both sides of the number of readers from which a short call is no longer one launch."""
import pytest
import torch

from test_gpu_shared import Batch, run

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32

# type, heads, readers: stages of prefix and own rows x readers x kv heads at the bound, and above it
CASES = [
    (BF16, (32, 8, 128), 64, 255, 64), (BF16, (32, 8, 128), 65, 255, 64), (F16, (4, 4, 128), 160, 200, 30),
    (F16, (4, 4, 128), 161, 200, 30), (BF16, (4, 2, 64), 1024, 280, 30), (BF16, (4, 2, 64), 1025, 280, 30),
    (F32, (4, 4, 128), 128, 96, 60), (F32, (4, 4, 128), 129, 96, 60),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%s-n%d-L%d-tail%d" % (str(c[0])[6:], "x".join(map(str, c[1])), *c[2:]))
def test_many_readers_of_a_short_prefix(case):
    dt, heads, n, L, tcap = case
    run(Batch(dt, heads, n, 1, L, [i % tcap for i in range(n)], tcap, rope_base=1e4, seed=n))


@pytest.mark.parametrize("append", [True, False], ids=["append", "keep"])
@pytest.mark.parametrize("dt,heads", [(BF16, (16, 4, 128)), (F16, (4, 4, 64)), (F32, (4, 2, 64))], ids=str)
def test_a_long_prompt_of_a_later_turn(dt, heads, append):
    """Hundreds of new tokens a reader: many row tiles, and stages of new keys that the first of them do not see."""
    run(Batch(dt, heads, 3, 257, 100, [0, 5, 300], 560, rope_base=1e4), append)
