"""kvr_cache_weigh: a token's key gets no weight from the tokens before it, however large its score is there.

One late token has a key for which every query of its kv head scores far above all others: the queries from that
token on give it all their weight, those before it none.  Tolerance as in test_gpu_evict.py."""
import math

import numpy as np
import pytest
import torch

from oracle import readers as O
from paper_2606_13361_amd import kvr

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
DEV = "cuda"

# late token in the first stage of the new rows and in a later one; up to 16 query rows of a kv head, more, and
# so many that a wave has four row tiles; head_dim 64
CASES = [
    (BF16, (32, 8, 128), 3, 40, 2), (BF16, (32, 8, 128), 3, 40, 1), (F16, (8, 8, 64), 40, 5, 35), (BF16, (32, 8, 128), 40, 33, 2),
    (BF16, (32, 8, 128), 40, 33, 35), (BF16, (4, 1, 128), 100, 8200, 70), (F16, (16, 2, 64), 70, 300, 69), (F32, (32, 8, 128), 3, 40, 2),
    (F32, (16, 2, 64), 20, 77, 18), (F32, (16, 2, 64), 40, 0, 17),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%s-S%d-L%d-late%d" % (str(c[0])[6:], "x".join(map(str, c[1])), *c[2:]))
def test_a_late_key_gets_weight_from_its_own_token_on(case):
    dt, (Hq, Hkv, d), S, L, late = case
    G = Hq // Hkv
    g = torch.Generator().manual_seed(S + L)
    q, k, kc = torch.randn((S, Hq, d), generator=g), torch.randn((S, Hkv, d), generator=g), torch.randn((Hkv, L + S, d), generator=g)
    # component 0: every query has it, of the keys that one alone, 60 nats high
    q[..., 0], k[..., 0], kc[..., 0] = 4.0, 0.0, 0.0
    k[late, :, 0] = 15.0 * math.sqrt(d)
    q, k, kc = q.to(dt), k.to(dt), kc.to(dt)
    desc = kvr.make_desc(Hq, Hkv, d, dt, L + S)
    w = torch.zeros((Hkv, L + S), device=DEV)
    kvr.kvr_cache_weigh(desc, q.to(DEV), k.to(DEV), kc.to(DEV), L, S, w, kvr.workspace_for_weigh(desc, L, S))
    got, want = O._f64(w), O.weigh(q, k, kc, L, torch.zeros((Hkv, L + S)))
    top = np.abs(O._f64(k)).max(0)
    if L:
        top = np.maximum(top, np.abs(O._f64(kc)).max(1))
    dots = (np.abs(O._f64(q)) * np.repeat(top, G, 0)).sum(-1).max() / math.sqrt(d)
    rel = 2 * ((d + 2) * 2.0 ** -24 * dots + 2.0 ** -22 + (L + S) * 2.0 ** -24) + (S * G + 1) * 2.0 ** -24
    assert (np.abs(got - want) <= 1.1 * rel * want).all()
    # all of each later token's weight but e^-30 of it, and nothing of an earlier one's
    assert (np.abs(got[:, L + late] - (S - late) * G) <= (1.1 * rel + math.exp(-30)) * (S - late) * G).all()
