"""kvr_cache_weigh and kvr_cache_evict against the fp64 oracle, and the two with
kvr_prefill and kvr_continue_shared as a server uses them together.

Tolerance of weigh, derived: a weight p of a row with scores s differs by
2 p ((d + 2) 2^-24 sum |q k| scale + 2^-22 + n 2^-24) (score, exponential, the
normalizer's sum of n terms), and adding m rows' weights by m 2^-24 of the total.
"""
import numpy as np
import pytest
import torch

from oracle import readers as O
from oracle import ref
from paper_2606_13361_amd import kvr

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
DEV = "cuda"
Q = (32, 8, 128)


def weigh_case(dt, heads, S, L, extra=3, seed=0, peaky=False):
    Hq, Hkv, d = heads
    g = torch.Generator().manual_seed(seed)
    cap = L + S + extra
    q, k = torch.randn((S, Hq, d), generator=g), torch.randn((S, Hkv, d), generator=g)
    kc = torch.full((Hkv, cap, d), float("nan"))
    kc[:, :L] = torch.randn((Hkv, L, d), generator=g)
    if peaky and L:
        u = torch.randn((Hkv, d), generator=g)
        kc[:, L // 2] += 3 * u
        q += 2 * u.repeat_interleave(Hq // Hkv, 0)
    w = torch.rand((Hkv, cap), generator=g)
    return q.to(dt), k.to(dt), kc.to(dt), w, kvr.make_desc(Hq, Hkv, d, dt, cap)


def weigh_bound(q, k, kc, L, want, before):
    q, k = np.abs(O._f64(q)), np.abs(O._f64(k))
    S, Hq, d = q.shape
    Hkv = k.shape[1]
    top = np.nan_to_num(np.abs(O._f64(kc))[:, :L]).max(1, initial=0.0)
    top = np.maximum(top, k.max(0))                                                   # [Hkv, d]
    dots = (q * np.repeat(top, Hq // Hkv, 0)).sum(-1).max() / np.sqrt(d)
    rel = 2 * ((d + 2) * 2.0 ** -24 * dots + 2.0 ** -22 + (L + S) * 2.0 ** -24)
    return 1.1 * ((want - before) * rel + want * (S * Hq // Hkv + 1) * 2.0 ** -24)


WEIGH = [
    (BF16, Q, 1, 0), (BF16, Q, 1, 1), (BF16, Q, 1, 31), (F16, Q, 1, 3774), (BF16, Q, 2, 32), (BF16, Q, 24, 1000),
    (BF16, Q, 33, 65), (F16, (8, 8, 128), 7, 129), (BF16, (12, 3, 128), 5, 200), (BF16, (64, 8, 128), 200, 300),
    (BF16, (128, 2, 128), 20, 70), (BF16, (16, 2, 64), 3, 511), (F16, (8, 2, 64), 40, 5), (F32, Q, 1, 100),
    (F32, (16, 2, 64), 19, 77), (F32, (6, 3, 128), 50, 0),
    # query rows of a kv head where the passes take other tiles, and one more
    (BF16, (8, 8, 128), 16, 300), (BF16, (8, 8, 128), 17, 300), (F16, (8, 8, 64), 32, 300), (F16, (8, 8, 64), 33, 300),
    (BF16, (8, 8, 64), 64, 200), (BF16, (8, 8, 64), 65, 200), (BF16, (4, 4, 128), 128, 777), (BF16, (4, 4, 128), 129, 777),
    (F16, (2, 2, 64), 1024, 100), (F16, (2, 2, 64), 1025, 100), (F32, (2, 2, 64), 1025, 20), (BF16, (1, 1, 64), 300, 5000),
    (BF16, (2, 1, 128), 129, 8200), (F16, (4, 1, 64), 70, 8300), (F32, (64, 64, 64), 2, 1100), (F32, (64, 64, 64), 2, 900), (BF16, (4096, 4096, 64), 1, 40), (BF16, (4096, 1, 64), 2, 40),
]


@pytest.mark.parametrize("peaky", [False, True], ids=["flat", "peaky"])
@pytest.mark.parametrize("case", WEIGH, ids=lambda c: "%s-%s-S%d-L%d" % (str(c[0])[6:], "x".join(map(str, c[1])), *c[2:]))
def test_weigh(case, peaky):
    dt, heads, S, L = case
    q, k, kc, w, desc = weigh_case(dt, heads, S, L, peaky=peaky)
    want = O.weigh(q, k, kc, L, w)
    ws = kvr.workspace_for_weigh(desc, L, S)
    ws.fill_(255)
    gw = w.to(DEV)
    args = (q.to(DEV), k.to(DEV), kc.to(DEV))
    kvr.kvr_cache_weigh(desc, *args, L, S, gw, ws)
    got = O._f64(gw)
    assert np.array_equal(got[:, L + S:], O._f64(w)[:, L + S:])
    assert (np.abs(got - want) <= weigh_bound(q, k, kc, L, want, O._f64(w))).all()
    # the same call again adds the same again, bit for bit from the same start
    again = w.to(DEV)
    kvr.kvr_cache_weigh(desc, *args, L, S, again, ws)
    assert torch.equal(again, gw)
    kvr.kvr_cache_weigh(desc, *args, L, S, gw, ws)
    twice = O.weigh(q, k, kc, L, want)
    assert (np.abs(O._f64(gw) - twice) <= 2 * weigh_bound(q, k, kc, L, twice, O._f64(w))).all()


def test_weigh_later_keys_do_not_reach_earlier_rows():
    """A key that is no number is masked for the tokens before it."""
    q, k, kc, w, desc = weigh_case(BF16, Q, 3, 40)
    k[2] = float("nan")
    gw = torch.zeros_like(w).to(DEV)
    kvr.kvr_cache_weigh(desc, q[:2].to(DEV).contiguous(), k[:2].to(DEV).contiguous(), kc.to(DEV), 40, 2, gw,
                        kvr.workspace_for_weigh(desc, 40, 2))
    assert torch.isfinite(gw[:, :42]).all()
    total = O._f64(gw).sum()
    assert abs(total - 2 * 32) < 1e-3      # each query row gives out a weight of one


def test_weigh_far_rows():
    """Offsets past 2^32 bytes in the last kv head."""
    Hq, Hkv, d, cap, L, S = 16, 8, 128, 2_400_000, 50, 2
    q, k, kc, w, _ = weigh_case(BF16, (Hq, Hkv, d), S, L)
    desc = kvr.make_desc(Hq, Hkv, d, BF16, cap)
    big = torch.zeros((Hkv, cap, d), dtype=BF16, device=DEV)
    big[:, :L] = kc[:, :L].to(DEV)
    gw = torch.zeros((Hkv, cap), device=DEV)
    kvr.kvr_cache_weigh(desc, q.to(DEV), k.to(DEV), big, L, S, gw, kvr.workspace_for_weigh(desc, L, S))
    zero = torch.zeros((Hkv, L + S))
    want = O.weigh(q, k, kc[:, :L], L, zero)
    assert (np.abs(O._f64(gw[:, :L + S]) - want) <= weigh_bound(q, k, kc, L, want, O._f64(zero))).all()
    assert not gw[:, L + S:].any()


EVICT = [
    # L, keep, first, last, kind of weights
    (1, 1, 0, 0, "normal"), (1, 1, 1, 0, "normal"), (5, 3, 1, 1, "normal"), (100, 100, 0, 0, "normal"),
    (100, 99, 4, 3, "normal"), (1000, 1, 0, 0, "normal"), (1000, 7, 4, 3, "normal"), (1000, 333, 4, 32, "ties"),
    (1023, 500, 0, 0, "equal"), (1025, 500, 1, 0, "zeros"), (5000, 1250, 4, 24, "normal"), (4096, 4000, 0, 1, "ties"),
    (3333, 1000, 2, 2, "odd"), (20000, 5000, 4, 128, "normal"), (70001, 30000, 0, 0, "normal"),
    (500, 100, 0, 0, "tiny"), (1000, 200, 4, 3, "tiny"), (1000, 900, 4, 3, "tiny"), (40000, 100, 0, 5, "tiny"),
    (1000, 300, 4, 3, "negative"), (5000, 4000, 0, 0, "negative"), (40000, 30000, 0, 0, "negative"), (3333, 1800, 2, 2, "odd"),
    (3333, 2500, 2, 2, "odd"), (3333, 3330, 2, 2, "odd"), (50000, 40000, 2, 2, "odd"), (2048, 700, 0, 0, "normal"),
    (2049, 700, 0, 0, "normal"), (8192, 2100, 5, 64, "normal"), (8193, 2100, 5, 64, "normal"), (32768, 3000, 1, 63, "normal"),
    (32769, 3000, 1, 63, "normal"), (32768, 32768, 0, 0, "ties"), (32768, 32767, 0, 0, "equal"), (32769, 32768, 0, 1, "equal"),
    (3000, 2990, 2000, 980, "normal"), (3000, 2980, 2000, 980, "normal"),
]


def evict_weights(kind, Hkv, cap, g):
    w = (2 * torch.randn((Hkv, cap), generator=g)).exp()
    if kind == "ties":
        w = (w * 2).round() / 2
    elif kind == "equal":
        w = torch.full((Hkv, cap), 0.25)
    elif kind == "zeros":
        w[torch.rand((Hkv, cap), generator=g) < 0.8] = 0.0
    elif kind == "negative":
        w = -w
    elif kind == "tiny":       # the type's least weights among zeros
        w = torch.randint(1, 60, (Hkv, cap), generator=g) * 2.0 ** -149
        w[torch.rand((Hkv, cap), generator=g) < 0.7] = 0.0
    elif kind == "odd":        # signs, infinities, both zeros, no numbers, the type's extremes
        v = torch.tensor([0.0, -0.0, -1.0, 2.0, float("inf"), -float("inf"), float("nan"), 1e-45, -1e-45,
                          torch.finfo(F32).max, torch.finfo(F32).min])
        w = v[torch.randint(0, len(v), (Hkv, cap), generator=g)]
    return w


@pytest.mark.parametrize("dt,Hkv,d", [(BF16, 8, 128), (F16, 3, 64), (F32, 2, 128)], ids=lambda x: str(x))
@pytest.mark.parametrize("case", EVICT, ids=lambda c: "L%d-keep%d-%d-%d-%s" % c)
def test_evict(case, dt, Hkv, d):
    L, keep, first, last, kind = case
    g = torch.Generator().manual_seed(L)
    cap, cap_out = L + 2, keep + 3
    w = evict_weights(kind, Hkv, cap, g)
    w[:, L:] = float("inf")                    # behind the cache: never picked
    kc, vc = torch.randn((Hkv, cap, d), generator=g).to(dt), torch.randn((Hkv, cap, d), generator=g).to(dt)
    desc = kvr.make_desc(Hkv, Hkv, d, dt, cap)
    ko, vo = (torch.full((Hkv, cap_out, d), 7.0, dtype=dt, device=DEV) for _ in range(2))
    wo = torch.full((Hkv, cap_out), 7.0, device=DEV)
    index = torch.full((Hkv, keep), -1, dtype=torch.int32, device=DEV)
    ws = kvr.workspace_for_evict(desc, L)
    ws.fill_(255)
    kvr.kvr_cache_evict(desc, kc.to(DEV), vc.to(DEV), L, w.to(DEV), keep, ko, vo, n_first=first, n_last=last,
                        weight_out=wo, index=index, ws=ws)
    want = torch.from_numpy(O.evict(w, L, keep, first, last))
    assert torch.equal(index.cpu().long(), want)
    at = torch.arange(Hkv)[:, None]
    assert torch.equal(ko.cpu()[:, :keep], kc[at, want]) and torch.equal(vo.cpu()[:, :keep], vc[at, want])
    assert torch.equal(wo.cpu()[:, :keep].view(torch.int32), w[at, want].view(torch.int32))
    for t in (ko, vo, wo):
        assert (t[:, keep:] == 7.0).all()
    # without the optional outputs
    k2, v2 = torch.zeros_like(ko), torch.zeros_like(vo)
    kvr.kvr_cache_evict(desc, kc.to(DEV), vc.to(DEV), L, w.to(DEV), keep, k2, v2, n_first=first, n_last=last, ws=ws)
    assert torch.equal(k2[:, :keep], ko[:, :keep]) and torch.equal(v2[:, :keep], vo[:, :keep])


def test_evict_far_rows():
    """Offsets past 2^32 bytes in the last kv head of both caches."""
    Hkv, d, cap, L, keep = 8, 128, 2_400_000, 3000, 700
    g = torch.Generator().manual_seed(3)
    desc = kvr.make_desc(Hkv, Hkv, d, BF16, cap)
    kc, vc = (torch.zeros((Hkv, cap, d), dtype=BF16, device=DEV) for _ in range(2))
    w = torch.zeros((Hkv, cap), device=DEV)
    k0, v0 = torch.randn((Hkv, L, d), generator=g).to(BF16), torch.randn((Hkv, L, d), generator=g).to(BF16)
    w0 = torch.rand((Hkv, L), generator=g)
    kc[:, :L], vc[:, :L], w[:, :L] = k0.to(DEV), v0.to(DEV), w0.to(DEV)
    ko, vo = (torch.zeros((Hkv, cap, d), dtype=BF16, device=DEV) for _ in range(2))
    kvr.kvr_cache_evict(desc, kc, vc, L, w, keep, ko, vo, ws=kvr.workspace_for_evict(desc, L))
    want = torch.from_numpy(O.evict(w0, L, keep, 0, 0))
    at = torch.arange(Hkv)[:, None]
    assert torch.equal(ko[:, :keep].cpu(), k0[at, want]) and torch.equal(vo[:, :keep].cpu(), v0[at, want])


def test_weigh_and_evict_in_a_graph():
    """One captured weigh + evict, replayed on changed inputs, with eager work between: the eager bits."""
    q, k, kc, w, desc = weigh_case(BF16, Q, 24, 700)
    vc = torch.randn(kc.shape).to(BF16)
    L, S, keep = 700, 24, 200

    def state():
        t = [x.to(DEV) for x in (q, k, kc, w, vc)]
        ko, vo = (torch.zeros((8, keep, 128), dtype=BF16, device=DEV) for _ in range(2))
        ix = torch.zeros((8, keep), dtype=torch.int32, device=DEV)
        return t + [ko, vo, ix, kvr.workspace_for_weigh(desc, L, S), kvr.workspace_for_evict(desc, L + S)]

    def step(t):
        kvr.kvr_cache_weigh(desc, t[0], t[1], t[2], L, S, t[3], t[8])
        kvr.kvr_cache_evict(desc, t[2], t[4], L + S, t[3], keep, t[5], t[6], n_first=4, n_last=24, index=t[7], ws=t[9])

    a, e = state(), state()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        step(state())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a)
    gen = torch.Generator().manual_seed(1)
    for i in range(4):
        new = torch.randn(q.shape, generator=gen).to(BF16).to(DEV)
        a[0].copy_(new)
        e[0].copy_(new)
        graph.replay()
        step(e)
        float(a[3].nan_to_num().sum())
        for x, y in zip(a[3:8], e[3:8]):
            assert torch.equal(x.nan_to_num(), y.nan_to_num()), i


def test_two_streams_at_once():
    """Weighing and eviction of two caches on two streams, a workspace each: the bits of one after the other."""
    S, L, keep = 40, 5000, 1200
    sets = []
    for seed in (1, 2):
        q, k, kc, w, desc = weigh_case(BF16, Q, S, L, seed=seed)
        kc = kc.nan_to_num().to(DEV)
        sets.append(dict(desc=desc, q=q.to(DEV), k=k.to(DEV), kc=kc, vc=kc.flip(1).contiguous(), w=w.to(DEV),
                         ws=kvr.workspace_for_weigh(desc, L, S), ko=torch.zeros((8, keep, 128), dtype=BF16, device=DEV),
                         vo=torch.zeros((8, keep, 128), dtype=BF16, device=DEV),
                         ix=torch.zeros((8, keep), dtype=torch.int32, device=DEV)))

    def step(a, stream=None):
        kvr.kvr_cache_weigh(a["desc"], a["q"], a["k"], a["kc"], L, S, a["w"], a["ws"], stream=stream)
        kvr.kvr_cache_evict(a["desc"], a["kc"], a["vc"], L + S, a["w"], keep, a["ko"], a["vo"], n_last=S, index=a["ix"],
                            stream=stream)

    start = [a["w"].clone() for a in sets]
    for a in sets:
        for _ in range(3):
            step(a)
    want = [{x: a[x].clone() for x in ("w", "ko", "vo", "ix")} for a in sets]
    for a, w in zip(sets, start):
        a["w"].copy_(w)
        for x in ("ko", "vo", "ix"):
            a[x].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for a, s in zip(sets, streams):
            step(a, s)
    torch.cuda.synchronize()
    for a, w in zip(sets, want):
        for x in w:
            assert torch.equal(a[x], w[x]), x


@pytest.mark.parametrize("dt", [BF16, F16, F32], ids=str)
def test_a_document_weighed_evicted_and_read_by_many(dt):
    """Prefill with the rotary embedding, weights of its last tokens, a third of the rows
    kept, then four decode steps of five readers over what is left: each stage against
    the oracle on what the stage before left."""
    Hq, Hkv, d = heads = (16, 4, 64)
    L, W, keep, n, tcap = 300, 16, 100, 5, 12
    g = torch.Generator().manual_seed(5)
    r = lambda *s: torch.randn(s, generator=g).to(dt).to(DEV)
    desc = kvr.make_desc(Hq, Hkv, d, dt, L)
    rope = kvr.RopeTable(d, L + tcap, base=1e4)
    q, k, v = r(L, Hq, d), r(L, Hkv, d), r(L, Hkv, d)
    out = torch.empty_like(q)
    kc, vc = (torch.zeros((Hkv, L, d), dtype=dt, device=DEV) for _ in range(2))
    kvr.kvr_prefill_rope(desc, rope, q, k, v, L, out, kc, vc)
    qw = kvr.kvr_rope_apply(desc, rope, q[L - W:].contiguous(), L - W)
    kw = kc[:, L - W:].transpose(0, 1).contiguous()
    weight = torch.zeros((Hkv, L), device=DEV)
    kvr.kvr_cache_weigh(desc, qw, kw, kc, L - W, W, weight, kvr.workspace_for_weigh(desc, L - W, W))
    want = O.weigh(qw, kw, kc, L - W, torch.zeros((Hkv, L)))
    assert (np.abs(O._f64(weight) - want) <= weigh_bound(qw, kw, kc, L - W, want, 0 * want)).all()

    small = kvr.make_desc(Hq, Hkv, d, dt, keep)
    ko, vo = (torch.empty((Hkv, keep, d), dtype=dt, device=DEV) for _ in range(2))
    index = torch.empty((Hkv, keep), dtype=torch.int32, device=DEV)
    kvr.kvr_cache_evict(desc, kc, vc, L, weight, keep, ko, vo, n_first=4, n_last=W, index=index,
                        ws=kvr.workspace_for_evict(desc, L))
    kept = torch.from_numpy(O.evict(weight, L, keep, 4, W))
    assert torch.equal(index.cpu().long(), kept)

    kt, vt = (torch.full((n, Hkv, tcap, d), float("nan"), dtype=dt, device=DEV) for _ in range(2))
    ln = torch.tensor([0, 3, -1, 7, 2], dtype=torch.int32, device=DEV)
    for i, m in enumerate(ln.tolist()):
        if m > 0:
            kt[i, :, :m], vt[i, :, :m] = r(Hkv, m, d), r(Hkv, m, d)
    on = (ln >= 0).int()
    ws = kvr.workspace_for_shared(small, keep, n, 1, tcap)
    h = torch.finfo(dt).eps / 2
    for step in range(4):
        q, k, v = r(n, 1, Hq, d), r(n, 1, Hkv, d), r(n, 1, Hkv, d)
        out = torch.zeros_like(q)
        before = kt.clone(), vt.clone()
        kvr.kvr_continue_shared(small, q, k, v, ko, vo, keep, kt, vt, ln, out, ws, rope=rope, pos0=L, append=True)
        for i, m in enumerate(ln.tolist()):
            if m >= 0:
                kvr.kvr_rope_apply(small, rope, q[i], L + m)
                kvr.kvr_rope_apply(small, rope, k[i], L + m)
                assert torch.equal(kt[i, :, m], k[i, 0]) and torch.equal(vt[i, :, m], v[i, 0])
        want, mass = O.shared(q, k, v, ko, vo, keep, *before, ln.tolist())
        for i, m in enumerate(ln.tolist()):
            if m >= 0:
                # weights and output rounded once each (fp32: neither), and 2^-13 of the mass for fp32 sums of
                # up to 112 keys and 64 products of up to 4 sigma: 2 (66 * 2^-24 * 2^7 + 112 * 2^-24) < 2^-9.8 / 8
                far = 1.1 * (h * (np.abs(want[i]) + mass[i]) + 2.0 ** -12.8 * mass[i])
                assert (np.abs(O._f64(out[i]) - want[i]) <= far).all()
        ln += on
