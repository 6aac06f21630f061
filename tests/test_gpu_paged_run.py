"""The paged calls as a server runs them: prompts into pages, then steps of append and decode, against the
dense calls and the oracle; captured into a graph, on other streams, two at once.

Tolerances: keys and values are compared bit for bit with the dense calls' caches.  Attention of the dense
16-bit calls rounds each weight and each output once, h = eps / 2, ours each output: 3 h of values below 4
(means of N(0, 1) values; the single-key means are rows themselves), 2e-2 in bf16, 3e-3 in fp16; fp32 1e-5,
the bar that the library holds fp32 to."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2606_13361_amd import kvr
from test_gpu_paged_decode import bound

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
DEV = "cuda"
BASE = 1.0e6
TOL = {BF16: 2e-2, F16: 3e-3, F32: 1e-5}
DTYPES = pytest.mark.parametrize("dt", [BF16, F16, F32], ids=["bf16", "fp16", "f32"])


def draw(g, dt, *shape):
    return torch.randn(shape, generator=g, device=DEV).to(dt)


def same_bits(a, b):
    i = torch.int32 if a.dtype == F32 else torch.int16
    return torch.equal(a.contiguous().view(i), b.contiguous().view(i))


class Server:
    """n sequences in one pool; a table with room for `reach` rows each, pages drawn without an order."""

    def __init__(self, dt, heads, ps, n, reach, seed=0):
        Hq, Hkv, d = heads
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.dt, self.heads, self.ps, self.n = dt, heads, ps, n
        cols = -(-reach // ps)
        self.pool = torch.full((n * cols + 3, 2, Hkv, ps, d), float("nan"), dtype=dt, device=DEV)
        perm = torch.randperm(n * cols, generator=torch.Generator().manual_seed(seed))
        self.table = perm.to(torch.int32).view(n, cols).to(DEV).contiguous()
        self.desc = kvr.make_desc(Hq, Hkv, d, dt, cols * ps)
        self.cache = kvr.PagedCache(self.desc, self.pool[:, 0], self.pool[:, 1], self.table)
        self.rope = kvr.RopeTable(d, cols * ps, base=BASE)
        self.len = torch.zeros(n, dtype=torch.int32, device=DEV)
        self.ws = kvr.workspace_for_paged(self.desc, n, cols * ps)
        self.out = torch.zeros((n, Hq, d), dtype=dt, device=DEV)

    def step(self, q, k, v, stream=None, **kw):
        """One token of each sequence: q is rotated in place."""
        kvr.kvr_paged_append(self.desc, self.cache, k, v, self.len, rope=self.rope, q=q, stream=stream, **kw)
        kvr.kvr_paged_decode(self.desc, self.cache, q, self.len, self.out, self.ws, n_new=1, stream=stream)

    def rows(self, r, m):
        """(keys, values) [Hkv, m, d] of a sequence."""
        pages = self.table[r].long()
        return [torch.cat(self.pool[pages, i].unbind(0), 1)[:, :m] for i in (0, 1)]


@DTYPES
@pytest.mark.parametrize("ps", [16, 64])
def test_conversations_against_the_dense_calls(dt, ps):
    """Three prompts, then five steps of all three; each next to a dense cache of its own."""
    heads = (8, 2, 128)
    Hq, Hkv, d = heads
    prompts, steps = [37, 1, 200], 5
    s = Server(dt, heads, ps, 3, 256)
    dense = [[torch.zeros((Hkv, s.desc.capacity, d), dtype=dt, device=DEV) for _ in range(2)] for _ in prompts]
    x = [draw(s.g, dt, m, Hq + 2 * Hkv, d) for m in prompts]
    for (kc, vc), y in zip(dense, x):
        m = y.shape[0]
        kvr.kvr_prefill_rope(s.desc, s.rope, y[:, :Hq].contiguous(), y[:, Hq:Hq + Hkv].contiguous(), y[:, Hq + Hkv:].contiguous(), m,
                             torch.empty((m, Hq, d), dtype=dt, device=DEV), kc, vc)
    every = torch.cat(x)
    cu = torch.tensor([0, 37, 38, 238], dtype=torch.int32, device=DEV)
    kvr.kvr_paged_append(s.desc, s.cache, every[:, Hq:Hq + Hkv], every[:, Hq + Hkv:], s.len, rope=s.rope, cu_seqlens=cu)
    s.len += cu[1:] - cu[:-1]
    for i in range(steps):
        y = draw(s.g, dt, 3, Hq + 2 * Hkv, d)
        want = torch.empty((3, Hq, d), dtype=dt, device=DEV)
        for r, (kc, vc) in enumerate(dense):
            q, k, v = (z[r:r + 1].contiguous() for z in (y[:, :Hq], y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:]))
            m = prompts[r] + i
            kvr.kvr_continue_rope(s.desc, s.rope, q, k, v, kc, vc, m, 1, want[r:r + 1], kvr.workspace_for_rope(s.desc, m, 1), append=True)
        s.step(y[:, :Hq], y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:])
        s.len += 1
        torch.cuda.synchronize()
        for r, caches in enumerate(dense):
            m = prompts[r] + i + 1
            assert all(same_bits(a, c[:, :m]) for a, c in zip(s.rows(r, m), caches))
        assert float((s.out.float() - want.float()).abs().max()) <= TOL[dt]


@DTYPES
@pytest.mark.parametrize("reach", [208, 1600], ids=["one_launch", "shared_out"])
def test_a_captured_step_serves_a_whole_decode(dt, reach):
    """Append, decode and the lengths' update in one graph, replayed with new tokens, eager work between; an
    eager server does the same steps.  A slot leaves the batch on the way."""
    heads, n = (16, 2, 64), 5
    Hq, Hkv, d = heads
    a, b = (Server(dt, heads, 16, n, reach, seed=3) for _ in range(2))
    assert (a.ws.numel() > 0) == (reach == 1600)
    x = draw(a.g, dt, n, Hq + 2 * Hkv, d)
    w = [draw(a.g, dt, d) for _ in range(2)]
    q = torch.empty((n, Hq, d), dtype=dt, device=DEV)
    long = reach - 100
    start = torch.tensor([long, 0, 14, 15, long // 2], dtype=torch.int32, device=DEV)
    for s in (a, b):
        s.pool.normal_(generator=torch.Generator(device=DEV).manual_seed(9))
        s.len.copy_(start)

    def step(s, x, q):
        kvr.kvr_paged_append(s.desc, s.cache, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], s.len, rope=s.rope, q=x[:, :Hq], q_out=q,
                             q_norm=w[0], k_norm=w[1])
        kvr.kvr_paged_decode(s.desc, s.cache, q, s.len, s.out, s.ws, n_new=1)
        s.len += (s.len >= 0).to(torch.int32)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(a, x, q)
    torch.cuda.current_stream().wait_stream(side)
    a.len.copy_(start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, x, q)
    q2 = torch.empty_like(q)
    for i in range(6):
        x.copy_(draw(a.g, dt, n, Hq + 2 * Hkv, d))
        if i == 3:
            for s in (a, b):
                s.len[2] = -1
        graph.replay()
        step(b, x, q2)
        torch.cuda.synchronize()
        assert same_bits(a.out, b.out) and same_bits(a.pool, b.pool) and torch.equal(a.len, b.len)
        assert i >= 3 or same_bits(q, q2)
    assert a.len.tolist() == [long + 6, 6, -1, 21, long // 2 + 6]


def test_two_streams_at_once():
    """Each with its own server and workspace, many steps without a wait between the two."""
    heads = (32, 8, 128)
    Hq, Hkv, d = heads
    one = [Server(BF16, heads, 16, 3, 1200, seed=i) for i in range(2)]
    two = [Server(BF16, heads, 16, 3, 1200, seed=i) for i in range(2)]
    xs = [[draw(s.g, BF16, 3, Hq + 2 * Hkv, d) for _ in range(8)] for s in one]
    for s in one + two:
        s.pool.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
        s.len.copy_(torch.tensor([1100, 3, 640], dtype=torch.int32))
    outs = [[], []]
    for s, x, o in zip(one, xs, outs):
        for y in x:
            y = y.clone()
            s.step(y[:, :Hq], y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:])
            s.len += 1
            o.append(s.out.clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in two]
    got = [[], []]
    for j in range(8):
        for s, x, o, st in zip(two, xs, got, streams):
            with torch.cuda.stream(st):
                y = x[j].clone()
                s.step(y[:, :Hq], y[:, Hq:Hq + Hkv], y[:, Hq + Hkv:])
                s.len += 1
                o.append(s.out.clone())
    torch.cuda.synchronize()
    for a, b in zip(outs, got):
        assert all(same_bits(x, y) for x, y in zip(a, b))


def test_a_stream_that_is_given():
    s, t = (Server(F16, (8, 2, 64), 16, 4, 600, seed=2) for _ in range(2))
    for x in (s, t):
        x.pool.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
        x.len.fill_(555)
    y = draw(s.g, F16, 4, 12, 64)
    z = y.clone()
    s.step(y[:, :8], y[:, 8:10], y[:, 10:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    t.step(z[:, :8], z[:, 8:10], z[:, 10:], stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert same_bits(s.out, t.out) and same_bits(s.pool, t.pool) and same_bits(y, z)


@DTYPES
def test_a_batch_with_norms_against_the_oracle(dt):
    heads, lens = (12, 3, 128), [0, 900, -1, 63, 64]
    Hq, Hkv, d = heads
    s = Server(dt, heads, 32, 5, 1000, seed=6)
    s.pool.normal_(generator=s.g)
    s.len.copy_(torch.tensor(lens, dtype=torch.int32))
    x = draw(s.g, dt, 5, Hq + 2 * Hkv, d)
    qn, kn = (1 + 0.2 * torch.randn(d, generator=s.g, device=DEV).to(dt) for _ in range(2))
    q, k = x[:, :Hq].clone(), x[:, Hq:Hq + Hkv].clone()
    pos = torch.tensor([max(m, 0) for m in lens], dtype=torch.int32, device=DEV)
    kvr.kvr_qk_norm_rope(s.desc, q, k, rope=s.rope, q_norm=qn, k_norm=kn, pos=pos)
    s.step(x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], q_norm=qn, k_norm=kn)
    torch.cuda.synchronize()
    on = [r for r, m in enumerate(lens) if m >= 0]
    assert same_bits(x[on, :Hq], q[on])
    for r in on:
        assert same_bits(s.rows(r, lens[r] + 1)[0][:, -1], k[r])
    kp, vp, table = s.pool[:, 0].cpu(), s.pool[:, 1].cpu(), s.table.cpu().numpy()
    rows = [m + 1 if m >= 0 else -1 for m in lens]
    want, mass = P.decode(q, kp, vp, table, rows)
    b = bound(dt, want, mass, P._f64(q), np.abs(P._f64(kp)).max((0, 2)), np.maximum(rows, 0))
    err = np.abs(P._f64(s.out) - want)
    assert (err[on] <= b[on]).all()


def test_the_binding_refuses_what_does_not_fit_together():
    s = Server(BF16, (8, 2, 64), 16, 3, 64)
    q, k = draw(s.g, BF16, 3, 8, 64), draw(s.g, BF16, 3, 2, 64)
    before = s.pool.clone()
    kp, vp = s.pool[:, 0], s.pool[:, 1]
    ints = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    for f in (lambda: kvr.PagedCache(s.desc, kp, vp, s.table.long()),                       # the table's type
              lambda: kvr.PagedCache(s.desc, kp, vp, s.table[:, ::2]),                      # not contiguous
              lambda: kvr.PagedCache(s.desc, kp, vp.contiguous(), s.table),                 # pages another distance apart
              lambda: kvr.PagedCache(s.desc, kp.transpose(1, 2), vp.transpose(1, 2), s.table),
              lambda: kvr.PagedCache(s.desc, kp.half(), vp.half(), s.table),
              lambda: kvr.kvr_paged_append(s.desc, s.cache, k[:2], k, s.len),
              lambda: kvr.kvr_paged_append(s.desc, s.cache, k.float(), k, s.len),
              lambda: kvr.kvr_paged_append(s.desc, s.cache, k[..., ::2], k, s.len),
              lambda: kvr.kvr_paged_append(s.desc, s.cache, k, k, s.len.long()),
              lambda: kvr.kvr_paged_append(s.desc, s.cache, k, k, s.len[:2]),
              lambda: kvr.kvr_paged_append(s.desc, s.cache, k, k, s.len, cu_seqlens=ints(3)),
              lambda: kvr.kvr_paged_append(s.desc, s.cache, k, k, s.len, pos=ints(2)),
              lambda: kvr.kvr_paged_append(s.desc, s.cache, k, k, s.len, k_norm=k[0]),
              lambda: kvr.kvr_paged_append(s.desc, s.cache, k, k, s.len, q_out=q),
              lambda: kvr.kvr_paged_append(kvr.make_desc(8, 4, 64, BF16, 0), s.cache, k, k, s.len),
              lambda: kvr.kvr_paged_append(s.desc, s.cache, k, k, s.len, rope=kvr.RopeTable(128, 64)),
              lambda: kvr.kvr_paged_decode(s.desc, s.cache, k, s.len, s.out, s.ws),
              lambda: kvr.kvr_paged_decode(s.desc, s.cache, q, s.len, s.out[:2], s.ws),
              lambda: kvr.kvr_paged_decode(s.desc, s.cache, q, s.len, s.out.transpose(0, 1).contiguous().transpose(0, 1), s.ws),
              lambda: kvr.kvr_qk_norm_rope(s.desc, q, k, k_out=q),
              lambda: kvr.kvr_qk_norm_rope(s.desc, None, k, q_out=q)):
        with pytest.raises(ValueError):
            f()
    for f, status in ((lambda: kvr.kvr_paged_decode(s.desc, s.cache, q, s.len, s.out, s.ws, max_len=65), kvr.KVR_ERR_CAPACITY),
                      (lambda: kvr.kvr_paged_append(s.desc, s.cache, k, k, s.len, rope=kvr.RopeTable(64, 63)), kvr.KVR_ERR_POSITION),
                      (lambda: kvr.kvr_paged_append(s.desc, s.cache, k[:2], k[:2], s.len), kvr.KVR_ERR_SHAPE),
                      (lambda: kvr.kvr_qk_norm_rope(s.desc, q[:, :1].expand(3, 8, 64), None), kvr.KVR_ERR_SHAPE)):
        with pytest.raises(kvr.KvrError) as e:
            f()
        assert e.value.status == status
    torch.cuda.synchronize()
    assert same_bits(s.pool, before)
