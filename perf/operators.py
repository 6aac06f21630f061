"""Timed calls of the operators that serve many readers from one cached document.

  shared  attention of a batch of readers that share a long cached prefix and
          each have cached rows of their own (`kvr_continue_shared`): the
          prefix is computed once for all, the new rows go to the readers' own
          caches in the same call
  weigh   the attention weight that each cached row receives, accumulated over
          the query rows and heads of its kv head (`kvr_cache_weigh`)
  evict   a smaller cache of the rows with the most accumulated weight
          (`kvr_cache_evict`)

With `own` false, `run` computes them from elementary torch operations in 32
bits, rounded once at the end; with `own` true it calls the library.

The definitions.  Query row (r, i) of reader r, head h, kv head g = h / G:

  shared  position P = pos0 + len[r] + i; q and the new keys are rotated there
          (rotary embedding, half-split pairs, base 10^6) and rounded to the
          element type where the case says so;
          out = softmax(scale * q . k) v over the prefix rows 0 .. L - 1, the
          reader's own cached rows 0 .. len[r] - 1 and its new rows 0 .. i;
          own rows len[r] .. len[r] + S - 1 receive the new keys and values.
          A reader with len[r] < 0 takes no part: its rows stay as they were.
  weigh   weight[g][j] += sum of softmax_j(scale * q_(i,h) . k_g) over the
          query rows i and the heads h of g, row i at position L + i seeing
          keys 0 .. L + i (the last S of them its own rows)
  evict   of rows 0 .. L - 1 of each kv head the first n_first, the last
          n_last, and of the others those with the largest weight (the lower
          row where weights are equal), n_keep in all, in ascending order
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
ELT = {"bf16": 2, "fp16": 2, "f32": 4}
ROPE_BASE = 1.0e6


def _case(name, op, **kw):
    c = {"name": name, "op": op, "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16"}
    c.update(kw)
    return c


def listed():
    return [
        # two readers of a short document begin their answers: launches and latency count
        _case("shared_2x1_255", "shared", L=255, n=2, S=1, lo=1, hi=13, cap=64, rope=True, append=True, dtype="fp16"),
        # a handful of readers in the middle of their answers, one slot of the batch empty
        _case("shared_9x1_3774", "shared", L=3774, n=9, S=1, lo=-1, hi=256, cap=512, rope=True, append=True),
        # the full batch decodes over one document
        _case("shared_64x1_3774", "shared", L=3774, n=64, S=1, lo=24, hi=512, cap=600, rope=True, append=True),
        # drafted tokens: four query rows a reader, not kept until they are accepted
        _case("shared_16x4_16384", "shared", L=16384, n=16, S=4, lo=100, hi=300, cap=304, rope=False, append=False,
              dtype="fp16"),
        # the longest document, the largest batch, long answers
        _case("shared_64x1_32768", "shared", L=32768, n=64, S=1, lo=300, hi=1000, cap=1024, rope=True, append=True),
        # the full-precision path at head_dim 64, odd sizes
        _case("shared_3x5_945_f32", "shared", L=945, n=3, S=5, lo=0, hi=77, cap=96, rope=True, append=True, dtype="f32",
              hq=16, hkv=2, d=64),
        # each decoded token adds its weights
        _case("weigh_1_3774", "weigh", L=3774, S=1),
        # a question's tokens
        _case("weigh_24_16384", "weigh", L=16384, S=24, dtype="fp16"),
        # the last tokens of a long prefill as the window that decides what is kept
        _case("weigh_128_32640", "weigh", L=32640, S=128),
        # a paragraph's cache halved
        _case("evict_1024", "evict", L=1024, keep=512, first=4, last=32),
        # a document's cache with its question, to a quarter
        _case("evict_3798", "evict", L=3798, keep=945, first=4, last=24, dtype="fp16"),
        # the longest document, to a quarter
        _case("evict_32768", "evict", L=32768, keep=8192, first=4, last=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["shared", "shared", "weigh", "evict"])
    heads = rng.choice([(32, 8, 128), (32, 8, 128), (32, 8, 128), (8, 8, 128), (12, 3, 128), (64, 8, 128),
                        (16, 2, 64), (8, 2, 64)])
    c = {"op": op, "hq": heads[0], "hkv": heads[1], "d": heads[2],
         "dtype": rng.choice(["bf16", "bf16", "fp16", "f32"])}
    f32 = c["dtype"] == "f32"
    if op == "shared":
        n, S = _log(rng, 1, 16 if f32 else 64), rng.choice([1, 1, 1, 2, 3, 5, 8])
        while n * S * c["hq"] > 2048:      # at most the rows of the largest listed case
            n = (n + 1) // 2
            S = (S + 1) // 2
        hi = _log(rng, 8, 1000)
        c.update(L=_log(rng, 64, 4096 if f32 else 32768), n=n, S=S, lo=rng.choice([-1, 0, hi // 3]), hi=hi,
                 cap=hi + S + rng.randint(0, 8), rope=rng.choice([True, True, False]),
                 append=rng.choice([True, True, False]))
    elif op == "weigh":
        S = _log(rng, 1, 24 if f32 else 128)
        while S * c["hq"] > 4096:
            S = (S + 1) // 2
        c.update(L=_log(rng, 64, 4096 if f32 else 32640), S=S)
    else:
        L = _log(rng, 256, 8192 if f32 else 32768)
        first, last = rng.choice([0, 1, 4]), rng.choice([0, 24, 32])
        c.update(L=L, first=first, last=last, keep=max(first + last, int(L * rng.choice([0.1, 0.25, 0.5, 0.9]))))
    return c


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _lengths(c, seed):
    """Cached rows of each reader: n values spread evenly over [lo, hi], in the seed's order."""
    n = c["n"]
    v = [c["lo"] + (c["hi"] - c["lo"]) * i // max(1, n - 1) for i in range(n)]
    g = torch.Generator()
    g.manual_seed(int(seed))
    return [v[i] for i in torch.randperm(n, generator=g).tolist()]


def _direction(g, c):
    """Per kv head, the unit vector along which queries lean and by which some keys draw attention."""
    u = _randn(g, c["hkv"], c["d"])
    return u / u.norm(dim=1, keepdim=True)


def _queries(g, c, u, *rows):
    """N(0, 1) plus a common component, which gives keys along u a head start."""
    G = c["hq"] // c["hkv"]
    q = _randn(g, *rows, c["hq"], c["d"]) + 4.0 * u.repeat_interleave(G, 0)
    return q.to(DTYPES[c["dtype"]])


def _keys(g, c, u, L):
    """[hkv, L, d]: N(0, 1) plus u times a strength, large on the first four rows and on a few others."""
    k = _randn(g, c["hkv"], L, c["d"])
    a = torch.empty((c["hkv"], L, 1), device="cuda").exponential_(1.0, generator=g)
    a[:, :4] = 14.0
    return (k + a * u[:, None, :]).to(DTYPES[c["dtype"]])


def prepare(case, seed):
    c = case
    g = _gen(seed)
    dt = DTYPES[c["dtype"]]
    hkv, d, L = c["hkv"], c["d"], c["L"]
    st = {"case": c}
    if c["op"] == "shared":
        n, S, cap = c["n"], c["S"], c["cap"]
        u = _direction(g, c)
        st.update(q=_queries(g, c, u, n, S), k=_randn(g, n, S, hkv, d).to(dt), v=_randn(g, n, S, hkv, d).to(dt),
                  kc=_keys(g, c, u, L), vc=_randn(g, hkv, L, d).to(dt), kt=_randn(g, n, hkv, cap, d).to(dt),
                  vt=_randn(g, n, hkv, cap, d).to(dt), len=torch.tensor(_lengths(c, seed), dtype=torch.int32, device="cuda"),
                  out=torch.zeros((n, S, c["hq"], d), dtype=dt, device="cuda"))
        if c["rope"]:
            angle = _angles(torch.arange(L + cap + S, device="cuda"), d)
            st["cs"] = torch.stack((angle.cos(), angle.sin()), -1).float()
    elif c["op"] == "weigh":
        S = c["S"]
        u = _direction(g, c)
        st.update(q=_queries(g, c, u, S), k=_randn(g, S, hkv, d).to(dt), kc=_keys(g, c, u, L + S),
                  weight=torch.rand((hkv, L + S), generator=g, device="cuda"))
    else:
        weight = _randn(g, hkv, L).mul_(2.0).exp_()
        weight[torch.rand((hkv, L), generator=g, device="cuda") < 0.1] = 0.0      # rows that nobody looked at
        st.update(kc=_randn(g, hkv, L, d).to(dt), vc=_randn(g, hkv, L, d).to(dt), weight=weight,
                  ko=torch.zeros((hkv, c["keep"], d), dtype=dt, device="cuda"),
                  vo=torch.zeros((hkv, c["keep"], d), dtype=dt, device="cuda"),
                  wo=torch.zeros((hkv, c["keep"]), device="cuda"),
                  index=torch.zeros((hkv, c["keep"]), dtype=torch.int32, device="cuda"))
    if own:
        st.update(_handles(c))
    return st


def _angles(pos, d):
    """Angles of positions' pairs, in 64 bits: [..., d / 2]."""
    i = torch.arange(d // 2, dtype=torch.float64, device=pos.device)
    return pos.double()[..., None] * ROPE_BASE ** (-2.0 * i / d)


def _handles(c):
    """What a program keeps beside its tensors: descriptor, workspace, rotary table."""
    from paper_2606_13361_amd import kvr
    capacity = c["L"] + c["S"] if c["op"] == "weigh" else c["L"]
    desc = kvr.make_desc(c["hq"], c["hkv"], c["d"], DTYPES[c["dtype"]], capacity)
    if c["op"] == "shared":
        rope = kvr.RopeTable(c["d"], c["L"] + c["cap"] + c["S"], base=ROPE_BASE) if c["rope"] else None
        return {"desc": desc, "rope": rope, "ws": kvr.workspace_for_shared(desc, c["L"], c["n"], c["S"], c["cap"])}
    if c["op"] == "weigh":
        return {"desc": desc, "ws": kvr.workspace_for_weigh(desc, c["L"], c["S"])}
    return {"desc": desc, "ws": kvr.workspace_for_evict(desc, c["L"])}


# ------------------------------------------------------------------ one pass
def run(state):
    op = state["case"]["op"]
    if own:
        return {"shared": _own_shared, "weigh": _own_weigh, "evict": _own_evict}[op](state)
    return {"shared": _plain_shared, "weigh": _plain_weigh, "evict": _plain_evict}[op](state)


def _own_shared(s):
    from paper_2606_13361_amd import kvr
    c = s["case"]
    kvr.kvr_continue_shared(s["desc"], s["q"], s["k"], s["v"], s["kc"], s["vc"], c["L"], s["kt"], s["vt"], s["len"],
                            s["out"], s["ws"], rope=s["rope"], append=c["append"])
    return {"out": s["out"], "ktail": s["kt"], "vtail": s["vt"]}


def _own_weigh(s):
    from paper_2606_13361_amd import kvr
    c = s["case"]
    kvr.kvr_cache_weigh(s["desc"], s["q"], s["k"], s["kc"], c["L"], c["S"], s["weight"], s["ws"])
    return s["weight"]


def _own_evict(s):
    from paper_2606_13361_amd import kvr
    c = s["case"]
    kvr.kvr_cache_evict(s["desc"], s["kc"], s["vc"], c["L"], s["weight"], c["keep"], s["ko"], s["vo"],
                        n_first=c["first"], n_last=c["last"], weight_out=s["wo"], index=s["index"], ws=s["ws"])
    return {"k": s["ko"], "v": s["vo"], "weight": s["wo"], "index": s["index"]}


# ------------------------------------------------------------------ plain forms
def _rotate(x, cs):
    """x [n, S, heads, d] by the (cos, sin) of its positions, cs [n, S, d / 2, 2], rounded to x's type."""
    h = x.shape[-1] // 2
    a, b = x[..., :h].float(), x[..., h:].float()
    cos, sin = cs[:, :, None, :, 0], cs[:, :, None, :, 1]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(x.dtype)


def _plain_shared(s):
    c = s["case"]
    n, S, L, cap, hkv, d = c["n"], c["S"], c["L"], c["cap"], c["hkv"], c["d"]
    G = c["hq"] // hkv
    dev = s["q"].device
    on = s["len"] >= 0
    ln = s["len"].clamp(min=0).long()
    q, k = s["q"], s["k"]
    at = ln[:, None] + torch.arange(S, device=dev)                       # [n, S] rows of the new tokens
    if c["rope"]:
        cs = s["cs"][L + at]
        q, k = _rotate(q, cs), _rotate(k, cs)
    # [hkv, n, S G, d] queries; scores against prefix, own cached rows, new rows
    qh = q.float().view(n, S, hkv, G, d).permute(2, 0, 1, 3, 4).reshape(hkv, n * S * G, d)
    qr = qh.view(hkv, n, S * G, d).transpose(0, 1).reshape(n * hkv, S * G, d)
    new_k = k.float().transpose(1, 2).reshape(n * hkv, S, d)
    new_v = s["v"].float().transpose(1, 2).reshape(n * hkv, S, d)
    s1 = torch.bmm(qh, s["kc"].float().transpose(1, 2).contiguous()).view(hkv, n, S * G, L).transpose(0, 1)
    s2 = torch.bmm(qr, s["kt"].float().view(n * hkv, cap, d).transpose(1, 2).contiguous()).view(n, hkv, S * G, cap)
    s3 = torch.bmm(qr, new_k.transpose(1, 2).contiguous()).view(n, hkv, S * G, S)
    s2 = s2.masked_fill((torch.arange(cap, device=dev) >= ln[:, None])[:, None, None, :], -math.inf)
    row = torch.arange(S * G, device=dev) // G
    s3 = s3.masked_fill(torch.arange(S, device=dev) > row[:, None], -math.inf)
    p = torch.cat((s1, s2, s3), -1) * (1.0 / math.sqrt(d))
    p = (p - p.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1, keepdim=True)
    p1, p2, p3 = p.split((L, cap, S), -1)
    vt = s["vt"].float().masked_fill((torch.arange(cap, device=dev) >= ln[:, None])[:, None, :, None], 0.0)
    o = torch.bmm(p1.transpose(0, 1).reshape(hkv, n * S * G, L), s["vc"].float()).view(hkv, n, S * G, d).transpose(0, 1)
    o = o + torch.bmm(p2.reshape(n * hkv, S * G, cap), vt.view(n * hkv, cap, d)).view(n, hkv, S * G, d)
    o = (o + torch.bmm(p3.reshape(n * hkv, S * G, S), new_v).view(n, hkv, S * G, d)) / total
    o = o.view(n, hkv, S, G, d).transpose(1, 2).reshape(n, S, c["hq"], d).to(s["out"].dtype)
    s["out"].copy_(torch.where(on[:, None, None, None], o, s["out"]))
    if c["append"]:
        # a slot that takes no part writes back what its rows hold
        r = torch.arange(n, device=dev)[:, None]
        for_all = on[:, None, None, None]
        s["kt"][r, :, at] = torch.where(for_all, k, s["kt"][r, :, at])
        s["vt"][r, :, at] = torch.where(for_all, s["v"], s["vt"][r, :, at])
    return {"out": s["out"], "ktail": s["kt"], "vtail": s["vt"]}


def _plain_weigh(s):
    c = s["case"]
    S, L, hkv, d = c["S"], c["L"], c["hkv"], c["d"]
    G = c["hq"] // hkv
    q = s["q"].float().view(S, hkv, G, d).permute(1, 0, 2, 3).reshape(hkv, S * G, d)
    k = torch.cat((s["kc"][:, :L], s["k"].transpose(0, 1)), 1).float()
    p = torch.bmm(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(d))
    row = torch.arange(S * G, device=p.device) // G
    p = p.masked_fill(torch.arange(L + S, device=p.device) > L + row[:, None], -math.inf)
    p = (p - p.amax(-1, keepdim=True)).exp_()
    s["weight"] += (p / p.sum(-1, keepdim=True)).sum(1)
    return s["weight"]


def _plain_evict(s):
    c = s["case"]
    L, keep, d = c["L"], c["keep"], c["d"]
    w = s["weight"].clone()
    w[:, :c["first"]] = math.inf
    w[:, L - c["last"]:] = math.inf
    index = torch.sort(w, dim=1, descending=True, stable=True)[1][:, :keep].sort(1)[0]
    rows = index[:, :, None].expand(-1, -1, d)
    s["ko"].copy_(s["kc"].gather(1, rows))
    s["vo"].copy_(s["vc"].gather(1, rows))
    s["wo"].copy_(s["weight"].gather(1, index))
    s["index"].copy_(index)
    return {"k": s["ko"], "v": s["vo"], "weight": s["wo"], "index": s["index"]}


# ------------------------------------------------------------------ work
def work(case):
    c = case
    e, hq, hkv, d, L = ELT[c["dtype"]], c["hq"], c["hkv"], c["d"], c["L"]
    if c["op"] == "shared":
        lens = [v for v in _lengths(c, 0) if v >= 0]
        S, rows, own_rows = c["S"], len(lens) * c["S"], sum(lens)
        # queries and outputs, new rows (and where they go), own cached rows, the prefix once
        moved = 2 * rows * hq + 2 * (rows * (2 if c["append"] else 1) + own_rows + L) * hkv
        keys = rows * L + S * own_rows + len(lens) * S * (S + 1) // 2
        return {"bytes": moved * d * e + 4 * c["n"], "flops": 4.0 * d * hq * keys}
    if c["op"] == "weigh":
        S = c["S"]
        return {"bytes": (S * hq + (L + S) * hkv) * d * e + 8 * hkv * (L + S),
                "flops": 2.0 * d * hq * (S * L + S * (S + 1) // 2)}
    # every weight; the kept rows, read and written, with their weights and indices
    return {"bytes": hkv * (4 * L + c["keep"] * (4 * d * e + 8)), "flops": float(hkv * L)}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return {"shared": _exact_shared, "weigh": _exact_weigh, "evict": _exact_evict}[case["op"]](s)


def _softmax64(scores):
    e = torch.exp(scores - scores.max(-1, keepdim=True).values)
    return e / e.sum(-1, keepdim=True)


def _turn64(x, angle):
    """Each pair (x[i], x[i + d/2]) as a complex number, times e^(i angle), then rounded to x's type."""
    h = x.shape[-1] // 2
    z = torch.complex(x[..., :h].double(), x[..., h:].double()) * torch.polar(torch.ones_like(angle), angle)
    return torch.cat((z.real, z.imag), -1).to(x.dtype)


def _exact_shared(s):
    """Reader by reader, over its whole key sequence."""
    c = s["case"]
    S, L, hq, hkv, d = c["S"], c["L"], c["hq"], c["hkv"], c["d"]
    G = hq // hkv
    out, kt, vt = s["out"].double(), s["kt"].double(), s["vt"].double()
    kc, vc = s["kc"].double(), s["vc"].double()
    for r, n in enumerate(s["len"].tolist()):
        if n < 0:
            continue
        q, k, v = s["q"][r], s["k"][r], s["v"][r]
        if c["rope"]:
            angle = _angles(L + n + torch.arange(S, device=q.device), d)[:, None, :]
            q, k = _turn64(q, angle), _turn64(k, angle)
        k, v = k.double().transpose(0, 1), v.double().transpose(0, 1)           # [hkv, S, d]
        keys = torch.cat((kc, kt[r, :, :n], k), 1)
        vals = torch.cat((vc, vt[r, :, :n], v), 1)
        qg = q.double().view(S, hkv, G, d).permute(1, 2, 0, 3)                  # [hkv, G, S, d]
        sc = torch.matmul(qg.reshape(hkv, G * S, d), keys.transpose(1, 2)).view(hkv, G, S, L + n + S) / math.sqrt(d)
        late = torch.ones((S, S), dtype=torch.bool, device=q.device).triu(1)
        sc[..., L + n:].masked_fill_(late, -math.inf)
        o = torch.matmul(_softmax64(sc).view(hkv, G * S, -1), vals).view(hkv, G, S, d)
        out[r] = o.permute(2, 0, 1, 3).reshape(S, hq, d)
        if c["append"]:
            kt[r, :, n:n + S], vt[r, :, n:n + S] = k, v
    return {"out": out, "ktail": kt, "vtail": vt}


def _exact_weigh(s):
    """Query token by query token."""
    c = s["case"]
    S, L, hkv, d = c["S"], c["L"], c["hkv"], c["d"]
    G = c["hq"] // hkv
    weight = s["weight"].double()
    keys = torch.cat((s["kc"][:, :L].double(), s["k"].double().transpose(0, 1)), 1)
    for i in range(S):
        q = s["q"][i].double().view(hkv, G, d)
        p = _softmax64(torch.matmul(q, keys[:, :L + i + 1].transpose(1, 2)) / math.sqrt(d))
        weight[:, :L + i + 1] += p.sum(1)
    return weight


def _exact_evict(s):
    """Weight by weight on the host: rows ordered by (weight falling, row rising)."""
    c = s["case"]
    L, first, last = c["L"], c["first"], c["last"]
    always = set(range(first)) | set(range(L - last, L))
    index = []
    for w in s["weight"].double().tolist():
        others = sorted((j for j in range(first, L - last)), key=lambda j: (-w[j], j))
        index.append(sorted(always | set(others[:c["keep"] - len(always)])))
    at = torch.tensor(index, device=s["kc"].device)
    head = torch.arange(c["hkv"], device=at.device)[:, None]
    return {"k": s["kc"][head, at].double(), "v": s["vc"][head, at].double(), "weight": s["weight"][head, at].double(),
            "index": at.int()}
