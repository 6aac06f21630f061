"""kvr_continue_shared, kvr_cache_weigh and kvr_cache_evict without a GPU: every
invalid argument is rejected on the host before any HIP call, zero-length work is a
no-op, and the Python binding checks tensors before it calls.  Pointers are fake
integers, never dereferenced."""
import ctypes
import os

import pytest
import torch

from paper_2606_13361_amd import kvr

A = 0x10000
MIS = 0x10008
FAR = 1 << 44       # buffers of evict are this far apart


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kvr.LIB_PATH):
        from paper_2606_13361_amd import build
        build.build()
    return kvr.load()


def desc(**kw):
    d = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=kvr.KVR_BF16, capacity=4096, scale=0.0)
    d.update(kw)
    return kvr.make_desc(**d)


def shared(lib, d=None, rope=None, Q=A, K=A, V=A, n=4, S=2, kc=A, vc=A, L=100, pos0=100, kt=A, vt=A, tcap=64, ln=A,
           append=1, out=A, ws=A, wsb=1 << 40):
    d = desc() if d is None else d
    r = None if rope is None else ctypes.byref(rope)
    return lib.kvr_continue_shared(ctypes.byref(d), r, Q, K, V, n, S, kc, vc, L, pos0, kt, vt, tcap, ln, append, out, ws,
                                   wsb, None)


def weigh(lib, d=None, Q=A, K=A, kc=A, L=100, S=2, w=A, ws=A, wsb=1 << 40):
    d = desc() if d is None else d
    return lib.kvr_cache_weigh(ctypes.byref(d), Q, K, kc, L, S, w, ws, wsb, None)


def evict(lib, d=None, kc=FAR, vc=2 * FAR, L=100, w=3 * FAR, first=1, last=2, keep=50, ko=4 * FAR, vo=5 * FAR, cap=64,
          wo=6 * FAR, ix=7 * FAR, ws=8 * FAR, wsb=1 << 40):
    d = desc() if d is None else d
    return lib.kvr_cache_evict(ctypes.byref(d), kc, vc, L, w, first, last, keep, ko, vo, cap, wo, ix, ws, wsb, None)


BAD_DESC = [
    (dict(n_q_heads=30), kvr.KVR_ERR_SHAPE), (dict(n_kv_heads=0), kvr.KVR_ERR_SHAPE), (dict(head_dim=96), kvr.KVR_ERR_SHAPE),
    (dict(dtype=7), kvr.KVR_ERR_DTYPE), (dict(capacity=-1), kvr.KVR_ERR_SHAPE), (dict(scale=float("nan")), kvr.KVR_ERR_SHAPE),
]


@pytest.mark.parametrize("bad,code", BAD_DESC)
def test_descriptor(lib, bad, code):
    d = desc(**bad)
    assert shared(lib, d) == code and weigh(lib, d) == code and evict(lib, d) == code
    none = ctypes.c_size_t(-1).value
    assert lib.kvr_workspace_bytes_shared(ctypes.byref(d), 10, 1, 1, 10) == none
    assert lib.kvr_workspace_bytes_weigh(ctypes.byref(d), 10, 1) == none
    assert lib.kvr_workspace_bytes_evict(ctypes.byref(d), 10) == none


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), "SHAPE"), (dict(S=-1), "SHAPE"), (dict(L=-1), "SHAPE"), (dict(tcap=-1), "SHAPE"),
    (dict(n=1 << 20, S=1 << 10), "SHAPE"), (dict(L=1 << 31), "SHAPE"), (dict(tcap=1 << 31), "SHAPE"),
    (dict(L=4097), "CAPACITY"), (dict(S=65), "CAPACITY"),
    (dict(Q=None), "NULL"), (dict(K=None), "NULL"), (dict(V=None), "NULL"), (dict(out=None), "NULL"), (dict(ln=None), "NULL"),
    (dict(kc=None), "NULL"), (dict(vc=None), "NULL"), (dict(kt=None), "NULL"), (dict(vt=None), "NULL"),
    (dict(Q=MIS), "ALIGN"), (dict(K=MIS), "ALIGN"), (dict(V=MIS), "ALIGN"), (dict(out=MIS), "ALIGN"), (dict(kc=MIS), "ALIGN"),
    (dict(vc=MIS), "ALIGN"), (dict(kt=MIS), "ALIGN"), (dict(vt=MIS), "ALIGN"), (dict(ws=MIS), "ALIGN"), (dict(ln=A + 2), "ALIGN"),
    (dict(ws=None), "WORKSPACE"), (dict(wsb=64), "WORKSPACE"),
])
def test_shared_refusals(lib, kw, code):
    assert shared(lib, **kw) == getattr(kvr, "KVR_ERR_" + code)


def test_shared_rope_refusals(lib):
    table = lambda n, p=A: kvr.kvr_rope(p, n)
    assert shared(lib, rope=table(163)) == kvr.KVR_ERR_POSITION             # 100 + 64 rows
    assert shared(lib, rope=table(165), append=0) == kvr.KVR_ERR_POSITION   # ... and two tokens past a full one
    assert shared(lib, rope=table(1 << 20), pos0=-1) == kvr.KVR_ERR_POSITION
    assert shared(lib, rope=table(1 << 20, None)) == kvr.KVR_ERR_NULL
    assert shared(lib, rope=table(1 << 20, MIS)) == kvr.KVR_ERR_ALIGN
    assert shared(lib, rope=table(-5)) == kvr.KVR_ERR_POSITION


def test_shared_no_work(lib):
    assert shared(lib, n=0, Q=None, out=None, ws=None, ln=None) == kvr.KVR_OK
    assert shared(lib, S=0, Q=None, out=None, ws=None, ln=None) == kvr.KVR_OK


@pytest.mark.parametrize("kw,code", [
    (dict(L=-1), "SHAPE"), (dict(S=-1), "SHAPE"), (dict(L=1 << 31), "SHAPE"), (dict(S=1 << 30), "SHAPE"),
    (dict(L=4095), "CAPACITY"), (dict(Q=None), "NULL"), (dict(K=None), "NULL"), (dict(kc=None), "NULL"), (dict(w=None), "NULL"),
    (dict(Q=MIS), "ALIGN"), (dict(K=MIS), "ALIGN"), (dict(kc=MIS), "ALIGN"), (dict(w=A + 2), "ALIGN"), (dict(ws=MIS), "ALIGN"),
    (dict(ws=None), "WORKSPACE"), (dict(wsb=8), "WORKSPACE"),
])
def test_weigh_refusals(lib, kw, code):
    assert weigh(lib, **kw) == getattr(kvr, "KVR_ERR_" + code)


def test_weigh_no_work(lib):
    assert weigh(lib, S=0, Q=None, K=None, w=None, ws=None) == kvr.KVR_OK


@pytest.mark.parametrize("kw,code", [
    (dict(L=-1), "SHAPE"), (dict(first=-1), "SHAPE"), (dict(last=-1), "SHAPE"), (dict(keep=-1, first=0, last=0), "SHAPE"),
    (dict(keep=101), "SHAPE"), (dict(first=30, last=21), "SHAPE"), (dict(first=51), "SHAPE"), (dict(cap=-1), "SHAPE"),
    (dict(first=1 << 62, last=1 << 62), "SHAPE"), (dict(L=1 << 31), "SHAPE"),
    (dict(L=4097), "CAPACITY"), (dict(cap=49), "CAPACITY"),
    (dict(kc=None), "NULL"), (dict(vc=None), "NULL"), (dict(w=None), "NULL"), (dict(ko=None), "NULL"), (dict(vo=None), "NULL"),
    (dict(kc=FAR + 8), "ALIGN"), (dict(ko=FAR + 8), "ALIGN"), (dict(w=FAR + 2), "ALIGN"), (dict(ix=FAR + 1), "ALIGN"),
    (dict(wo=FAR + 1), "ALIGN"), (dict(ws=FAR + 4), "ALIGN"),
    # outputs over inputs or each other
    (dict(ko=FAR), "SHAPE"), (dict(vo=FAR + 4096 * 8 * 256 - 16), "SHAPE"), (dict(ko=2 * FAR - 16), "SHAPE"),
    (dict(vo=4 * FAR), "SHAPE"), (dict(wo=3 * FAR), "SHAPE"), (dict(ix=3 * FAR + 16), "SHAPE"),
])
def test_evict_refusals(lib, kw, code):
    assert evict(lib, **kw) == getattr(kvr, "KVR_ERR_" + code)


def test_evict_workspace_of_long_caches(lib):
    d = desc(capacity=70000)
    need = 70000 * 8 * 4
    assert kvr.kvr_workspace_bytes_evict(d, 70000) == need
    assert kvr.kvr_workspace_bytes_evict(d, 32768) == 0
    long = lambda **kw: evict(lib, d, L=70000, **kw)
    assert long(ws=None) == kvr.KVR_ERR_WORKSPACE
    assert long(wsb=need - 1) == kvr.KVR_ERR_WORKSPACE
    assert long(wsb=need, ix=8 * FAR) == kvr.KVR_ERR_SHAPE        # an output in the workspace
    assert long(wsb=need, ws=4 * FAR) == kvr.KVR_ERR_SHAPE


def test_evict_no_work(lib):
    assert evict(lib, keep=0, first=0, last=0, kc=None, vc=None, w=None, ko=None, vo=None, ws=None) == kvr.KVR_OK


def test_workspace_sizes(lib):
    d = desc()
    assert kvr.kvr_workspace_bytes_shared(d, 100, 0, 1, 10) == 0
    assert kvr.kvr_workspace_bytes_weigh(d, 100, 0) == 0
    for n, S in ((1, 1), (9, 1), (64, 2), (3, 40)):
        sizes = [kvr.kvr_workspace_bytes_shared(d, L, n, S, c) for L, c in ((0, 0), (1, 1), (300, 64), (3774, 64), (3774, 600),
                                                                            (32768, 5000))]
        assert sizes == sorted(sizes) and sizes[0] > 0
    for S in (1, 24, 128):
        sizes = [kvr.kvr_workspace_bytes_weigh(d, L, S) for L in (0, 1, 31, 300, 3774, 32768)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    for f in (lambda: kvr.kvr_workspace_bytes_shared(d, -1, 1, 1, 1), lambda: kvr.kvr_workspace_bytes_weigh(d, 1, -1),
              lambda: kvr.kvr_workspace_bytes_evict(d, -1), lambda: kvr.workspace_for_evict(desc(head_dim=7), 4)):
        with pytest.raises(ValueError):
            f()


def test_binding_checks_tensors(lib):
    """CPU tensors, wrong ranks and types: ValueError, nothing called."""
    d = desc(capacity=8)
    q, k = torch.zeros((1, 1, 32, 128), dtype=torch.bfloat16), torch.zeros((1, 1, 8, 128), dtype=torch.bfloat16)
    c = torch.zeros((8, 8, 128), dtype=torch.bfloat16)
    ln = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        kvr.kvr_continue_shared(d, q, k, k, c, c, 4, None, None, ln, q, None)
    with pytest.raises(ValueError, match="Qs must be"):
        kvr.kvr_continue_shared(d, q[0], k, k, c, c, 4, None, None, ln, q, None)
    with pytest.raises(ValueError, match="on the GPU"):
        kvr.kvr_cache_weigh(d, q[0], k[0], c, 4, 1, torch.zeros((8, 8)), None)
    with pytest.raises(ValueError, match="on the GPU"):
        kvr.kvr_cache_evict(d, c, c, 4, torch.zeros((8, 8)), 2, c, c)
