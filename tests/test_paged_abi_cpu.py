"""kvr_qk_norm_rope, kvr_paged_append and kvr_paged_decode without a GPU: every invalid argument
is rejected on the host before any HIP call, work of no size is a no-op, and the Python
binding checks tensors before it calls.  Pointers are fake integers, never dereferenced."""
import ctypes
import os

import pytest
import torch

from paper_2606_13361_amd import kvr

A = 0x10000
MIS = 0x10008


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(kvr.LIB_PATH):
        from paper_2606_13361_amd import build
        build.build()
    return kvr.load()


def desc(**kw):
    d = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=kvr.KVR_BF16, capacity=0, scale=0.0)
    d.update(kw)
    return kvr.make_desc(**d)


def rows(heads=8, data=A, token=None, head=128):
    return kvr.kvr_rows(data, heads * 128 if token is None else token, head)


def pages(k=A, v=A, stride=8 * 16 * 128, n_pages=9, size=16, table=A, max_pages=5, reserved=0):
    return kvr.kvr_pages(k, v, stride, n_pages, size, table, max_pages, reserved)


def ref(x):
    return None if x is None else ctypes.byref(x)


DEFAULT = object()


def given(x, heads):
    return rows(heads) if x is DEFAULT else x


def norm_rope(lib, d=None, rope=None, q=DEFAULT, k=DEFAULT, qn=A, kn=A, eps=1e-6, n=4, pos=None, pos0=0, qo=DEFAULT, ko=DEFAULT):
    d = desc() if d is None else d
    return lib.kvr_qk_norm_rope(ctypes.byref(d), ref(rope), ref(given(q, 32)), ref(given(k, 8)), qn, kn, eps, n, pos, pos0,
                                ref(given(qo, 32)), ref(given(ko, 8)), None)


def append(lib, d=None, g=DEFAULT, rope=None, k=DEFAULT, v=DEFAULT, q=DEFAULT, qn=A, kn=A, eps=1e-6, n=4, T=6, cu=A, ln=A,
           pos=None, qo=DEFAULT):
    d = desc() if d is None else d
    g = pages() if g is DEFAULT else g
    return lib.kvr_paged_append(ctypes.byref(d), ref(g), ref(rope), ref(given(k, 8)), ref(given(v, 8)), ref(given(q, 32)), qn,
                                kn, eps, n, T, cu, ln, pos, ref(given(qo, 32)), None)


def decode(lib, d=None, g=DEFAULT, q=DEFAULT, n=4, ln=A, n_new=1, most=80, out=A, ws=A, wsb=1 << 40):
    d = desc() if d is None else d
    g = pages() if g is DEFAULT else g
    return lib.kvr_paged_decode(ctypes.byref(d), ref(g), ref(given(q, 32)), n, ln, n_new, most, out, ws, wsb, None)


LONG = dict(max_pages=4096)      # a table of 65536 rows: several workgroups to a sequence


@pytest.mark.parametrize("bad,code", [
    (dict(n_q_heads=30), kvr.KVR_ERR_SHAPE), (dict(n_kv_heads=0), kvr.KVR_ERR_SHAPE), (dict(head_dim=96), kvr.KVR_ERR_SHAPE),
    (dict(dtype=7), kvr.KVR_ERR_DTYPE), (dict(capacity=-1), kvr.KVR_ERR_SHAPE), (dict(scale=float("nan")), kvr.KVR_ERR_SHAPE),
])
def test_descriptor(lib, bad, code):
    d = desc(**bad)
    assert norm_rope(lib, d) == code and append(lib, d) == code and decode(lib, d) == code
    assert lib.kvr_workspace_bytes_paged(ctypes.byref(d), 4, 100) == ctypes.c_size_t(-1).value


PAGES = [
    (dict(size=0), "SHAPE"), (dict(size=-16), "SHAPE"), (dict(size=8), "SHAPE"), (dict(size=24), "SHAPE"),
    (dict(n_pages=-1), "SHAPE"), (dict(max_pages=-1), "SHAPE"), (dict(reserved=1), "SHAPE"),
    (dict(max_pages=1 << 27), "SHAPE"), (dict(stride=8 * 16 * 128 - 8), "SHAPE"), (dict(stride=1 << 41), "SHAPE"),
    (dict(stride=1 << 40, n_pages=1 << 21), "SHAPE"), (dict(size=(1 << 30) + 16, stride=1 << 40, max_pages=1), "SHAPE"),
    (dict(stride=8 * 16 * 128 + 4), "ALIGN"), (dict(k=None), "NULL"), (dict(v=None), "NULL"), (dict(table=None), "NULL"),
    (dict(k=MIS), "ALIGN"), (dict(v=MIS), "ALIGN"), (dict(table=A + 2), "ALIGN"),
]


@pytest.mark.parametrize("kw,code", PAGES)
def test_pages(lib, kw, code):
    want = getattr(kvr, "KVR_ERR_" + code)
    most = min(80, max(0, kw.get("max_pages", 5)) * 16)
    assert append(lib, g=pages(**kw)) == want and decode(lib, g=pages(**kw), most=most) == want


def test_pages_missing(lib):
    assert append(lib, g=None) == kvr.KVR_ERR_NULL and decode(lib, g=None) == kvr.KVR_ERR_NULL


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), "SHAPE"), (dict(n_new=-1), "SHAPE"), (dict(most=-1), "SHAPE"), (dict(most=(1 << 30) + 1), "SHAPE"),
    (dict(n=1 << 24), "SHAPE"), (dict(most=81), "CAPACITY"), (dict(q=None), "NULL"), (dict(q=rows(32, data=None)), "NULL"), (dict(q=rows(32, head=-128)), "SHAPE"), (dict(out=None), "NULL"),
    (dict(ln=None), "NULL"), (dict(q=rows(32, data=MIS)), "ALIGN"), (dict(q=rows(32, token=4100)), "ALIGN"), (dict(out=MIS), "ALIGN"), (dict(ws=MIS), "ALIGN"), (dict(ln=A + 2), "ALIGN"),
])
def test_decode_refusals(lib, kw, code):
    assert decode(lib, **kw) == getattr(kvr, "KVR_ERR_" + code)


def test_decode_workspace(lib):
    d = desc()
    need = kvr.kvr_workspace_bytes_paged(d, 4, 65536)
    assert need > 0
    assert decode(lib, g=pages(**LONG), most=65536, ws=None) == kvr.KVR_ERR_WORKSPACE
    assert decode(lib, g=pages(**LONG), most=65536, wsb=need - 1) == kvr.KVR_ERR_WORKSPACE
    for n in (1, 3, 64, 500):
        sizes = [kvr.kvr_workspace_bytes_paged(d, n, m) for m in (0, 1, 128, 600, 3774, 32768, 1 << 20)]
        assert sizes == sorted(sizes) and sizes[-1] > 0
    assert kvr.kvr_workspace_bytes_paged(d, 0, 100) == 0
    for f in (lambda: kvr.kvr_workspace_bytes_paged(d, -1, 1), lambda: kvr.kvr_workspace_bytes_paged(d, 1, -1),
              lambda: kvr.workspace_for_paged(desc(head_dim=7), 1, 1), lambda: kvr.kvr_workspace_bytes_paged(d, 1 << 20, 1 << 30)):
        with pytest.raises(ValueError):
            f()


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), "SHAPE"), (dict(n=1 << 24), "SHAPE"), (dict(T=-1), "SHAPE"), (dict(T=1 << 31), "SHAPE"), (dict(cu=None), "SHAPE"), (dict(eps=-1.0), "SHAPE"),
    (dict(eps=float("nan")), "SHAPE"), (dict(eps=float("inf")), "SHAPE"),
    (dict(k=None), "NULL"), (dict(v=None), "NULL"), (dict(ln=None), "NULL"), (dict(q=None), "NULL"), (dict(qo=None), "NULL"),
    (dict(q=None, qo=None), "NULL"),      # norm weights without queries
    (dict(k=rows(data=None)), "NULL"), (dict(k=rows(data=MIS)), "ALIGN"), (dict(v=rows(token=-128)), "SHAPE"),
    (dict(v=rows(token=1028)), "ALIGN"), (dict(k=rows(head=132)), "ALIGN"), (dict(k=rows(head=-128)), "SHAPE"),
    (dict(k=rows(token=1 << 41)), "SHAPE"), (dict(q=rows(32, data=MIS)), "ALIGN"), (dict(qo=rows(32, data=None)), "NULL"),
    (dict(qo=rows(32, token=128)), "SHAPE"), (dict(qo=rows(32, head=64)), "SHAPE"), (dict(qo=rows(32, token=0)), "SHAPE"),
    (dict(qn=MIS), "ALIGN"), (dict(kn=MIS), "ALIGN"), (dict(cu=A + 1), "ALIGN"), (dict(ln=A + 2), "ALIGN"), (dict(pos=A + 2), "ALIGN"),
])
def test_append_refusals(lib, kw, code):
    assert append(lib, **kw) == getattr(kvr, "KVR_ERR_" + code)


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), "SHAPE"), (dict(n=1 << 31), "SHAPE"), (dict(eps=-1.0), "SHAPE"), (dict(q=None), "NULL"), (dict(qo=None), "NULL"),
    (dict(k=None), "NULL"), (dict(ko=None), "NULL"), (dict(q=None, qo=None), "NULL"), (dict(k=None, ko=None), "NULL"),
    (dict(q=None, qo=None, k=None, ko=None, qn=None, kn=None), "NULL"),
    (dict(ko=rows(token=512)), "SHAPE"), (dict(ko=rows(token=128, head=256)), "SHAPE"), (dict(q=rows(32, data=MIS)), "ALIGN"),
    (dict(ko=rows(head=1 << 41)), "SHAPE"), (dict(kn=MIS), "ALIGN"), (dict(pos=A + 1), "ALIGN"),
])
def test_norm_rope_refusals(lib, kw, code):
    assert norm_rope(lib, **kw) == getattr(kvr, "KVR_ERR_" + code)


def test_tables(lib):
    table = lambda n, p=A: kvr.kvr_rope(p, n)
    assert append(lib, rope=table(79)) == kvr.KVR_ERR_POSITION                 # rows up to 80
    assert append(lib, rope=table(0), pos=A) == kvr.KVR_ERR_POSITION           # given positions: an entry at least
    assert append(lib, rope=table(80, None)) == kvr.KVR_ERR_NULL
    assert append(lib, rope=table(80, MIS)) == kvr.KVR_ERR_ALIGN
    assert norm_rope(lib, rope=table(13), pos0=10) == kvr.KVR_ERR_POSITION
    assert norm_rope(lib, rope=table(13), pos0=-1) == kvr.KVR_ERR_POSITION
    assert norm_rope(lib, rope=table(0), pos=A) == kvr.KVR_ERR_POSITION
    assert norm_rope(lib, rope=table(14, MIS), pos0=10) == kvr.KVR_ERR_ALIGN


def test_heads_that_the_kernels_do_not_count(lib):
    d = desc(n_q_heads=65536, n_kv_heads=1)
    wide = lambda: rows(65536)
    assert norm_rope(lib, d, q=wide(), qo=wide(), k=None, ko=None, kn=None) == kvr.KVR_ERR_SHAPE


def test_the_stride_of_a_single_token_or_head_is_not_used(lib):
    """Negative strides, which are a shape's error where they are used; what is checked behind them is not aligned."""
    d = desc(n_q_heads=4, n_kv_heads=1)
    one = lambda token=-3, head=-5: kvr.kvr_rows(A, token, head)
    key = lambda n, **kw: norm_rope(lib, d, n=n, q=None, qo=None, qn=None, kn=MIS, k=one(**kw), ko=one(**kw))
    assert decode(lib, d, n=1, q=one(head=128), out=MIS) == kvr.KVR_ERR_ALIGN
    assert decode(lib, d, n=2, q=one(head=128), out=MIS) == kvr.KVR_ERR_SHAPE
    assert key(1) == kvr.KVR_ERR_ALIGN and key(2, token=128) == kvr.KVR_ERR_ALIGN and key(2) == kvr.KVR_ERR_SHAPE


def test_no_work(lib):
    none = dict(q=None, qo=None, qn=None, kn=None)
    assert norm_rope(lib, n=0, k=None, ko=None, **none) == kvr.KVR_OK
    assert append(lib, n=0, k=None, v=None, ln=None, **none) == kvr.KVR_OK
    assert append(lib, T=0, k=None, v=None, ln=None, **none) == kvr.KVR_OK
    assert append(lib, g=pages(n_pages=0, k=None, v=None)) == kvr.KVR_OK          # no token has a place
    assert append(lib, g=pages(max_pages=0, table=None)) == kvr.KVR_OK
    assert decode(lib, n=0, q=None, out=None, ln=None, ws=None) == kvr.KVR_OK


def test_binding_checks_tensors(lib):
    """CPU tensors, wrong types of objects: ValueError, nothing called."""
    d = desc()
    x, p = torch.zeros((2, 32, 128), dtype=torch.bfloat16), torch.zeros((3, 8, 16, 128), dtype=torch.bfloat16)
    t = torch.zeros((2, 4), dtype=torch.int32)
    with pytest.raises(ValueError, match="on the GPU"):
        kvr.PagedCache(d, p, p, t)
    with pytest.raises(ValueError, match="on the GPU"):
        kvr.kvr_qk_norm_rope(d, x, x[:, :8])
    with pytest.raises(ValueError, match="torch tensor"):
        kvr.kvr_qk_norm_rope(d, None, None)
    with pytest.raises(ValueError, match="PagedCache"):
        kvr.kvr_paged_append(d, None, x[:, :8], x[:, :8], t[:, 0])
    with pytest.raises(ValueError, match="PagedCache"):
        kvr.kvr_paged_decode(d, (p, p), x, t[:, 0], x)
