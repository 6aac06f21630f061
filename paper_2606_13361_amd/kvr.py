"""Python binding of libkvr (include/kvr.h): argument marshalling only.

Every function has the name of the C entry point it calls.  Tensors are torch
tensors on the GPU (PyTorch provides device memory and streams); their
dtype, device, contiguity and shape are checked against the layer descriptor
before the call -- the consumer-side metadata check of the paper's Alg. 2 --
and a ValueError is raised on a mismatch.  A nonzero kvr_status raises
KvrError.  There is no fallback: without the built library every call fails.
"""
import ctypes
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libkvr.so")

KVR_OK, KVR_ERR_NULL, KVR_ERR_SHAPE, KVR_ERR_DTYPE = 0, 1, 2, 3
KVR_ERR_CAPACITY, KVR_ERR_WORKSPACE, KVR_ERR_ALIGN, KVR_ERR_DEVICE = 4, 5, 6, 7
KVR_ERR_MISMATCH, KVR_ERR_POSITION, KVR_ERR_TOO_LARGE = 8, 9, 10
KVR_NOALLOC_SCRATCH_BYTES = 16 << 20
KVR_ARTIFACT_HEADER_BYTES = 256
KVR_BF16, KVR_F32, KVR_F16 = 0, 1, 2

EXPORTS = ("kvr_prefill", "kvr_continue", "kvr_continue_append", "kvr_continue_noalloc", "kvr_continue_batched",
           "kvr_cache_append",
           "kvr_workspace_bytes", "kvr_strerror", "kvr_abi_version",
           "kvr_q8_bytes", "kvr_quantize_cache", "kvr_continue_q8",
           "kvr_artifact_bytes", "kvr_artifact_save", "kvr_artifact_load",
           "kvr_rope_table", "kvr_rope_apply", "kvr_prefill_rope", "kvr_continue_rope",
           "kvr_continue_batched_rope", "kvr_workspace_bytes_rope",
           "kvr_continue_shared", "kvr_workspace_bytes_shared", "kvr_cache_weigh", "kvr_workspace_bytes_weigh",
           "kvr_cache_evict", "kvr_workspace_bytes_evict",
           "kvr_qk_norm_rope", "kvr_paged_append", "kvr_paged_decode", "kvr_workspace_bytes_paged")

_TORCH_DTYPE = {KVR_BF16: torch.bfloat16, KVR_F32: torch.float32, KVR_F16: torch.float16}


class kvr_desc(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("scale", ctypes.c_float), ("reserved", ctypes.c_int32),
                ("capacity", ctypes.c_int64)]


class kvr_rope(ctypes.Structure):
    _fields_ = [("cos_sin", ctypes.c_void_p), ("n_pos", ctypes.c_int64)]


class kvr_pages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_stride", ctypes.c_int64),
                ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32), ("table", ctypes.c_void_p),
                ("max_pages", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class kvr_rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64)]


class KvrError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: %s (status %d)" % (where, strerror(status), status))


_lib = None


def load():
    """Load the in-tree libkvr.so; raise if it was not built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libkvr.so is not built (run __graft_entry__.build() or "
                           "python -m paper_2606_13361_amd.build)")
    lib = ctypes.CDLL(LIB_PATH)
    P, I64, SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    D = ctypes.POINTER(kvr_desc)
    lib.kvr_prefill.argtypes = [D, P, P, P, I64, P, P, P, P]
    lib.kvr_continue.argtypes = [D, P, P, P, P, P, I64, I64, P, P, SZ, P]
    lib.kvr_continue_append.argtypes = [D, P, P, P, P, P, I64, I64, P, P, SZ, P]
    lib.kvr_continue_noalloc.argtypes = [D, P, P, P, P, P, I64, I64, P, P]
    lib.kvr_continue_batched.argtypes = [D, P, P, P, ctypes.POINTER(ctypes.c_int32), ctypes.c_int32,
                                         P, P, I64, P, P, SZ, P]
    lib.kvr_cache_append.argtypes = [D, P, P, I64, P, P, I64, P]
    lib.kvr_workspace_bytes.argtypes = [D, I64, I64, ctypes.c_int32]
    lib.kvr_workspace_bytes.restype = SZ
    lib.kvr_q8_bytes.argtypes = [D]
    lib.kvr_q8_bytes.restype = SZ
    lib.kvr_quantize_cache.argtypes = [D, P, P, I64, P, P, P, P]
    lib.kvr_continue_q8.argtypes = [D, P, P, P, P, P, P, I64, I64, P, P, SZ, P]
    PP = ctypes.POINTER(ctypes.c_void_p)
    lib.kvr_artifact_bytes.argtypes = [D, ctypes.c_int32, I64]
    lib.kvr_artifact_bytes.restype = SZ
    lib.kvr_artifact_save.argtypes = [D, ctypes.c_char_p, ctypes.c_int32, I64, PP, PP, P, SZ, P]
    lib.kvr_artifact_load.argtypes = [D, ctypes.c_char_p, ctypes.c_int32, P, SZ, PP, PP,
                                      ctypes.POINTER(ctypes.c_int64), P]
    R = ctypes.POINTER(kvr_rope)
    lib.kvr_rope_table.argtypes = [ctypes.c_int32, ctypes.c_double, I64, P, P]
    lib.kvr_rope_apply.argtypes = [D, R, P, I64, ctypes.c_int32, I64, P, P]
    lib.kvr_prefill_rope.argtypes = [D, R, P, P, P, I64, P, P, P, P]
    lib.kvr_continue_rope.argtypes = [D, R, P, P, P, P, P, I64, I64, ctypes.c_int32, P, P, SZ, P]
    lib.kvr_continue_batched_rope.argtypes = [D, R, P, P, P, ctypes.POINTER(ctypes.c_int32), ctypes.c_int32,
                                              P, P, I64, P, P, SZ, P]
    lib.kvr_workspace_bytes_rope.argtypes = [D, I64, I64, ctypes.c_int32]
    lib.kvr_workspace_bytes_rope.restype = SZ
    I32 = ctypes.c_int32
    lib.kvr_continue_shared.argtypes = [D, R, P, P, P, I32, I32, P, P, I64, I64, P, P, I64, P, I32, P, P, SZ, P]
    lib.kvr_workspace_bytes_shared.argtypes = [D, I64, I32, I32, I64]
    lib.kvr_workspace_bytes_shared.restype = SZ
    lib.kvr_cache_weigh.argtypes = [D, P, P, P, I64, I64, P, P, SZ, P]
    lib.kvr_workspace_bytes_weigh.argtypes = [D, I64, I64]
    lib.kvr_workspace_bytes_weigh.restype = SZ
    lib.kvr_cache_evict.argtypes = [D, P, P, I64, P, I64, I64, I64, P, P, I64, P, P, P, SZ, P]
    lib.kvr_workspace_bytes_evict.argtypes = [D, I64]
    lib.kvr_workspace_bytes_evict.restype = SZ
    G, T = ctypes.POINTER(kvr_pages), ctypes.POINTER(kvr_rows)
    lib.kvr_qk_norm_rope.argtypes = [D, R, T, T, P, P, ctypes.c_float, I64, P, I64, T, T, P]
    lib.kvr_paged_append.argtypes = [D, G, R, T, T, T, P, P, ctypes.c_float, I32, I64, P, P, P, T, P]
    lib.kvr_paged_decode.argtypes = [D, G, T, I32, P, I32, I64, P, P, SZ, P]
    lib.kvr_workspace_bytes_paged.argtypes = [D, I32, I64]
    lib.kvr_workspace_bytes_paged.restype = SZ
    lib.kvr_strerror.argtypes = [ctypes.c_int]
    lib.kvr_strerror.restype = ctypes.c_char_p
    lib.kvr_abi_version.argtypes = []
    for f in (lib.kvr_prefill, lib.kvr_continue, lib.kvr_continue_append, lib.kvr_continue_noalloc,
              lib.kvr_continue_batched,
              lib.kvr_cache_append,
              lib.kvr_abi_version, lib.kvr_quantize_cache, lib.kvr_continue_q8, lib.kvr_artifact_save,
              lib.kvr_artifact_load, lib.kvr_rope_table, lib.kvr_rope_apply, lib.kvr_prefill_rope,
              lib.kvr_continue_rope, lib.kvr_continue_batched_rope, lib.kvr_continue_shared,
              lib.kvr_cache_weigh, lib.kvr_cache_evict, lib.kvr_qk_norm_rope, lib.kvr_paged_append,
              lib.kvr_paged_decode):
        f.restype = ctypes.c_int
    _lib = lib
    return lib


def strerror(status):
    return load().kvr_strerror(int(status)).decode()


def kvr_abi_version():
    return load().kvr_abi_version()


def make_desc(n_q_heads, n_kv_heads, head_dim, dtype, capacity, scale=0.0):
    """dtype: torch.bfloat16 / torch.float16 / torch.float32 or KVR_BF16 / KVR_F16 / KVR_F32."""
    if isinstance(dtype, torch.dtype):
        dtype = {torch.bfloat16: KVR_BF16, torch.float16: KVR_F16, torch.float32: KVR_F32}.get(dtype, -1)
    return kvr_desc(int(n_q_heads), int(n_kv_heads), int(head_dim), int(dtype), float(scale), 0,
                    int(capacity))


def _stream(stream):
    if stream is None:
        # the handle of torch.cuda.current_stream() without building a Stream object
        # (2.8 us of a small call's 11 us on the host; 0.3 this way)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _check(t, name, desc, shape):
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s must be a torch tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be on the GPU" % name)
    want = _TORCH_DTYPE.get(desc.dtype)
    if t.dtype != want:
        raise ValueError("%s has dtype %s, the layer descriptor says %s" % (name, t.dtype, want))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if t.shape != shape and tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    return t.data_ptr()


def _cache_ptrs(desc, kcache, vcache, required):
    if kcache is None and vcache is None and not required:
        return None, None
    shape = (desc.n_kv_heads, desc.capacity, desc.head_dim)
    return _check(kcache, "kcache", desc, shape), _check(vcache, "vcache", desc, shape)


def _raise(st, where):
    if st != KVR_OK:
        raise KvrError(st, where)


def kvr_workspace_bytes(desc, L_prefix, total_S, n=1):
    return load().kvr_workspace_bytes(ctypes.byref(desc), int(L_prefix), int(total_S), int(n))


def kvr_prefill(desc, Q, K, V, L, out, kcache, vcache, stream=None):
    Hq, Hkv, d = desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    q = _check(Q, "Q", desc, (L, Hq, d))
    k = _check(K, "K", desc, (L, Hkv, d))
    v = _check(V, "V", desc, (L, Hkv, d))
    o = _check(out, "out", desc, (L, Hq, d))
    kc, vc = _cache_ptrs(desc, kcache, vcache, True)
    _raise(load().kvr_prefill(ctypes.byref(desc), q, k, v, int(L), o, kc, vc, _stream(stream)),
           "kvr_prefill")


def kvr_continue(desc, Qs, Ks, Vs, kcache, vcache, L_prefix, S, out, ws=None, stream=None):
    Hq, Hkv, d = desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    q = _check(Qs, "Qs", desc, (S, Hq, d))
    k = _check(Ks, "Ks", desc, (S, Hkv, d))
    v = _check(Vs, "Vs", desc, (S, Hkv, d))
    o = _check(out, "out", desc, (S, Hq, d))
    kc, vc = _cache_ptrs(desc, kcache, vcache, L_prefix > 0)
    wp, wn = _workspace(ws)
    _raise(load().kvr_continue(ctypes.byref(desc), q, k, v, kc, vc, int(L_prefix), int(S), o, wp, wn,
                               _stream(stream)), "kvr_continue")


def kvr_continue_noalloc(desc, Qs, Ks, Vs, kcache, vcache, L_prefix, S, out, stream=None):
    """kvr_continue with its split partials in the library's fixed per-device buffer."""
    Hq, Hkv, d = desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    q = _check(Qs, "Qs", desc, (S, Hq, d))
    k = _check(Ks, "Ks", desc, (S, Hkv, d))
    v = _check(Vs, "Vs", desc, (S, Hkv, d))
    o = _check(out, "out", desc, (S, Hq, d))
    kc, vc = _cache_ptrs(desc, kcache, vcache, L_prefix > 0)
    _raise(load().kvr_continue_noalloc(ctypes.byref(desc), q, k, v, kc, vc, int(L_prefix), int(S), o,
                                       _stream(stream)), "kvr_continue_noalloc")


def kvr_continue_append(desc, Qs, Ks, Vs, kcache, vcache, L_prefix, S, out, ws=None, stream=None):
    """kvr_continue plus the cache update of the S tokens at rows L_prefix.. ."""
    Hq, Hkv, d = desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    q = _check(Qs, "Qs", desc, (S, Hq, d))
    k = _check(Ks, "Ks", desc, (S, Hkv, d))
    v = _check(Vs, "Vs", desc, (S, Hkv, d))
    o = _check(out, "out", desc, (S, Hq, d))
    kc, vc = _cache_ptrs(desc, kcache, vcache, True)
    wp, wn = _workspace(ws)
    _raise(load().kvr_continue_append(ctypes.byref(desc), q, k, v, kc, vc, int(L_prefix), int(S), o, wp, wn,
                                      _stream(stream)), "kvr_continue_append")


def kvr_continue_batched(desc, Qs, Ks, Vs, cu_seqlens, kcache, vcache, L_prefix, out, ws=None,
                         stream=None):
    """cu_seqlens: host sequence of n+1 ints (a list or a CPU tensor).  ws: the
    workspace of workspace_for(desc, L_prefix, cu_seqlens[-1], n) (None when
    that is None: the call's plan splits no row tile over the keys)."""
    Hq, Hkv, d = desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    cu = [int(x) for x in (cu_seqlens.tolist() if isinstance(cu_seqlens, torch.Tensor) else cu_seqlens)]
    n = len(cu) - 1
    if n < 0:
        raise ValueError("cu_seqlens needs at least one entry")
    total = cu[-1]
    q = _check(Qs, "Qs", desc, (total, Hq, d))
    k = _check(Ks, "Ks", desc, (total, Hkv, d))
    v = _check(Vs, "Vs", desc, (total, Hkv, d))
    o = _check(out, "out", desc, (total, Hq, d))
    kc, vc = _cache_ptrs(desc, kcache, vcache, L_prefix > 0)
    arr = (ctypes.c_int32 * len(cu))(*cu)
    wp, wn = _workspace(ws)
    _raise(load().kvr_continue_batched(ctypes.byref(desc), q, k, v, arr, n, kc, vc, int(L_prefix), o,
                                       wp, wn, _stream(stream)), "kvr_continue_batched")


def kvr_cache_append(desc, Ks, Vs, S, kcache, vcache, L_cur, stream=None):
    Hkv, d = desc.n_kv_heads, desc.head_dim
    k = _check(Ks, "Ks", desc, (S, Hkv, d))
    v = _check(Vs, "Vs", desc, (S, Hkv, d))
    kc, vc = _cache_ptrs(desc, kcache, vcache, True)
    _raise(load().kvr_cache_append(ctypes.byref(desc), k, v, int(S), kc, vc, int(L_cur), _stream(stream)),
           "kvr_cache_append")


_SIZE_ERR = ctypes.c_size_t(-1).value   # a kvr_*_bytes call's answer to invalid arguments


def kvr_q8_bytes(desc):
    """Bytes of each int8 artifact tensor (kq, vq) for this descriptor."""
    nb = load().kvr_q8_bytes(ctypes.byref(desc))
    if nb == _SIZE_ERR:
        raise ValueError("invalid layer descriptor")
    return nb


def q8_artifact(desc, device="cuda"):
    """Allocate (with torch) an int8 artifact: (kq, vq, scales)."""
    nb = kvr_q8_bytes(desc)
    return (torch.empty(nb, dtype=torch.int8, device=device), torch.empty(nb, dtype=torch.int8, device=device),
            torch.empty(2, dtype=torch.float32, device=device))


def _check_q8(desc, kq, vq, scales):
    nb = kvr_q8_bytes(desc)
    for t, name in ((kq, "kq"), (vq, "vq")):
        if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != torch.int8 or not t.is_contiguous():
            raise ValueError("%s must be a contiguous int8 GPU tensor" % name)
        if t.numel() != nb:
            raise ValueError("%s holds %d bytes, the descriptor needs %d" % (name, t.numel(), nb))
    if (not isinstance(scales, torch.Tensor) or not scales.is_cuda or scales.dtype != torch.float32
            or scales.numel() != 2 or not scales.is_contiguous()):
        raise ValueError("scales must be a contiguous float32 GPU tensor of 2 values")
    return kq.data_ptr(), vq.data_ptr(), scales.data_ptr()


def kvr_quantize_cache(desc, kcache, vcache, L, kq, vq, scales, stream=None):
    kc, vc = _cache_ptrs(desc, kcache, vcache, True)
    a, b, sc = _check_q8(desc, kq, vq, scales)
    _raise(load().kvr_quantize_cache(ctypes.byref(desc), kc, vc, int(L), a, b, sc, _stream(stream)),
           "kvr_quantize_cache")


def kvr_continue_q8(desc, Qs, Ks, Vs, kq, vq, scales, L_prefix, S, out, ws=None, stream=None):
    Hq, Hkv, d = desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    q = _check(Qs, "Qs", desc, (S, Hq, d))
    k = _check(Ks, "Ks", desc, (S, Hkv, d))
    v = _check(Vs, "Vs", desc, (S, Hkv, d))
    o = _check(out, "out", desc, (S, Hq, d))
    a, b, sc = _check_q8(desc, kq, vq, scales)
    wp, wn = _workspace(ws)
    _raise(load().kvr_continue_q8(ctypes.byref(desc), q, k, v, a, b, sc, int(L_prefix), int(S), o, wp, wn,
                                  _stream(stream)), "kvr_continue_q8")


def kvr_artifact_bytes(desc, n_layers, L):
    nb = load().kvr_artifact_bytes(ctypes.byref(desc), int(n_layers), int(L))
    if nb == ctypes.c_size_t(-1).value:
        raise ValueError("invalid descriptor, layer count or length")
    return nb


def _host_buffer(host, name):
    if not isinstance(host, torch.Tensor) or host.is_cuda or host.dtype != torch.uint8 or not host.is_contiguous():
        raise ValueError("%s must be a contiguous uint8 CPU tensor (pinned for asynchronous copies)" % name)
    return host.data_ptr(), host.numel()


def _layer_ptrs(desc, caches, name):
    arr = (ctypes.c_void_p * len(caches))()
    shape = (desc.n_kv_heads, desc.capacity, desc.head_dim)
    for i, c in enumerate(caches):
        arr[i] = _check(c, "%s[%d]" % (name, i), desc, shape)
    return arr


def kvr_artifact_save(desc, model_id, kcaches, vcaches, L, host, stream=None):
    """Serialize rows [0, L) of every layer's caches into the host tensor (Alg. 1)."""
    if len(kcaches) != len(vcaches) or not kcaches:
        raise ValueError("one K and one V cache per layer")
    hp, hn = _host_buffer(host, "host")
    _raise(load().kvr_artifact_save(ctypes.byref(desc), model_id.encode(), len(kcaches), int(L),
                                    _layer_ptrs(desc, kcaches, "kcaches"), _layer_ptrs(desc, vcaches, "vcaches"),
                                    hp, hn, _stream(stream)), "kvr_artifact_save")


def kvr_artifact_load(desc, model_id, host, kcaches, vcaches, stream=None):
    """Check the artifact's metadata against (model_id, desc, layer count) and load it
    into the caches (Alg. 2); returns L, where the continuation starts."""
    if len(kcaches) != len(vcaches) or not kcaches:
        raise ValueError("one K and one V cache per layer")
    hp, hn = _host_buffer(host, "host")
    L = ctypes.c_int64(-1)
    _raise(load().kvr_artifact_load(ctypes.byref(desc), model_id.encode(), len(kcaches), hp, hn,
                                    _layer_ptrs(desc, kcaches, "kcaches"), _layer_ptrs(desc, vcaches, "vcaches"),
                                    ctypes.byref(L), _stream(stream)), "kvr_artifact_load")
    return L.value


def _workspace(ws):
    if ws is None:
        return None, 0
    if not isinstance(ws, torch.Tensor) or not ws.is_cuda or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous GPU tensor")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def workspace_for(desc, L_prefix, total_S, n=1, device="cuda"):
    """Allocate (with torch) the workspace a continuation needs, or None."""
    nb = kvr_workspace_bytes(desc, L_prefix, total_S, n)
    if nb == ctypes.c_size_t(-1).value:
        raise ValueError("invalid layer descriptor")
    if nb == 0:
        return None
    return torch.empty(nb, dtype=torch.uint8, device=device)


# ---------------------------------------------------------------- RoPE
QWEN3_ROPE_BASE = 1.0e6


class RopeTable:
    """A device cos/sin table (float [n_pos][head_dim/2][2], torch-allocated)
    filled by kvr_rope_table; pass it to the *_rope entry points."""

    def __init__(self, head_dim, n_pos, base=QWEN3_ROPE_BASE, device="cuda", stream=None):
        self.head_dim, self.n_pos, self.base = int(head_dim), int(n_pos), float(base)
        self.cos_sin = torch.empty((max(self.n_pos, 1), self.head_dim // 2, 2), dtype=torch.float32, device=device)
        kvr_rope_table(self.head_dim, self.base, self.n_pos, self.cos_sin, stream)

    def c(self):
        return kvr_rope(self.cos_sin.data_ptr(), self.n_pos)


def kvr_rope_table(head_dim, base, n_pos, cos_sin, stream=None):
    if (not isinstance(cos_sin, torch.Tensor) or not cos_sin.is_cuda or cos_sin.dtype != torch.float32
            or not cos_sin.is_contiguous() or cos_sin.numel() < int(n_pos) * int(head_dim)):
        raise ValueError("cos_sin must be a contiguous float32 GPU tensor of n_pos * head_dim values")
    _raise(load().kvr_rope_table(int(head_dim), float(base), int(n_pos), cos_sin.data_ptr(), _stream(stream)),
           "kvr_rope_table")


def _rope(rope, desc):
    if not isinstance(rope, RopeTable):
        raise ValueError("rope must be a RopeTable")
    if rope.head_dim != desc.head_dim:
        raise ValueError("RoPE table head_dim %d, descriptor %d" % (rope.head_dim, desc.head_dim))
    return ctypes.byref(rope.c())


def kvr_rope_apply(desc, rope, x, pos0, y=None, stream=None):
    """Rotate rows x [n_tok, n_heads, head_dim] at positions pos0.. into y (default: in place)."""
    if x.dim() != 3:
        raise ValueError("x must be [n_tok, n_heads, head_dim]")
    n_tok, n_heads = x.shape[0], x.shape[1]
    y = x if y is None else y
    xp = _check(x, "x", desc, (n_tok, n_heads, desc.head_dim))
    yp = _check(y, "y", desc, (n_tok, n_heads, desc.head_dim))
    _raise(load().kvr_rope_apply(ctypes.byref(desc), _rope(rope, desc), xp, int(n_tok), int(n_heads), int(pos0),
                                 yp, _stream(stream)), "kvr_rope_apply")
    return y


def kvr_prefill_rope(desc, rope, Q, K, V, L, out, kcache, vcache, stream=None):
    Hq, Hkv, d = desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    q = _check(Q, "Q", desc, (L, Hq, d))
    k = _check(K, "K", desc, (L, Hkv, d))
    v = _check(V, "V", desc, (L, Hkv, d))
    o = _check(out, "out", desc, (L, Hq, d))
    kc, vc = _cache_ptrs(desc, kcache, vcache, True)
    _raise(load().kvr_prefill_rope(ctypes.byref(desc), _rope(rope, desc), q, k, v, int(L), o, kc, vc,
                                   _stream(stream)), "kvr_prefill_rope")


def kvr_workspace_bytes_rope(desc, L_prefix, total_S, n=1):
    return load().kvr_workspace_bytes_rope(ctypes.byref(desc), int(L_prefix), int(total_S), int(n))


def workspace_for_rope(desc, L_prefix, total_S, n=1, device="cuda"):
    """Allocate (with torch) the workspace of a RoPE continuation."""
    nb = kvr_workspace_bytes_rope(desc, L_prefix, total_S, n)
    if nb == ctypes.c_size_t(-1).value:
        raise ValueError("invalid layer descriptor")
    return torch.empty(max(nb, 1), dtype=torch.uint8, device=device)


def kvr_continue_rope(desc, rope, Qs, Ks, Vs, kcache, vcache, L_prefix, S, out, ws, append=False, stream=None):
    Hq, Hkv, d = desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    q = _check(Qs, "Qs", desc, (S, Hq, d))
    k = _check(Ks, "Ks", desc, (S, Hkv, d))
    v = _check(Vs, "Vs", desc, (S, Hkv, d))
    o = _check(out, "out", desc, (S, Hq, d))
    kc, vc = _cache_ptrs(desc, kcache, vcache, L_prefix > 0 or append)
    wp, wn = _workspace(ws)
    _raise(load().kvr_continue_rope(ctypes.byref(desc), _rope(rope, desc), q, k, v, kc, vc, int(L_prefix), int(S),
                                    1 if append else 0, o, wp, wn, _stream(stream)), "kvr_continue_rope")


def kvr_continue_batched_rope(desc, rope, Qs, Ks, Vs, cu_seqlens, kcache, vcache, L_prefix, out, ws,
                              stream=None):
    Hq, Hkv, d = desc.n_q_heads, desc.n_kv_heads, desc.head_dim
    cu = [int(x) for x in (cu_seqlens.tolist() if isinstance(cu_seqlens, torch.Tensor) else cu_seqlens)]
    n = len(cu) - 1
    if n < 0:
        raise ValueError("cu_seqlens needs at least one entry")
    total = cu[-1]
    q = _check(Qs, "Qs", desc, (total, Hq, d))
    k = _check(Ks, "Ks", desc, (total, Hkv, d))
    v = _check(Vs, "Vs", desc, (total, Hkv, d))
    o = _check(out, "out", desc, (total, Hq, d))
    kc, vc = _cache_ptrs(desc, kcache, vcache, L_prefix > 0)
    arr = (ctypes.c_int32 * len(cu))(*cu)
    wp, wn = _workspace(ws)
    _raise(load().kvr_continue_batched_rope(ctypes.byref(desc), _rope(rope, desc), q, k, v, arr, n, kc, vc,
                                            int(L_prefix), o, wp, wn, _stream(stream)),
           "kvr_continue_batched_rope")


# ---------------------------------------------------------------- many readers, later turns
def _device(t, name):
    """The GPU of a call's first tensor; the others have to be there (_at)."""
    if not isinstance(t, torch.Tensor):
        raise ValueError("%s must be a torch tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be on the GPU" % name)
    return t.get_device()


def _at(t, name, dtype, shape, dev):
    """Address of a contiguous tensor of this type and shape (a tuple) on GPU dev.  One
    expression where all is well: a small call is bound by its checks on the host."""
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.get_device() == dev and t.is_contiguous()
            and t.shape == shape):
        return t.data_ptr()
    _device(t, name)
    if t.dtype != dtype or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor, not %s" % (name, dtype, t.dtype))
    if t.get_device() != dev:
        raise ValueError("%s is on GPU %d, other tensors of the call on GPU %d" % (name, t.get_device(), dev))
    raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), shape))


def _pair(a, a_name, b, b_name, dtype, shape, dev):
    """_at of two tensors of one type and shape, a seventh of the time less."""
    try:
        if (a.dtype is dtype and b.dtype is dtype and a.get_device() == dev and b.get_device() == dev
                and a.is_contiguous() and b.is_contiguous() and a.shape == shape and b.shape == shape):
            return a.data_ptr(), b.data_ptr()
    except AttributeError:      # one is no tensor
        pass
    return _at(a, a_name, dtype, shape, dev), _at(b, b_name, dtype, shape, dev)


def _scratch(ws, dev):
    if ws is None:
        return None, 0
    if isinstance(ws, torch.Tensor) and ws.is_cuda and ws.get_device() != dev:
        raise ValueError("ws is on GPU %d, other tensors of the call on GPU %d" % (ws.get_device(), dev))
    return _workspace(ws)


def _launch(call, where, stream, dev):
    """call(stream handle) with GPU dev current."""
    if isinstance(stream, torch.cuda.Stream) and stream.device.index != dev:
        raise ValueError("%s: tensors on GPU %d, the stream is of %s" % (where, dev, stream.device))
    if dev == torch._C._cuda_getDevice():
        _raise(call(torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream)), where)
    else:
        with torch.cuda.device(dev):
            _raise(call(_stream(stream)), where)


def _bytes(nb):
    if nb == _SIZE_ERR:
        raise ValueError("invalid layer descriptor or sizes")
    return nb


def kvr_workspace_bytes_shared(desc, L_prefix, n, S, tail_capacity):
    return _bytes(load().kvr_workspace_bytes_shared(ctypes.byref(desc), int(L_prefix), int(n), int(S),
                                                    int(tail_capacity)))


def workspace_for_shared(desc, L_prefix, n, S, tail_capacity, device="cuda"):
    """Allocate (with torch) the workspace of kvr_continue_shared."""
    return torch.empty(kvr_workspace_bytes_shared(desc, L_prefix, n, S, tail_capacity), dtype=torch.uint8, device=device)


def kvr_continue_shared(desc, Qs, Ks, Vs, kcache, vcache, L_prefix, ktail, vtail, tail_len, out, ws, rope=None,
                        pos0=None, append=False, stream=None):
    """One step of n readers of a shared prefix, each with cached rows of its own.

    Qs, out [n, S, n_q_heads, head_dim]; Ks, Vs [n, S, n_kv_heads, head_dim];
    ktail, vtail [n, n_kv_heads, tail_capacity, head_dim] (None: the readers have no
    rows); tail_len: int32 GPU tensor [n].  rope: a RopeTable that rotates the rows
    at pos0 + tail_len[r] + i (pos0: L_prefix by default)."""
    Hq, Hkv, d, dt = desc.n_q_heads, desc.n_kv_heads, desc.head_dim, _TORCH_DTYPE.get(desc.dtype)
    dev = _device(Qs, "Qs")
    if Qs.dim() != 4:
        raise ValueError("Qs must be a tensor [n, S, n_q_heads, head_dim]")
    n, S = Qs.shape[:2]
    q, o = _pair(Qs, "Qs", out, "out", dt, (n, S, Hq, d), dev)
    k, v = _pair(Ks, "Ks", Vs, "Vs", dt, (n, S, Hkv, d), dev)
    kc = vc = kt = vt = rp = None
    if L_prefix > 0 or kcache is not None or vcache is not None:
        kc, vc = _pair(kcache, "kcache", vcache, "vcache", dt, (Hkv, desc.capacity, d), dev)
    cap = 0
    if ktail is not None or vtail is not None:
        if not isinstance(ktail, torch.Tensor) or ktail.dim() != 4:
            raise ValueError("ktail must be a tensor [n, n_kv_heads, tail_capacity, head_dim]")
        cap = ktail.shape[2]
        kt, vt = _pair(ktail, "ktail", vtail, "vtail", dt, (n, Hkv, cap, d), dev)
    ln = _at(tail_len, "tail_len", torch.int32, (n,), dev)
    wp, wn = _scratch(ws, dev)
    if rope is not None:
        rp = _rope(rope, desc)
        if rope.cos_sin.get_device() != dev:
            raise ValueError("rope is on GPU %d, other tensors of the call on GPU %d" % (rope.cos_sin.get_device(), dev))
    at = int(L_prefix if pos0 is None else pos0)
    _launch(lambda s: load().kvr_continue_shared(ctypes.byref(desc), rp, q, k, v, n, S, kc, vc, int(L_prefix), at, kt,
                                                 vt, cap, ln, 1 if append else 0, o, wp, wn, s),
            "kvr_continue_shared", stream, dev)


def kvr_workspace_bytes_weigh(desc, L_prefix, S):
    return _bytes(load().kvr_workspace_bytes_weigh(ctypes.byref(desc), int(L_prefix), int(S)))


def workspace_for_weigh(desc, L_prefix, S, device="cuda"):
    """Allocate (with torch) the workspace of kvr_cache_weigh."""
    return torch.empty(kvr_workspace_bytes_weigh(desc, L_prefix, S), dtype=torch.uint8, device=device)


def kvr_cache_weigh(desc, Qs, Ks, kcache, L_prefix, S, weight, ws, stream=None):
    """Add to weight [n_kv_heads, capacity] (float32) the attention weight that each row
    receives from the S tokens at positions L_prefix.. ."""
    Hq, Hkv, d, dt = desc.n_q_heads, desc.n_kv_heads, desc.head_dim, _TORCH_DTYPE.get(desc.dtype)
    dev = _device(Qs, "Qs")
    q = _at(Qs, "Qs", dt, (S, Hq, d), dev)
    k = _at(Ks, "Ks", dt, (S, Hkv, d), dev)
    kc = _at(kcache, "kcache", dt, (Hkv, desc.capacity, d), dev) if L_prefix > 0 or kcache is not None else None
    w = _at(weight, "weight", torch.float32, (Hkv, desc.capacity), dev)
    wp, wn = _scratch(ws, dev)
    _launch(lambda s: load().kvr_cache_weigh(ctypes.byref(desc), q, k, kc, int(L_prefix), int(S), w, wp, wn, s),
            "kvr_cache_weigh", stream, dev)


def kvr_workspace_bytes_evict(desc, L):
    return _bytes(load().kvr_workspace_bytes_evict(ctypes.byref(desc), int(L)))


def workspace_for_evict(desc, L, device="cuda"):
    """Allocate (with torch) the workspace of kvr_cache_evict."""
    return torch.empty(kvr_workspace_bytes_evict(desc, L), dtype=torch.uint8, device=device)


def kvr_cache_evict(desc, kcache, vcache, L, weight, n_keep, kout, vout, n_first=0, n_last=0, weight_out=None,
                    index=None, ws=None, stream=None):
    """Copy the n_keep rows of [0, L) with the most weight (the first n_first and the last
    n_last always) into kout, vout [n_kv_heads, capacity_out, head_dim]; weight_out
    [n_kv_heads, capacity_out] and index (int32 [n_kv_heads, n_keep]) are optional."""
    Hkv, d, dt = desc.n_kv_heads, desc.head_dim, _TORCH_DTYPE.get(desc.dtype)
    dev = _device(kcache, "kcache")
    kc, vc = _pair(kcache, "kcache", vcache, "vcache", dt, (Hkv, desc.capacity, d), dev)
    w = _at(weight, "weight", torch.float32, (Hkv, desc.capacity), dev)
    if not isinstance(kout, torch.Tensor) or kout.dim() != 3:
        raise ValueError("kout must be a tensor [n_kv_heads, capacity_out, head_dim]")
    cap = kout.shape[1]
    ko, vo = _pair(kout, "kout", vout, "vout", dt, (Hkv, cap, d), dev)
    wo = None if weight_out is None else _at(weight_out, "weight_out", torch.float32, (Hkv, cap), dev)
    ix = None if index is None else _at(index, "index", torch.int32, (Hkv, n_keep), dev)
    wp, wn = _scratch(ws, dev)
    _launch(lambda s: load().kvr_cache_evict(ctypes.byref(desc), kc, vc, int(L), w, int(n_first), int(n_last),
                                             int(n_keep), ko, vo, cap, wo, ix, wp, wn, s),
            "kvr_cache_evict", stream, dev)


# ---------------------------------------------------------------- paged caches
def _fits(x, name, bits=32):
    """x as an integer of the C call's type: ctypes would drop what is above it"""
    x = int(x)
    if not -(1 << (bits - 1)) <= x < 1 << (bits - 1):
        raise ValueError("%s is %d, beyond %d bits" % (name, x, bits))
    return x


class PagedCache:
    """Sequences in the pages of a pool: k, v [n_pages, n_kv_heads, page_size, head_dim] and a
    page table, int32 [n, max_pages], all on one GPU.  A page is contiguous; pages may be any
    distance apart (k = pool[:, 0], v = pool[:, 1] of [n_pages, 2, ...]).  page_size is a
    multiple of 16.  Entries of the table that are no page of the pool are skipped; they may
    change between calls, the tensors may not."""

    def __init__(self, desc, k, v, table):
        dev, dt = _device(k, "k"), _TORCH_DTYPE.get(desc.dtype)
        if k.dim() != 4:
            raise ValueError("k must be a tensor [n_pages, n_kv_heads, page_size, head_dim]")
        n_pages, ps = k.shape[0], k.shape[2]
        page = (desc.n_kv_heads, ps, desc.head_dim)
        inner = (ps * desc.head_dim, desc.head_dim, 1)
        for t, name in ((k, "k"), (v, "v")):
            _device(t, name)
            if t.dtype != dt or t.get_device() != dev or t.shape != (n_pages,) + page:
                raise ValueError("%s must be a %s tensor %s on GPU %d" % (name, dt, (n_pages,) + page, dev))
            if any(a != b for a, b, m in zip(t.stride()[1:], inner, page) if m > 1):
                raise ValueError("the rows of a page of %s must be contiguous" % name)
        # (the stride of a pool of one page is not used, and may be anything)
        stride = [t.stride(0) if n_pages > 1 else desc.n_kv_heads * ps * desc.head_dim for t in (k, v)]
        if stride[0] != stride[1]:
            raise ValueError("pages of k are %d elements apart, those of v %d" % tuple(stride))
        if not isinstance(table, torch.Tensor) or table.dim() != 2:
            raise ValueError("table must be an int32 tensor [n, max_pages]")
        for size, what in ((n_pages, "pages"), (ps, "rows of a page"), (table.shape[0], "rows of table"), (table.shape[1], "columns of table")):
            _fits(size, "the number of " + what)
        tp = _at(table, "table", torch.int32, table.shape, dev)
        self.k, self.v, self.table = k, v, table
        self.device, self.n, self.reach = dev, table.shape[0], table.shape[1] * ps
        self.kv_heads, self.head_dim, self.dtype = desc.n_kv_heads, desc.head_dim, desc.dtype
        self._c = kvr_pages(k.data_ptr(), v.data_ptr(), stride[0], n_pages, ps, tp, table.shape[1], 0)

    def c(self, kv_heads, head_dim, dtype):
        if kv_heads != self.kv_heads or head_dim != self.head_dim or dtype != self.dtype:
            raise ValueError("the cache has kv heads, head_dim, dtype %s, the descriptor %s"
                             % ((self.kv_heads, self.head_dim, self.dtype), (kv_heads, head_dim, dtype)))
        return _byref(self._c)


_byref = ctypes.byref


def _cache(cache, kv_heads, head_dim, dtype):
    if not isinstance(cache, PagedCache):
        raise ValueError("cache must be a PagedCache")
    return cache.c(kv_heads, head_dim, dtype)


def _rows(t, name, dt, shape, dev):
    """Rows [tokens, heads, head_dim] of any token and head stride.  One expression where all is well: a
    small call is bound by its checks on the host."""
    try:
        st, sh, one = t.stride()
        if one == 1 and t.dtype is dt and t.shape == shape and t.get_device() == dev:
            return _byref(kvr_rows(t.data_ptr(), st, sh))
    except (AttributeError, TypeError, ValueError):      # no tensor, or of another rank
        pass
    _device(t, name)
    if t.dtype != dt:
        raise ValueError("%s must be a %s tensor, not %s" % (name, dt, t.dtype))
    if t.get_device() != dev:
        raise ValueError("%s is on GPU %d, other tensors of the call on GPU %d" % (name, t.get_device(), dev))
    if t.shape != shape:
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), shape))
    raise ValueError("%s: the elements of a row must be contiguous" % name)


def _vector(t, name, dtype, n, dev):
    """_at of a tensor of n values, or None"""
    if t is None:
        return None
    try:
        if t.dtype is dtype and t.shape == (n,) and t.get_device() == dev and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:      # no tensor
        pass
    return _at(t, name, dtype, (n,), dev)


def _rope_at(rope, desc, dev):
    if rope is None:
        return None
    r = _rope(rope, desc)
    if rope.cos_sin.get_device() != dev:
        raise ValueError("rope is on GPU %d, other tensors of the call on GPU %d" % (rope.cos_sin.get_device(), dev))
    return r


def kvr_qk_norm_rope(desc, q, k, q_out=None, k_out=None, rope=None, q_norm=None, k_norm=None, eps=1e-6, pos=None,
                     pos0=0, stream=None):
    """Head norms and rotation of rows q [n_tok, n_q_heads, head_dim] and k [n_tok, n_kv_heads,
    head_dim] (views with any token and head stride; either may be None) into q_out and k_out
    (default: in place).  q_norm, k_norm: weights [head_dim] or None; rope: a RopeTable or
    None; pos: int32 GPU tensor [n_tok], or token t is at pos0 + t."""
    Hq, Hkv, d, dt = desc.n_q_heads, desc.n_kv_heads, desc.head_dim, _TORCH_DTYPE.get(desc.dtype)
    some = k if q is None else q
    dev = _device(some, "k" if q is None else "q")
    if some.dim() != 3:
        raise ValueError("q and k must be tensors [n_tok, heads, head_dim]")
    n = some.shape[0]
    qi = qo = ki = ko = None
    if q is not None:
        qi = _rows(q, "q", dt, (n, Hq, d), dev)
        qo = qi if q_out is None else _rows(q_out, "q_out", dt, (n, Hq, d), dev)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if k is not None:
        ki = _rows(k, "k", dt, (n, Hkv, d), dev)
        ko = ki if k_out is None else _rows(k_out, "k_out", dt, (n, Hkv, d), dev)
    elif k_out is not None:
        raise ValueError("k_out without k")
    qn, kn = _vector(q_norm, "q_norm", dt, d, dev), _vector(k_norm, "k_norm", dt, d, dev)
    at, rp, p0 = _vector(pos, "pos", torch.int32, n, dev), _rope_at(rope, desc, dev), _fits(pos0, "pos0", 64)
    _launch(lambda s: load().kvr_qk_norm_rope(_byref(desc), rp, qi, ki, qn, kn, eps, n, at, p0, qo, ko, s),
            "kvr_qk_norm_rope", stream, dev)


def kvr_paged_append(desc, cache, k, v, length, rope=None, cu_seqlens=None, pos=None, q=None, q_out=None, q_norm=None,
                     k_norm=None, eps=1e-6, stream=None):
    """New tokens' keys and values k, v [n_tok, n_kv_heads, head_dim] (views with any token and
    head stride) into the pages of a PagedCache, the keys normalized (k_norm) and rotated
    (rope); their queries q [n_tok, n_q_heads, head_dim] likewise into q_out (default: in
    place).  length: int32 GPU tensor [n], rows that each sequence has; cu_seqlens: int32 GPU
    tensor [n + 1] of the packed tokens' sequences (None: one token each); pos: int32 GPU
    tensor [n_tok] of positions (None: the rows)."""
    Hkv, d, code = desc.n_kv_heads, desc.head_dim, desc.dtype
    pages = _cache(cache, Hkv, d, code)
    dt, dev, n = _TORCH_DTYPE[code], cache.device, cache.n
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("k must be a tensor [n_tok, n_kv_heads, head_dim]")
    T = k.shape[0]
    ki, vi = _rows(k, "k", dt, (T, Hkv, d), dev), _rows(v, "v", dt, (T, Hkv, d), dev)
    qi = qo = None
    if q is not None:
        shape = (T, desc.n_q_heads, d)
        qi = _rows(q, "q", dt, shape, dev)
        qo = qi if q_out is None else _rows(q_out, "q_out", dt, shape, dev)
    elif q_out is not None or q_norm is not None:
        raise ValueError("q_out or q_norm without q")
    qn, kn = _vector(q_norm, "q_norm", dt, d, dev), _vector(k_norm, "k_norm", dt, d, dev)
    ln = _at(length, "length", torch.int32, (n,), dev)
    cu, at = _vector(cu_seqlens, "cu_seqlens", torch.int32, n + 1, dev), _vector(pos, "pos", torch.int32, T, dev)
    rp = _rope_at(rope, desc, dev)
    _launch(lambda s: load().kvr_paged_append(_byref(desc), pages, rp, ki, vi, qi, qn, kn, eps, n, T, cu, ln, at, qo, s),
            "kvr_paged_append", stream, dev)


def kvr_workspace_bytes_paged(desc, n, max_len):
    return _bytes(load().kvr_workspace_bytes_paged(ctypes.byref(desc), _fits(n, "n"), _fits(max_len, "max_len", 64)))


def workspace_for_paged(desc, n, max_len, device="cuda"):
    """Allocate (with torch) the workspace of kvr_paged_decode."""
    return torch.empty(kvr_workspace_bytes_paged(desc, n, max_len), dtype=torch.uint8, device=device)


def kvr_paged_decode(desc, cache, q, length, out, ws=None, n_new=0, max_len=None, stream=None):
    """Attention of one token of each sequence, q [n, n_q_heads, head_dim] (a view with any
    token and head stride), into out, over rows [0, length + n_new) of a PagedCache.  length: int32 GPU tensor [n]; max_len: no sequence
    has more rows (default: all that the page table holds)."""
    Hkv, d, code = desc.n_kv_heads, desc.head_dim, desc.dtype
    pages = _cache(cache, Hkv, d, code)
    dt, dev, n = _TORCH_DTYPE[code], cache.device, cache.n
    shape = (n, desc.n_q_heads, d)
    qi, o = _rows(q, "q", dt, shape, dev), _at(out, "out", dt, shape, dev)
    ln = _at(length, "length", torch.int32, (n,), dev)
    wp, wn = _scratch(ws, dev)
    most, new = cache.reach if max_len is None else _fits(max_len, "max_len", 64), _fits(n_new, "n_new")
    _launch(lambda s: load().kvr_paged_decode(_byref(desc), pages, qi, n, ln, new, most, o, wp, wn, s),
            "kvr_paged_decode", stream, dev)
