"""Binding of the attention operators of ``libdeltanet_hip.so`` (declared in ``include/deltanet.h``): the norm and rotation of
queries and keys with its gradient, the paged cache, and attention over it.  Argument marshalling only, as ``binding``."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

from . import binding
from .binding import DN_BF16, DN_F32, _check, _p, _stream

DN_FP8 = 2


class dn_rope(ctypes.Structure):
    _fields_ = [("rot", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("max_pos", ctypes.c_int32), ("eps", ctypes.c_float)]


class dn_qk_shape(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("seq_len", ctypes.c_int32), ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64)]


class dn_paged_shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("num_seqs", "T", "Hq", "Hkv", "d", "dtype", "cache_dtype", "page_size", "num_pages",
                                              "max_pages", "max_q", "max_kv")] + [
        (n, ctypes.c_void_p) for n in ("cu_q", "kv_len", "page_table")] + [
        (n, ctypes.c_int64) for n in ("q_stride", "k_stride", "v_stride")]


class dn_paged_cache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("k_pages", "v_pages", "k_scale", "v_scale")]


torch = _TYPES = _lib = None


def _library():
    """The library; with the first call torch, which importing the package alone does not need (as in ``binding``)."""
    global torch, _TYPES, _lib
    if _lib is None:
        import torch as t
        torch, _TYPES = t, {t.float32: DN_F32, t.bfloat16: DN_BF16, t.float8_e4m3fn: DN_FP8}
        lib = binding.load_library()
        vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
        qk, ro, pg, ca = (ctypes.POINTER(t) for t in (dn_qk_shape, dn_rope, dn_paged_shape, dn_paged_cache))
        for name, args in (
                ("deltanet_qk_norm_rope_fwd", [qk, ro] + [vp] * 9),
                ("deltanet_qk_norm_rope_workspace_bytes", [qk, ctypes.POINTER(sz)]),
                ("deltanet_qk_norm_rope_bwd", [qk, ro] + [vp] * 13 + [sz, vp]),
                ("deltanet_paged_append", [pg, vp, vp, ca, vp]),
                ("deltanet_paged_norm_rope_append", [pg, ro] + [vp] * 7 + [ca, vp]),
                ("deltanet_paged_read", [pg, ca, vp, i32, vp, vp, vp]),
                ("deltanet_paged_attn_workspace_bytes", [pg, i32, ctypes.POINTER(sz)]),
                ("deltanet_paged_attn_fwd", [pg, vp, ca, ctypes.c_float, i32, vp, vp, sz, vp])):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = ctypes.c_int, args
        _lib = lib
    return _lib


def _type_of(t, name) -> int:
    if t.dtype != torch.float32 and t.dtype != torch.bfloat16:
        raise TypeError("%s must be float32 or bfloat16, got %s" % (name, t.dtype))
    return _TYPES[t.dtype]


def _rows(t, name, dtype, heads=None, d=None, T=None) -> int:
    """t is a device tensor [T, heads, d] whose rows are contiguous; returns the elements between rows"""
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.dim() != 3 or (T is not None and t.shape != (T, heads, d)):
        raise ValueError("%s must have shape %s, got %s" % (name, ("T", "heads", "d") if T is None else (T, heads, d), tuple(t.shape)))
    s = t.stride()
    if (s[2] != 1 and t.shape[2] > 1) or (s[1] != t.shape[2] and t.shape[1] > 1):
        raise ValueError("%s must have contiguous rows of heads x d" % name)
    return s[0] if t.shape[0] > 1 else t.shape[1] * t.shape[2]


def _whole(t, name, dtype, shape):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous device tensor" % name)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))


def _flat(t, name):
    """[B, L, H, d] (rows of a batch evenly spaced) as [B L, H, d]"""
    if t.dim() == 4:
        if t.shape[0] > 1 and t.shape[1] > 0 and t.stride(0) != t.shape[1] * t.stride(1):
            raise ValueError("%s must have evenly spaced rows" % name)
        return t.as_strided((t.shape[0] * t.shape[1],) + tuple(t.shape[2:]), t.stride()[1:] if t.shape[1] > 1 or t.shape[0] <= 1
                            else (t.stride(0),) + t.stride()[2:])
    return t


def _rope(rope, d, eps, interleaved, device) -> dn_rope:
    r = dn_rope()
    r.interleaved, r.eps = int(bool(interleaved)), eps
    if rope is not None:
        if rope.dim() != 2:
            raise ValueError("rope must be [max_pos, rot], cosines then sines")
        _whole(rope, "rope", torch.float32, rope.shape)
        r.max_pos, r.rot = rope.shape
    return r


def _weights(q_weight, k_weight, dtype, d):
    for w, name in ((q_weight, "q_weight"), (k_weight, "k_weight")):
        if w is not None:
            _whole(w, name, dtype, (d,))


def _qk_shape(q, k, positions) -> Tuple[dn_qk_shape, "torch.Tensor", "torch.Tensor"]:
    s = dn_qk_shape()
    s.seq_len = q.shape[1] if q.dim() == 4 else q.shape[0]
    s.dtype = _type_of(q, "q")
    if k.dim() != q.dim() or (q.dim() == 4 and k.shape[:2] != q.shape[:2]):
        raise ValueError("q and k must have the same rows")
    q, k = _flat(q, "q"), _flat(k, "k")
    s.q_stride = _rows(q, "q", q.dtype)
    s.T, s.Hq, s.d = q.shape
    s.Hkv = k.shape[1] if k.dim() == 3 else 0
    s.k_stride = _rows(k, "k", q.dtype, s.Hkv, s.d, s.T)
    s.seq_len = max(s.seq_len, 1)
    if positions is not None:
        _whole(positions, "positions", torch.int32, (s.T,))
    return s, q, k


def _out(t, name, like_shape, dtype, device):
    if t is None:
        return torch.empty(like_shape, dtype=dtype, device=device)
    _whole(t, name, dtype, like_shape)
    return t


def deltanet_qk_norm_rope_fwd(q, k, q_weight=None, k_weight=None, rope=None, positions=None, *, eps: float = 1e-6,
                              interleaved: bool = False, q_out=None, k_out=None, stream=None) -> Tuple["torch.Tensor", "torch.Tensor"]:
    """RMS norm of every head's query and key, times its weight, then rotated by the row's position; returns (q_out, k_out).
    q [T, Hq, d] or [B, L, Hq, d] and k may be column blocks of one projection's output (rows apart).  rope: fp32 [max_pos, rot],
    the rot / 2 cosines and then the rot / 2 sines of every position, or None for no rotation.  positions: int32, one per
    row; without it a row's place in its sequence (dense) or in the tensor (packed)."""
    lib = _library()
    q_shape, k_shape = q.shape, k.shape
    s, q, k = _qk_shape(q, k, positions)
    r = _rope(rope, s.d, eps, interleaved, q.device)
    _weights(q_weight, k_weight, q.dtype, s.d)
    q_out = _out(q_out, "q_out", q_shape, q.dtype, q.device)
    k_out = _out(k_out, "k_out", k_shape, q.dtype, q.device)
    _check(lib.deltanet_qk_norm_rope_fwd(s, r, _p(q), _p(k), _p(q_weight), _p(k_weight), _p(rope), _p(positions), _p(q_out), _p(k_out),
                                         _stream(stream)))
    return q_out, k_out


def deltanet_qk_norm_rope_bwd(q, k, dq_out, dk_out, q_weight=None, k_weight=None, rope=None, positions=None, *, eps: float = 1e-6,
                              interleaved: bool = False, dq=None, dk=None, dq_weight=None, dk_weight=None, workspace=None,
                              stream=None):
    """Gradient of deltanet_qk_norm_rope_fwd; returns (dq, dk, dq_weight, dk_weight), the last two in fp32 and None where there is no
    weight.  dq and dk may be dq_out and dk_out themselves."""
    lib = _library()
    q_shape, k_shape = q.shape, k.shape
    s, q, k = _qk_shape(q, k, positions)
    r = _rope(rope, s.d, eps, interleaved, q.device)
    _weights(q_weight, k_weight, q.dtype, s.d)
    _whole(dq_out, "dq_out", q.dtype, q_shape)
    _whole(dk_out, "dk_out", q.dtype, k_shape)
    dq = _out(dq, "dq", q_shape, q.dtype, q.device)
    dk = _out(dk, "dk", k_shape, q.dtype, q.device)
    if q_weight is not None:
        dq_weight = _out(dq_weight, "dq_weight", (s.d,), torch.float32, q.device)
    if k_weight is not None:
        dk_weight = _out(dk_weight, "dk_weight", (s.d,), torch.float32, q.device)
    if (q_weight is None and dq_weight is not None) or (k_weight is None and dk_weight is not None):
        raise ValueError("no gradient of a weight that is not there")
    need = ctypes.c_size_t(0)
    _check(lib.deltanet_qk_norm_rope_workspace_bytes(s, need))
    if workspace is None:
        workspace = torch.empty(max(need.value, 16), dtype=torch.uint8, device=q.device)
    _check(lib.deltanet_qk_norm_rope_bwd(s, r, _p(q), _p(k), _p(dq_out), _p(dk_out), _p(q_weight), _p(k_weight), _p(rope), _p(positions),
                                         _p(dq), _p(dk), _p(dq_weight), _p(dk_weight), _p(workspace),
                                         workspace.numel() * workspace.element_size(), _stream(stream)))
    return dq, dk, dq_weight, dk_weight


def deltanet_paged_cache(num_pages: int, page_size: int, heads: int, d: int, dtype=None, device="cuda"):
    """The tensors of one layer's cache: (k_pages, v_pages, k_scale, v_scale), the scales None unless dtype (bfloat16 by default)
    is float8_e4m3fn."""
    _library()
    dtype = torch.bfloat16 if dtype is None else dtype
    if dtype not in _TYPES:
        raise TypeError("a cache is float32, bfloat16 or float8_e4m3fn, got %s" % dtype)
    k, v = (torch.empty(num_pages, heads, page_size, d, dtype=dtype, device=device) for _ in range(2))
    ks, vs = ((torch.empty(num_pages, heads, page_size, dtype=torch.float32, device=device) if dtype == torch.float8_e4m3fn else None)
              for _ in range(2))
    return k, v, ks, vs


def _paged(k_pages, v_pages, k_scale, v_scale, page_table, kv_len, cu_q, dtype) -> Tuple[dn_paged_shape, dn_paged_cache]:
    if k_pages.dim() != 4:
        raise ValueError("k_pages must be [num_pages, heads, page_size, d]")
    if k_pages.dtype not in _TYPES:
        raise TypeError("k_pages must be float32, bfloat16 or float8_e4m3fn, got %s" % k_pages.dtype)
    shape = k_pages.shape
    _whole(k_pages, "k_pages", k_pages.dtype, shape)
    _whole(v_pages, "v_pages", k_pages.dtype, shape)
    quantised = k_pages.dtype == torch.float8_e4m3fn
    if not quantised and k_pages.dtype != dtype:
        raise TypeError("pages must be %s or float8_e4m3fn, got %s" % (dtype, k_pages.dtype))
    for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
        if quantised:
            if t is None:
                raise ValueError("%s is needed for an 8-bit cache" % name)
            _whole(t, name, torch.float32, shape[:3])
        elif t is not None:
            raise ValueError("%s belongs to an 8-bit cache" % name)
    s = dn_paged_shape()
    if page_table.dim() != 2:
        raise ValueError("page_table must be [sequences, max_pages]")
    N, M = page_table.shape
    _whole(page_table, "page_table", torch.int32, page_table.shape)
    _whole(kv_len, "kv_len", torch.int32, (N,))
    _whole(cu_q, "cu_q", torch.int32, (N + 1,))
    s.num_seqs, s.max_pages = N, M
    s.num_pages, s.Hkv, s.page_size, s.d = shape
    s.dtype, s.cache_dtype = _TYPES[dtype], _TYPES[k_pages.dtype]
    s.max_kv = min(M * shape[2], 2 ** 31 - 1)
    s.cu_q, s.kv_len, s.page_table = cu_q.data_ptr(), kv_len.data_ptr(), page_table.data_ptr()
    c = dn_paged_cache(k_pages.data_ptr(), v_pages.data_ptr(), _p(k_scale), _p(v_scale))
    return s, c


def deltanet_paged_append(k, v, k_pages, v_pages, page_table, kv_len, cu_q, *, k_scale=None, v_scale=None, stream=None) -> None:
    """Writes the new tokens' k and v [T, Hkv, d] to the paged cache (8-bit pages: quantised on the way).  Sequence n's new tokens are
    rows cu_q[n] .. cu_q[n + 1] - 1, the last of them token kv_len[n] - 1 of its context; its token p stands in page
    page_table[n, p // page_size], slot p % page_size."""
    lib = _library()
    dt = _type_of(k, "k")
    s, c = _paged(k_pages, v_pages, k_scale, v_scale, page_table, kv_len, cu_q, k.dtype)
    s.dtype, s.T, s.Hq = dt, k.shape[0], s.Hkv
    s.k_stride = _rows(k, "k", k.dtype, s.Hkv, s.d, s.T)
    s.v_stride = _rows(v, "v", k.dtype, s.Hkv, s.d, s.T)
    _check(lib.deltanet_paged_append(s, _p(k), _p(v), c, _stream(stream)))


def deltanet_paged_norm_rope_append(q, k, v, k_pages, v_pages, page_table, kv_len, cu_q, q_weight=None, k_weight=None, rope=None, *,
                                    k_scale=None, v_scale=None, eps: float = 1e-6, interleaved: bool = False, q_out=None,
                                    stream=None) -> "torch.Tensor":
    """The serving form of deltanet_qk_norm_rope_fwd, in one pass with deltanet_paged_append: k normalised and rotated, and v, go to the
    cache; returns q normalised and rotated.  Positions are the tokens' places in their contexts."""
    lib = _library()
    dt = _type_of(q, "q")
    s, c = _paged(k_pages, v_pages, k_scale, v_scale, page_table, kv_len, cu_q, q.dtype)
    s.dtype = dt
    s.q_stride = _rows(q, "q", q.dtype)
    s.T, s.Hq = q.shape[:2]
    if q.shape[2] != s.d:
        raise ValueError("q must have the cache's head size")
    s.k_stride = _rows(k, "k", q.dtype, s.Hkv, s.d, s.T)
    s.v_stride = _rows(v, "v", q.dtype, s.Hkv, s.d, s.T)
    r = _rope(rope, s.d, eps, interleaved, q.device)
    _weights(q_weight, k_weight, q.dtype, s.d)
    q_out = _out(q_out, "q_out", q.shape, q.dtype, q.device)
    _check(lib.deltanet_paged_norm_rope_append(s, r, _p(q), _p(k), _p(v), _p(q_weight), _p(k_weight), _p(rope), _p(q_out), c, _stream(stream)))
    return q_out


def deltanet_paged_read(k_pages, v_pages, page_table, kv_len, cu_out, rows: int, *, dtype=None, k_scale=None, v_scale=None, k_out=None,
                        v_out=None, stream=None) -> Tuple["torch.Tensor", "torch.Tensor"]:
    """Reads tokens back from the paged cache, as k, v [rows, Hkv, d] of `dtype` (the pages' type; bfloat16 for 8-bit pages): rows
    cu_out[n] .. cu_out[n + 1] - 1 are the last tokens of sequence n's context, zeros in front of its start."""
    lib = _library()
    if dtype is None:
        dtype = torch.bfloat16 if k_pages.dtype == torch.float8_e4m3fn else k_pages.dtype
    if dtype != torch.float32 and dtype != torch.bfloat16:
        raise TypeError("dtype must be float32 or bfloat16, got %s" % dtype)
    s, c = _paged(k_pages, v_pages, k_scale, v_scale, page_table, kv_len, cu_out, dtype)
    s.T, s.Hq = 0, s.Hkv
    shape = (rows, s.Hkv, s.d)
    k_out = _out(k_out, "k_out", shape, dtype, k_pages.device)
    v_out = _out(v_out, "v_out", shape, dtype, k_pages.device)
    _check(lib.deltanet_paged_read(s, c, cu_out.data_ptr(), rows, _p(k_out), _p(v_out), _stream(stream)))
    return k_out, v_out


def deltanet_paged_attn_workspace_bytes(shape: dn_paged_shape, window: int = 0) -> int:
    out = ctypes.c_size_t(0)
    _check(_library().deltanet_paged_attn_workspace_bytes(shape, window, out))
    return int(out.value)


def deltanet_paged_attn_fwd(q, k_pages, v_pages, page_table, kv_len, cu_q, *, k_scale=None, v_scale=None, scale: Optional[float] = None,
                            window: int = 0, max_q: Optional[int] = None, max_kv: Optional[int] = None, o=None, workspace=None,
                            stream=None) -> "torch.Tensor":
    """Attention of the new tokens q [T, Hq, d] over the paged cache, which holds their own keys and values already; returns o
    [T, Hq, d].  The row at position p sees keys max(0, p - window + 1) .. p (window 0: its whole past); scale is d ** -0.5 by
    default.  max_q and max_kv: bounds on the longest chunk and the longest context (T and the page table's width by default; close bounds
    make for better-sized launches)."""
    lib = _library()
    dt = _type_of(q, "q")
    s, c = _paged(k_pages, v_pages, k_scale, v_scale, page_table, kv_len, cu_q, q.dtype)
    s.dtype = dt
    s.q_stride = _rows(q, "q", q.dtype)
    s.T, s.Hq = q.shape[:2]
    if q.shape[2] != s.d:
        raise ValueError("q must have the cache's head size")
    s.max_q = s.T if max_q is None else max_q
    if max_kv is not None:
        s.max_kv = max_kv
    o = _out(o, "o", q.shape, q.dtype, q.device)
    need = deltanet_paged_attn_workspace_bytes(s, window)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
    _check(lib.deltanet_paged_attn_fwd(s, _p(q), c, s.d ** -0.5 if scale is None else scale, window, _p(o), _p(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream)))
    return o
