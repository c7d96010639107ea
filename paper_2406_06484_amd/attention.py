"""Binding of the attention operators of ``libdeltanet_hip.so`` (declared in ``include/deltanet.h``): the norm and rotation of
queries and keys with its gradient, the paged cache, and attention over it.  Argument marshalling only, as ``binding``."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

from . import binding
from .binding import DN_BF16, DN_F32, _check, _p

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


# A decode step calls these functions some tens of times, and the device is done with each call in a few microseconds: the checks are
# written for the call that passes them (one condition per tensor; what was wrong is found out afterwards).

def _type_of(t, name) -> int:
    if t.dtype is not torch.float32 and t.dtype is not torch.bfloat16:
        raise TypeError("%s must be float32 or bfloat16, got %s" % (name, t.dtype))
    return _TYPES[t.dtype]


def _refuse(t, name, dtype, shape):
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    raise ValueError("%s must be contiguous%s" % (name, " within its rows of heads x d" if t.dim() == 3 else ""))


def _rows(t, name, dtype, shape) -> int:
    """t is a device tensor [T, heads, d] whose rows are contiguous; returns the elements between rows"""
    T, H, d = shape
    if not (t.is_cuda and t.dtype is dtype and t.shape == shape):
        _refuse(t, name, dtype, shape)
    s0, s1, s2 = t.stride()
    if s2 != 1 or s1 != d:      # (strides of axes with one element say nothing)
        if (s2 != 1 and d > 1) or (s1 != d and H > 1):
            _refuse(t, name, dtype, shape)
    return s0 if T > 1 else H * d


def _whole(t, name, dtype, shape):
    if not (t.is_cuda and t.dtype is dtype and t.is_contiguous() and t.shape == shape):
        _refuse(t, name, dtype, shape)


def _three(t, name):
    if t.dim() != 3:
        raise ValueError("%s must be [T, heads, d], got %s" % (name, tuple(t.shape)))
    return t.shape


def _stream_of(stream, t) -> Optional[int]:
    """The given stream's handle, or that of the current stream of t's device."""
    return (torch._C._cuda_getCurrentRawStream(t.get_device()) if stream is None else stream.cuda_stream) or None


def _flat(t, name):
    """[B, L, H, d] (rows of a batch evenly spaced) as [B L, H, d]"""
    if t.dim() == 4:
        if t.shape[0] > 1 and t.shape[1] > 0 and t.stride(0) != t.shape[1] * t.stride(1):
            raise ValueError("%s must have evenly spaced rows" % name)
        return t.as_strided((t.shape[0] * t.shape[1],) + tuple(t.shape[2:]), t.stride()[1:] if t.shape[1] > 1 or t.shape[0] <= 1
                            else (t.stride(0),) + t.stride()[2:])
    return t


def _rope(rope, d, eps, interleaved) -> dn_rope:
    r = dn_rope()
    r.interleaved, r.eps = bool(interleaved), eps
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
    seq_len = q.shape[0]
    if q.dim() == 4 and k.dim() == 4:
        if k.shape[:2] != q.shape[:2]:
            raise ValueError("q and k must have the same rows")
        seq_len = q.shape[1]
        q, k = _flat(q, "q"), _flat(k, "k")
    s.dtype = _type_of(q, "q")
    T, Hq, d = shape = _three(q, "q")
    Hkv = _three(k, "k")[1]
    s.q_stride = _rows(q, "q", q.dtype, shape)
    s.k_stride = _rows(k, "k", q.dtype, (T, Hkv, d))
    s.T, s.Hq, s.Hkv, s.d, s.seq_len = T, Hq, Hkv, d, max(seq_len, 1)
    if positions is not None:
        _whole(positions, "positions", torch.int32, (T,))
    return s, q, k


def _out(t, name, shape, like):
    if t is None:
        return like.new_empty(shape)
    _whole(t, name, like.dtype, shape)
    return t


def _sum_out(t, name, d, like):
    if t is None:
        return torch.empty(d, dtype=torch.float32, device=like.device)
    _whole(t, name, torch.float32, (d,))
    return t


def _scratch(workspace, need, like):
    """(pointer, bytes) of the caller's workspace, or of one for this call, and what keeps it alive"""
    if workspace is None:
        if need == 0:
            return None, 0, None
        workspace = torch.empty(need, dtype=torch.uint8, device=like.device)
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def deltanet_qk_norm_rope_fwd(q, k, q_weight=None, k_weight=None, rope=None, positions=None, *, eps: float = 1e-6,
                              interleaved: bool = False, q_out=None, k_out=None, stream=None) -> Tuple["torch.Tensor", "torch.Tensor"]:
    """RMS norm of every head's query and key, times its weight, then rotated by the row's position; returns (q_out, k_out).
    q [T, Hq, d] or [B, L, Hq, d] and k may be column blocks of one projection's output (rows apart).  rope: fp32 [max_pos, rot],
    the rot / 2 cosines and then the rot / 2 sines of every position, or None for no rotation.  positions: int32, one per
    row; without it a row's place in its sequence (dense) or in the tensor (packed)."""
    lib = _library()
    q_shape, k_shape = q.shape, k.shape
    s, q, k = _qk_shape(q, k, positions)
    r = _rope(rope, s.d, eps, interleaved)
    _weights(q_weight, k_weight, q.dtype, s.d)
    q_out = _out(q_out, "q_out", q_shape, q)
    k_out = _out(k_out, "k_out", k_shape, q)
    _check(lib.deltanet_qk_norm_rope_fwd(s, r, _p(q), _p(k), _p(q_weight), _p(k_weight), _p(rope), _p(positions), _p(q_out), _p(k_out),
                                         _stream_of(stream, q)))
    return q_out, k_out


def deltanet_qk_norm_rope_bwd(q, k, dq_out, dk_out, q_weight=None, k_weight=None, rope=None, positions=None, *, eps: float = 1e-6,
                              interleaved: bool = False, dq=None, dk=None, dq_weight=None, dk_weight=None, workspace=None,
                              stream=None):
    """Gradient of deltanet_qk_norm_rope_fwd; returns (dq, dk, dq_weight, dk_weight), the last two in fp32 and None where there is no
    weight.  dq and dk may be dq_out and dk_out themselves."""
    lib = _library()
    q_shape, k_shape = q.shape, k.shape
    s, q, k = _qk_shape(q, k, positions)
    r = _rope(rope, s.d, eps, interleaved)
    _weights(q_weight, k_weight, q.dtype, s.d)
    _whole(dq_out, "dq_out", q.dtype, q_shape)
    _whole(dk_out, "dk_out", q.dtype, k_shape)
    dq = _out(dq, "dq", q_shape, q)
    dk = _out(dk, "dk", k_shape, q)
    if q_weight is not None:
        dq_weight = _sum_out(dq_weight, "dq_weight", s.d, q)
    if k_weight is not None:
        dk_weight = _sum_out(dk_weight, "dk_weight", s.d, q)
    if (q_weight is None and dq_weight is not None) or (k_weight is None and dk_weight is not None):
        raise ValueError("no gradient of a weight that is not there")
    need = ctypes.c_size_t(0)
    _check(lib.deltanet_qk_norm_rope_workspace_bytes(s, need))
    ws, ws_bytes, workspace = _scratch(workspace, need.value if dq_weight is not None or dk_weight is not None else 0, q)
    _check(lib.deltanet_qk_norm_rope_bwd(s, r, _p(q), _p(k), _p(dq_out), _p(dk_out), _p(q_weight), _p(k_weight), _p(rope), _p(positions),
                                         _p(dq), _p(dk), _p(dq_weight), _p(dk_weight), ws, ws_bytes, _stream_of(stream, q)))
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
    if k_pages.dim() != 4 or page_table.dim() != 2:
        raise ValueError("k_pages must be [num_pages, heads, page_size, d], page_table [sequences, max_pages]")
    pages, heads, page_size, d = shape = k_pages.shape
    N, width = of_table = page_table.shape
    held, i32 = k_pages.dtype, torch.int32
    if held not in _TYPES:
        raise TypeError("k_pages must be float32, bfloat16 or float8_e4m3fn, got %s" % held)
    _whole(k_pages, "k_pages", held, shape)
    _whole(v_pages, "v_pages", held, shape)
    c = dn_paged_cache(k_pages.data_ptr(), v_pages.data_ptr())
    if held is torch.float8_e4m3fn:
        if k_scale is None or v_scale is None:
            raise ValueError("k_scale and v_scale are needed for an 8-bit cache")
        _whole(k_scale, "k_scale", torch.float32, (pages, heads, page_size))
        _whole(v_scale, "v_scale", torch.float32, (pages, heads, page_size))
        c.k_scale, c.v_scale = k_scale.data_ptr(), v_scale.data_ptr()
    elif held is not dtype:
        raise TypeError("pages must be %s or float8_e4m3fn, got %s" % (dtype, held))
    elif k_scale is not None or v_scale is not None:
        raise ValueError("scales belong to an 8-bit cache")
    _whole(page_table, "page_table", i32, of_table)
    _whole(kv_len, "kv_len", i32, (N,))
    _whole(cu_q, "cu_q", i32, (N + 1,))
    s = dn_paged_shape()
    s.num_seqs, s.max_pages = N, width
    s.num_pages, s.Hkv, s.page_size, s.d = pages, heads, page_size, d
    s.dtype, s.cache_dtype = _TYPES[dtype], _TYPES[held]
    s.max_kv = min(width * page_size, 2 ** 31 - 1)
    s.cu_q, s.kv_len, s.page_table = cu_q.data_ptr(), kv_len.data_ptr(), page_table.data_ptr()
    return s, c


def deltanet_paged_append(k, v, k_pages, v_pages, page_table, kv_len, cu_q, *, k_scale=None, v_scale=None, stream=None) -> None:
    """Writes the new tokens' k and v [T, Hkv, d] to the paged cache (8-bit pages: quantised on the way).  Sequence n's new tokens are
    rows cu_q[n] .. cu_q[n + 1] - 1, the last of them token kv_len[n] - 1 of its context; its token p stands in page
    page_table[n, p // page_size], slot p % page_size."""
    lib = _library()
    _type_of(k, "k")
    s, c = _paged(k_pages, v_pages, k_scale, v_scale, page_table, kv_len, cu_q, k.dtype)
    T = _three(k, "k")[0]
    s.T, s.Hq = T, s.Hkv
    s.k_stride = _rows(k, "k", k.dtype, (T, s.Hkv, s.d))
    s.v_stride = _rows(v, "v", k.dtype, (T, s.Hkv, s.d))
    _check(lib.deltanet_paged_append(s, k.data_ptr(), v.data_ptr(), c, _stream_of(stream, k)))


def deltanet_paged_norm_rope_append(q, k, v, k_pages, v_pages, page_table, kv_len, cu_q, q_weight=None, k_weight=None, rope=None, *,
                                    k_scale=None, v_scale=None, eps: float = 1e-6, interleaved: bool = False, q_out=None,
                                    stream=None) -> "torch.Tensor":
    """The serving form of deltanet_qk_norm_rope_fwd, in one pass with deltanet_paged_append: k normalised and rotated, and v, go to the
    cache; returns q normalised and rotated.  Positions are the tokens' places in their contexts."""
    lib = _library()
    _type_of(q, "q")
    s, c = _paged(k_pages, v_pages, k_scale, v_scale, page_table, kv_len, cu_q, q.dtype)
    T, Hq, _ = shape = _three(q, "q")
    Hkv, d = s.Hkv, s.d
    s.T, s.Hq = T, Hq
    s.q_stride = _rows(q, "q", q.dtype, (T, Hq, d))
    s.k_stride = _rows(k, "k", q.dtype, (T, Hkv, d))
    s.v_stride = _rows(v, "v", q.dtype, (T, Hkv, d))
    r = _rope(rope, d, eps, interleaved)
    _weights(q_weight, k_weight, q.dtype, d)
    q_out = _out(q_out, "q_out", shape, q)
    _check(lib.deltanet_paged_norm_rope_append(s, r, q.data_ptr(), k.data_ptr(), v.data_ptr(), _p(q_weight), _p(k_weight), _p(rope),
                                               q_out.data_ptr(), c, _stream_of(stream, q)))
    return q_out


def deltanet_paged_read(k_pages, v_pages, page_table, kv_len, cu_out, rows: int, *, dtype=None, k_scale=None, v_scale=None, k_out=None,
                        v_out=None, stream=None) -> Tuple["torch.Tensor", "torch.Tensor"]:
    """Reads tokens back from the paged cache, as k, v [rows, Hkv, d] of `dtype` (the pages' type; bfloat16 for 8-bit pages): rows
    cu_out[n] .. cu_out[n + 1] - 1 are the last tokens of sequence n's context, zeros in front of its start."""
    lib = _library()
    if dtype is None:
        dtype = torch.bfloat16 if k_pages.dtype == torch.float8_e4m3fn else k_pages.dtype
    if dtype is not torch.float32 and dtype is not torch.bfloat16:
        raise TypeError("dtype must be float32 or bfloat16, got %s" % dtype)
    s, c = _paged(k_pages, v_pages, k_scale, v_scale, page_table, kv_len, cu_out, dtype)
    s.T, s.Hq = 0, s.Hkv
    shape = (rows, s.Hkv, s.d)
    if k_out is None:
        k_out = torch.empty(shape, dtype=dtype, device=k_pages.device)
    if v_out is None:
        v_out = torch.empty(shape, dtype=dtype, device=k_pages.device)
    _whole(k_out, "k_out", dtype, shape)
    _whole(v_out, "v_out", dtype, shape)
    _check(lib.deltanet_paged_read(s, c, cu_out.data_ptr(), rows, k_out.data_ptr(), v_out.data_ptr(), _stream_of(stream, k_pages)))
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
    _type_of(q, "q")
    s, c = _paged(k_pages, v_pages, k_scale, v_scale, page_table, kv_len, cu_q, q.dtype)
    T, Hq, _ = shape = _three(q, "q")
    s.T, s.Hq = T, Hq
    s.q_stride = _rows(q, "q", q.dtype, (T, Hq, s.d))
    s.max_q = T if max_q is None else max_q
    if max_kv is not None:
        s.max_kv = max_kv
    o = _out(o, "o", shape, q)
    need = ctypes.c_size_t(0)
    _check(lib.deltanet_paged_attn_workspace_bytes(s, window, need))
    ws, ws_bytes, workspace = _scratch(workspace, need.value, q)
    _check(lib.deltanet_paged_attn_fwd(s, q.data_ptr(), c, s.d ** -0.5 if scale is None else scale, window, o.data_ptr(), ws, ws_bytes,
                                       _stream_of(stream, q)))
    return o
