"""Binding of the attention operators of ``libdeltanet_hip.so`` (declared in ``include/deltanet.h``): the norm and rotation of
queries and keys with its gradient, the paged cache, and attention over it.  Argument marshalling only, as ``binding``; the calls go through the
compiled module ``_attention`` (csrc/dn_attention_binding.cpp), which checks tensors and allocates what the caller did not bring (the library wants arrays of 16-byte
alignment: offsets, lengths, tables and positions that are parts of larger ones are copied on the way where they need it).  A missing
library or module raises; there is no fallback."""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

from . import binding
from .binding import DN_BF16, DN_F32, _check

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


_lib = _ext = None


def _library():
    """The C ABI of the attention operators through ctypes."""
    global _lib
    if _lib is None:
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


def _module():
    """The compiled module, opened on the library (and with it torch, which importing the package alone does not need)."""
    global _ext
    if _ext is None:
        import importlib.util

        import torch
        binding.load_library()
        path = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_attention.so")
        if not os.path.exists(path):
            raise FileNotFoundError("%s is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`" % path)
        spec = importlib.util.spec_from_file_location("_attention", path)
        ext = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(ext)
        ext.open(binding.library_path(), torch._C._cuda_getCurrentRawStream)
        _ext = ext
    return _ext


def _call(name: str, stream, *args):
    fn = getattr(_ext or _module(), name)
    if stream is None:
        r = fn(*args)
    else:
        import torch
        with torch.cuda.stream(stream):     # what the call allocates belongs to the stream that works on it
            r = fn(*args)
    if type(r) is int:
        _check(r)
    return r


def deltanet_qk_norm_rope_fwd(q, k, q_weight=None, k_weight=None, rope=None, positions=None, *, eps: float = 1e-6,
                              interleaved: bool = False, q_out=None, k_out=None, stream=None) -> Tuple["torch.Tensor", "torch.Tensor"]:
    """RMS norm of every head's query and key, times its weight, then rotated by the row's position; returns (q_out, k_out).
    q [T, Hq, d] or [B, L, Hq, d] and k may be column blocks of one projection's output (rows apart).  rope: fp32 [max_pos, rot],
    the rot / 2 cosines and then the rot / 2 sines of every position, or None for no rotation.  positions: int32, one per
    row; without it a row's place in its sequence (dense) or in the tensor (packed)."""
    return _call("norm_rope_fwd", stream, q, k, q_weight, k_weight, rope, positions, eps, interleaved, q_out, k_out)


def deltanet_qk_norm_rope_bwd(q, k, dq_out, dk_out, q_weight=None, k_weight=None, rope=None, positions=None, *, eps: float = 1e-6,
                              interleaved: bool = False, dq=None, dk=None, dq_weight=None, dk_weight=None, workspace=None,
                              stream=None):
    """Gradient of deltanet_qk_norm_rope_fwd; returns (dq, dk, dq_weight, dk_weight), the last two in fp32 and None where there is no
    weight.  dq and dk may be dq_out and dk_out themselves."""
    return _call("norm_rope_bwd", stream, q, k, dq_out, dk_out, q_weight, k_weight, rope, positions, eps, interleaved, dq, dk,
                 dq_weight, dk_weight, workspace)


def deltanet_paged_cache(num_pages: int, page_size: int, heads: int, d: int, dtype=None, device="cuda"):
    """The tensors of one layer's cache: (k_pages, v_pages, k_scale, v_scale), the scales None unless dtype (bfloat16 by default)
    is float8_e4m3fn."""
    import torch
    dtype = torch.bfloat16 if dtype is None else dtype
    if dtype not in (torch.float32, torch.bfloat16, torch.float8_e4m3fn):
        raise TypeError("a cache is float32, bfloat16 or float8_e4m3fn, got %s" % dtype)
    k, v = (torch.empty(num_pages, heads, page_size, d, dtype=dtype, device=device) for _ in range(2))
    ks, vs = ((torch.empty(num_pages, heads, page_size, dtype=torch.float32, device=device) if dtype == torch.float8_e4m3fn else None)
              for _ in range(2))
    return k, v, ks, vs


def deltanet_paged_append(k, v, k_pages, v_pages, page_table, kv_len, cu_q, *, k_scale=None, v_scale=None, stream=None) -> None:
    """Writes the new tokens' k and v [T, Hkv, d] to the paged cache (8-bit pages: quantised on the way).  Sequence n's new tokens are
    rows cu_q[n] .. cu_q[n + 1] - 1, the last of them token kv_len[n] - 1 of its context; its token p stands in page
    page_table[n, p // page_size], slot p % page_size."""
    return _call("append", stream, k, v, k_pages, v_pages, page_table, kv_len, cu_q, k_scale, v_scale)


def deltanet_paged_norm_rope_append(q, k, v, k_pages, v_pages, page_table, kv_len, cu_q, q_weight=None, k_weight=None, rope=None, *,
                                    k_scale=None, v_scale=None, eps: float = 1e-6, interleaved: bool = False, q_out=None,
                                    stream=None) -> "torch.Tensor":
    """The serving form of deltanet_qk_norm_rope_fwd, in one pass with deltanet_paged_append: k normalised and rotated, and v, go to the
    cache; returns q normalised and rotated.  Positions are the tokens' places in their contexts."""
    return _call("norm_rope_append", stream, q, k, v, k_pages, v_pages, page_table, kv_len, cu_q, q_weight, k_weight, rope,
                 k_scale, v_scale, eps, interleaved, q_out)


def deltanet_paged_read(k_pages, v_pages, page_table, kv_len, cu_out, rows: int, *, dtype=None, k_scale=None, v_scale=None, k_out=None,
                        v_out=None, stream=None) -> Tuple["torch.Tensor", "torch.Tensor"]:
    """Reads tokens back from the paged cache, as k, v [rows, Hkv, d] of `dtype` (the pages' type; bfloat16 for 8-bit pages): rows
    cu_out[n] .. cu_out[n + 1] - 1 are the last tokens of sequence n's context, zeros in front of its start."""
    import torch
    held = k_pages.dtype if dtype is None else dtype
    if held is torch.bfloat16 or (dtype is None and held is torch.float8_e4m3fn):
        code = DN_BF16
    elif held is torch.float32:
        code = DN_F32
    else:
        raise TypeError("dtype must be float32 or bfloat16, got %s" % held)
    return _call("read", stream, k_pages, v_pages, page_table, kv_len, cu_out, rows, code, k_scale, v_scale, k_out, v_out)


def deltanet_paged_attn_workspace_bytes(shape: dn_paged_shape, window: int = 0) -> int:
    out = ctypes.c_size_t(0)
    _check(_library().deltanet_paged_attn_workspace_bytes(shape, window, out))
    return int(out.value)


def deltanet_paged_attn_fwd(q, k_pages, v_pages, page_table, kv_len, cu_q, *, k_scale=None, v_scale=None, scale: Optional[float] = None,
                            window: int = 0, max_q: Optional[int] = None, max_kv: Optional[int] = None, o=None, workspace=None,
                            stream=None) -> "torch.Tensor":
    """Attention of the new tokens q [T, Hq, d] over the paged cache, which holds their own keys and values already; returns o
    [T, Hq, d].  The row at position p sees keys max(0, p - window + 1) .. p (window 0: its whole past); scale is d ** -0.5 by
    default.  max_q and max_kv: bounds on the longest chunk and the longest context, at most T and the tokens that the page table has room for, which they
    are by default (a constant bound of the caller's is passed as min(bound, T)); close bounds make for better-sized launches."""
    return _call("attn", stream, q, k_pages, v_pages, page_table, kv_len, cu_q, k_scale, v_scale, scale, window, max_q, max_kv, o,
                 workspace)
