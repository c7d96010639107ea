"""Binding of the operators around a mixer in ``libdeltanet_hip.so`` (declared in ``include/deltanet.h``): the short convolution in front of it, the norm of its
output with its gate, and what stands between two blocks (branch norm, gate, residual sum, next norm), each with its gradient.  Argument marshalling only; calls go through the
compiled module ``_attention`` (csrc/dn_layer_binding.cpp), as those of ``attention``.  A missing library or module raises; there is no fallback."""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence, Tuple, Union

from . import binding
from .attention import _call

_ACTS = {"silu": 1, "sigmoid": 2}


class dn_conv_shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "L", "C", "W", "dtype", "num_seqs")] + [
        ("cu_seqlens", ctypes.c_void_p), ("cu_seqlens_host", ctypes.c_void_p), ("parts", ctypes.c_int32),
        ("width", ctypes.c_int32 * 3), ("silu", ctypes.c_int32 * 3), ("x_stride", ctypes.c_int64), ("dx_stride", ctypes.c_int64)]


class dn_out_norm_shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "H", "d", "dtype", "act")] + [("eps", ctypes.c_float)] + [
        (n, ctypes.c_int64) for n in ("o_stride", "gate_stride", "dgate_stride")]


class dn_block_norm_shape(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("T", "D", "dtype", "stream_dtype", "post_norm")] + [
        (n, ctypes.c_float) for n in ("scale", "residual_scale", "eps")] + [(n, ctypes.c_int64) for n in ("x_stride", "residual_stride")]


_lib = None


def _library():
    """The C ABI of these operators through ctypes."""
    global _lib
    if _lib is None:
        lib = binding.load_library()
        vp, sz = ctypes.c_void_p, ctypes.c_size_t
        conv, out, block, vps = (ctypes.POINTER(t) for t in (dn_conv_shape, dn_out_norm_shape, dn_block_norm_shape, vp))
        for name, args in (
                ("deltanet_short_conv_fwd", [conv] + [vp] * 4 + [vps, vp, vp]),
                ("deltanet_short_conv_workspace_bytes", [conv, ctypes.POINTER(sz)]),
                ("deltanet_short_conv_bwd", [conv, vp, vp, vps] + [vp] * 8 + [sz, vp]),
                ("deltanet_out_norm_fwd", [out] + [vp] * 5),
                ("deltanet_out_norm_workspace_bytes", [out, ctypes.POINTER(sz)]),
                ("deltanet_out_norm_bwd", [out] + [vp] * 8 + [sz, vp]),
                ("deltanet_block_norm_fwd", [block] + [vp] * 7),
                ("deltanet_block_norm_workspace_bytes", [block, ctypes.POINTER(sz)]),
                ("deltanet_block_norm_bwd", [block] + [vp] * 11 + [sz, vp])):
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = ctypes.c_int, args
        _lib = lib
    return _lib


def _act(name: str) -> int:
    if name not in _ACTS:
        raise ValueError("act must be one of %s, got %r" % (sorted(_ACTS), name))
    return _ACTS[name]


def deltanet_short_conv_fwd(x, weight, bias=None, initial_state=None, *, splits: Optional[Sequence[int]] = None,
                            silu: Union[bool, Sequence[bool]] = True, cu_seqlens=None, cu_seqlens_host: Optional[Sequence[int]] = None,
                            output_final_state: bool = True, y=None, final_state=None, stream=None):
    """Causal convolution of every channel with its own weight [C, W] (W = 2, 3, 4), then SiLU where `silu` says so; returns (y, final_state or None).
    x [B, L, C], or packed [T, C] with cu_seqlens, may be a column block of a projection's output (rows apart).  splits: widths of up to three
    parts (q, k and v); y is then a tuple of contiguous tensors, and `silu` may hold a truth value for each.  States [N, W - 1, C]
    are the rows in front of a sequence, of x's type; final_state may be initial_state itself, as in generation.  cu_seqlens_host, the
    offsets on the host, is optional: given, it is validated."""
    return _call("short_conv_fwd", stream, x, weight, bias, initial_state, splits, silu, cu_seqlens, cu_seqlens_host, output_final_state, y, final_state)


def deltanet_short_conv_bwd(x, weight, dy, bias=None, initial_state=None, dfinal_state=None, *, splits: Optional[Sequence[int]] = None,
                            silu: Union[bool, Sequence[bool]] = True, cu_seqlens=None, cu_seqlens_host: Optional[Sequence[int]] = None,
                            dx=None, dweight=None, dbias=None, dinitial_state=None, workspace=None, stream=None):
    """Gradient of deltanet_short_conv_fwd for dy (a tuple with `splits`) and dfinal_state; returns (dx, dweight[fp32], dbias[fp32] or None, dinitial_state or None), the
    last where there is an initial_state.  dx may be a column block (rows apart) that the caller brings."""
    return _call("short_conv_bwd", stream, x, weight, dy, bias, initial_state, dfinal_state, splits, silu, cu_seqlens, cu_seqlens_host, dx, dweight,
                 dbias, dinitial_state, workspace)


def deltanet_out_norm_fwd(o, gate=None, weight=None, *, eps: float = 1e-6, act: str = "silu", y=None, stream=None) -> "torch.Tensor":
    """RMS norm of every head's output, times its weight [d] and act(gate); returns y.  o and gate [T, H, d] or [B, L, H, d] may be column blocks
    (rows apart); act is "silu" or "sigmoid"; without a gate there is no such factor."""
    return _call("out_norm_fwd", stream, o, gate, weight, eps, _act(act), y)


def deltanet_out_norm_bwd(o, dy, gate=None, weight=None, *, eps: float = 1e-6, act: str = "silu", d_o=None, dgate=None, dweight=None,
                          workspace=None, stream=None):
    """Gradient of deltanet_out_norm_fwd; returns (d_o, dgate or None, dweight[fp32] or None).  d_o may be dy itself; dgate may be a column
    block (rows apart) that the caller brings."""
    return _call("out_norm_bwd", stream, o, dy, gate, weight, eps, _act(act), d_o, dgate, dweight, workspace)


def deltanet_block_norm_fwd(x, residual=None, weight=None, *, gate=None, post_norm: bool = False, scale: float = 1.0, residual_scale: float = 1.0,
                            eps: float = 1e-6, y=None, h=None, stream=None) -> Tuple["torch.Tensor", "torch.Tensor"]:
    """Between two blocks: h = residual_scale * residual + scale * gate * x, with x normalised first if post_norm, and y, the RMS norm of h times
    weight; returns (y, h).  x and residual [T, D] or [B, L, D] may have rows apart; residual and h have x's type or are float32.  Without a residual (in front of the
    first block) h is the branch; x itself, where that is contiguous and nothing changes it."""
    return _call("block_norm_fwd", stream, x, residual, weight, gate, post_norm, scale, residual_scale, eps, y, h)


def deltanet_block_norm_bwd(dy, h, x=None, weight=None, dh=None, *, gate=None, post_norm: bool = False, scale: float = 1.0, residual_scale: float = 1.0,
                            eps: float = 1e-6, want_dresidual: bool = True, dx=None, dresidual=None, dweight=None, dgate=None,
                            workspace=None, stream=None):
    """Gradient of deltanet_block_norm_fwd for dy and dh, from the h that it returned and, with post_norm or a gate, x; returns (dx, dresidual or None, dweight[fp32] or
    None, dgate[fp32] or None).  Where dx and dresidual are the same numbers (nothing but a sum, one type) they are one tensor, unless the caller brings either."""
    return _call("block_norm_bwd", stream, dy, h, x, weight, dh, gate, post_norm, scale, residual_scale, eps, want_dresidual, dx, dresidual, dweight, dgate, workspace)
