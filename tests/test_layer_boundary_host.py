"""Refusals of the layer operators' C ABI and of their Python calls, which need no GPU: validation comes before the first device call."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2406_06484_amd", "libdeltanet_hip.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built (run __graft_entry__.build())")

NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE, CUSEQLENS = -1, -2, -3, -4, -5, -6
FAKE, ODD = 0x1000, 0x1004   # never dereferenced
MOST = 1 << 30


def _lib():
    from paper_2406_06484_amd import layer
    return layer, layer._library()


def _set(s, base, kw):
    for k, v in {**base, **kw}.items():
        if isinstance(v, tuple):
            getattr(s, k)[:] = v
        else:
            setattr(s, k, v)
    return s


def conv(**kw):
    la, _ = _lib()
    return _set(la.dn_conv_shape(), dict(B=2, L=8, C=64, W=4, dtype=1, num_seqs=0, cu_seqlens=None, cu_seqlens_host=None, parts=2, width=(16, 48, 0), silu=(0, 1, 0),
                                         x_stride=64, dx_stride=64), kw)


def out(**kw):
    la, _ = _lib()
    return _set(la.dn_out_norm_shape(), dict(T=8, H=4, d=64, dtype=1, act=1, eps=1e-6, o_stride=256, gate_stride=256, dgate_stride=256), kw)


def block(**kw):
    la, _ = _lib()
    return _set(la.dn_block_norm_shape(), dict(T=8, D=64, dtype=1, stream_dtype=1, post_norm=0, scale=1.0, residual_scale=1.0, eps=1e-6, x_stride=64, residual_stride=64), kw)


def three(*p):
    return (ctypes.c_void_p * 3)(*p)


def conv_fwd(s, y=(FAKE, FAKE, None), **kw):
    _, lib = _lib()
    p = dict(x=FAKE, w=FAKE, b=FAKE, s0=FAKE, y=y, sT=FAKE)
    p.update(kw)
    return lib.deltanet_short_conv_fwd(s, p["x"], p["w"], p["b"], p["s0"], None if p["y"] is None else three(*p["y"]), p["sT"], None)


def conv_bwd(s, dy=(FAKE, FAKE, None), **kw):
    _, lib = _lib()
    p = dict(x=FAKE, w=FAKE, b=FAKE, s0=FAKE, dsT=FAKE, dx=FAKE, dw=FAKE, db=FAKE, ds0=FAKE, ws=FAKE, n=1 << 40)
    p.update(kw)
    return lib.deltanet_short_conv_bwd(s, p["x"], p["w"], None if dy is None else three(*dy), *(p[k] for k in ("b", "s0", "dsT", "dx", "dw", "db", "ds0", "ws", "n")), None)


@pytest.mark.parametrize("field,value,status", [
    ("B", -1, SHAPE), ("L", -1, SHAPE), ("L", MOST, SHAPE), ("C", 0, SHAPE), ("C", 72, SHAPE), ("W", 1, UNSUPPORTED), ("W", 5, UNSUPPORTED), ("dtype", 2, UNSUPPORTED), ("parts", 0, SHAPE),
    ("parts", 4, SHAPE), ("parts", 1, SHAPE), ("width", (20, 44, 0), ALIGN), ("width", (80, -16, 0), SHAPE), ("width", (64, 0, 0), SHAPE), ("x_stride", 56, SHAPE), ("x_stride", 65, ALIGN),
    ("x_stride", (1 << 31) + 8, SHAPE)])
def test_convolution_shapes(field, value, status):
    _, lib = _lib()
    s, n = conv(**{field: value}), ctypes.c_size_t(0)
    assert conv_fwd(s) == status and conv_bwd(s) == status
    assert lib.deltanet_short_conv_workspace_bytes(s, n) == status


def test_convolution_pointers_offsets_and_workspace():
    _, lib = _lib()
    assert lib.deltanet_short_conv_fwd(None, *[FAKE] * 4, three(FAKE), FAKE, None) == NULL
    for name in ("x", "w", "y"):
        assert conv_fwd(conv(), **{name: None}) == NULL, name
    assert conv_fwd(conv(), y=(FAKE, None, None)) == NULL and conv_fwd(conv(), y=(FAKE, ODD, None)) == ALIGN
    for name in ("x", "w", "b", "s0", "sT"):
        assert conv_fwd(conv(), **{name: ODD}) == ALIGN, name
    for name in ("x", "w", "dx"):
        assert conv_bwd(conv(), **{name: None}) == NULL, name
    assert conv_bwd(conv(), dy=None) == NULL and conv_bwd(conv(), dy=(None, FAKE, None)) == NULL and conv_bwd(conv(), dy=(FAKE, ODD, None)) == ALIGN
    for name in ("x", "w", "b", "s0", "dsT", "dx", "dw", "db", "ds0", "ws"):
        assert conv_bwd(conv(), **{name: ODD}) == ALIGN, name
    assert conv_bwd(conv(dx_stride=56)) == SHAPE and conv_bwd(conv(dx_stride=66)) == ALIGN
    large, n = conv(L=4096), ctypes.c_size_t(0)
    assert lib.deltanet_short_conv_workspace_bytes(large, n) == 0 and n.value > 0
    assert lib.deltanet_short_conv_workspace_bytes(large, None) == NULL
    assert conv_bwd(large, ws=None) == WORKSPACE and conv_bwd(large, n=n.value - 1) == WORKSPACE
    packed = dict(B=1, L=16, num_seqs=2, cu_seqlens=FAKE)
    assert conv_fwd(conv(**{**packed, "B": 2})) == SHAPE and conv_fwd(conv(**{**packed, "num_seqs": -1})) == SHAPE and conv_fwd(conv(**{**packed, "cu_seqlens": ODD})) == ALIGN
    for bad in ((1, 3, 16), (0, 5, 15), (0, 17, 16)):
        keep = (ctypes.c_int32 * 3)(*bad)
        assert conv_fwd(conv(**packed, cu_seqlens_host=ctypes.addressof(keep))) == CUSEQLENS
    assert lib.deltanet_short_conv_workspace_bytes(conv(B=1, L=MOST, width=(64, 0, 0), parts=1), n) == 0


@pytest.mark.parametrize("field,value,status", [("T", -1, SHAPE), ("T", MOST, SHAPE), ("H", 0, SHAPE), ("d", 96, UNSUPPORTED), ("dtype", 2, UNSUPPORTED), ("eps", -1.0, SHAPE),
                                                ("eps", float("nan"), SHAPE), ("eps", float("inf"), SHAPE), ("o_stride", 255, SHAPE), ("o_stride", 260, ALIGN), ("act", 0, UNSUPPORTED),
                                                ("act", 3, UNSUPPORTED), ("gate_stride", 128, SHAPE), ("gate_stride", 257, ALIGN)])
def test_output_norm_shapes(field, value, status):
    _, lib = _lib()
    s = out(**{field: value})
    assert lib.deltanet_out_norm_fwd(s, *[FAKE] * 4, None) == status
    assert lib.deltanet_out_norm_bwd(s, *[FAKE] * 8, 1 << 40, None) == status


def test_output_norm_pointers_and_workspace():
    _, lib = _lib()
    assert lib.deltanet_out_norm_fwd(None, *[FAKE] * 4, None) == NULL
    fwd = lambda i, v: lib.deltanet_out_norm_fwd(out(), *[v if k == i else FAKE for k in range(4)], None)  # noqa: E731
    bwd = lambda i, v: lib.deltanet_out_norm_bwd(out(), *[v if k == i else FAKE for k in range(8)], 1 << 40, None)  # noqa: E731
    assert [fwd(i, None) for i in (0, 3)] == [NULL] * 2 and [fwd(i, ODD) for i in range(4)] == [ALIGN] * 4
    assert [bwd(i, None) for i in (0, 1, 4, 5)] == [NULL] * 4 and [bwd(i, ODD) for i in range(8)] == [ALIGN] * 8
    assert lib.deltanet_out_norm_bwd(out(dgate_stride=128), *[FAKE] * 8, 1 << 40, None) == SHAPE
    s, n = out(T=4096), ctypes.c_size_t(0)
    assert lib.deltanet_out_norm_workspace_bytes(s, n) == 0 and n.value > 0 and lib.deltanet_out_norm_workspace_bytes(s, None) == NULL
    assert lib.deltanet_out_norm_bwd(s, *[FAKE] * 7, None, 1 << 40, None) == WORKSPACE and lib.deltanet_out_norm_bwd(s, *[FAKE] * 8, n.value - 1, None) == WORKSPACE


@pytest.mark.parametrize("field,value,status", [("T", -1, SHAPE), ("T", MOST + 1, SHAPE), ("D", 0, SHAPE), ("D", 60, UNSUPPORTED), ("D", 8200, UNSUPPORTED), ("dtype", 2, UNSUPPORTED),
                                                ("stream_dtype", 2, UNSUPPORTED), ("eps", -1.0, SHAPE), ("eps", float("nan"), SHAPE), ("scale", float("nan"), SHAPE), ("scale", float("inf"), SHAPE),
                                                ("residual_scale", float("inf"), SHAPE), ("x_stride", 56, SHAPE), ("x_stride", 65, ALIGN), ("residual_stride", 8, SHAPE), ("residual_stride", 66, ALIGN)])
def test_block_norm_shapes(field, value, status):
    _, lib = _lib()
    s = block(**{field: value})
    assert lib.deltanet_block_norm_fwd(s, *[FAKE] * 6, None) == status
    if field != "residual_stride":
        assert lib.deltanet_block_norm_bwd(s, *[FAKE] * 11, 1 << 40, None) == status
    assert lib.deltanet_block_norm_fwd(block(dtype=0, stream_dtype=1), *[FAKE] * 6, None) == UNSUPPORTED


def test_block_norm_pointers_and_workspace():
    _, lib = _lib()
    assert lib.deltanet_block_norm_fwd(None, *[FAKE] * 6, None) == NULL
    fwd = lambda i, v: lib.deltanet_block_norm_fwd(block(), *[v if k == i else FAKE for k in range(6)], None)  # noqa: E731
    bwd = lambda i, v, s=None: lib.deltanet_block_norm_bwd(s or block(), *[v if k == i else FAKE for k in range(11)], 1 << 40, None)  # noqa: E731
    assert [fwd(i, None) for i in (0, 4)] == [NULL] * 2 and [fwd(i, ODD) for i in range(6)] == [ALIGN] * 6
    assert [bwd(i, None) for i in (0, 2, 3)] == [NULL] * 3 and [bwd(i, ODD) for i in range(11)] == [ALIGN] * 11
    assert bwd(5, None) == NULL     # a gate's gradient without a gate
    assert bwd(3, None, block(post_norm=1)) == NULL
    s, n = block(T=4096), ctypes.c_size_t(0)
    assert lib.deltanet_block_norm_workspace_bytes(s, n) == 0 and n.value > 0 and lib.deltanet_block_norm_workspace_bytes(s, None) == NULL
    assert lib.deltanet_block_norm_bwd(s, *[FAKE] * 10, None, 1 << 40, None) == WORKSPACE and lib.deltanet_block_norm_bwd(s, *[FAKE] * 11, n.value - 1, None) == WORKSPACE


def test_the_calls_refuse_what_they_cannot_take():
    import torch

    import paper_2406_06484_amd as dn
    x, w = torch.zeros(2, 4, 16), torch.zeros(16, 4)
    with pytest.raises(ValueError, match="device tensor"):
        dn.deltanet_short_conv_fwd(x, w)
    with pytest.raises(ValueError, match="device tensor"):
        dn.deltanet_out_norm_fwd(torch.zeros(4, 2, 32))
    with pytest.raises(ValueError, match="device tensor"):
        dn.deltanet_block_norm_fwd(torch.zeros(4, 64))
    with pytest.raises(ValueError, match="act"):
        dn.deltanet_out_norm_fwd(torch.zeros(4, 2, 32), act="relu")
    with pytest.raises(TypeError):
        dn.deltanet_short_conv_fwd(torch.zeros(2, 4, 16, dtype=torch.float16), w)
    with pytest.raises(TypeError):
        dn.deltanet_block_norm_fwd([1.0])
