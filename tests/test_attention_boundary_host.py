"""Refusals of the attention operators' C ABI, which need no GPU: validation comes before the first device call."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2406_06484_amd", "libdeltanet_hip.so")
pytestmark = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built (run __graft_entry__.build())")

NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = -1, -2, -3, -4, -5
FAKE, ODD = 0x1000, 0x1004   # never dereferenced


def _lib():
    from paper_2406_06484_amd import attention
    return attention, attention._library()


def _set(s, base, kw):
    for k, v in {**base, **kw}.items():
        setattr(s, k, v)
    return s


def qk_shape(**kw):
    at, _ = _lib()
    return _set(at.dn_qk_shape(), dict(T=8, Hq=4, Hkv=2, d=64, dtype=1, seq_len=8, q_stride=256, k_stride=128), kw)


def rope(**kw):
    at, _ = _lib()
    return _set(at.dn_rope(), dict(rot=64, interleaved=0, max_pos=16, eps=1e-6), kw)


def paged(**kw):
    at, _ = _lib()
    return _set(at.dn_paged_shape(), dict(num_seqs=2, T=8, Hq=4, Hkv=2, d=64, dtype=1, cache_dtype=1, page_size=16, num_pages=9, max_pages=4, max_q=8,
                                          max_kv=64, cu_q=FAKE, kv_len=FAKE, page_table=FAKE, q_stride=256, k_stride=128, v_stride=128), kw)


def cache(**kw):
    at, _ = _lib()
    return _set(at.dn_paged_cache(), dict(k_pages=FAKE, v_pages=FAKE, k_scale=None, v_scale=None), kw)


def fwd(s=None, r=None, ptrs=None):
    _, lib = _lib()
    p = dict(q=FAKE, k=FAKE, qw=FAKE, kw=FAKE, cs=FAKE, pos=FAKE, qo=FAKE, ko=FAKE)
    p.update(ptrs or {})
    return lib.deltanet_qk_norm_rope_fwd(s or qk_shape(), r or rope(), *p.values(), None)


@pytest.mark.parametrize("field,value,status", [
    ("T", -1, SHAPE), ("Hq", 0, SHAPE), ("Hkv", 3, SHAPE), ("Hkv", 0, SHAPE), ("Hkv", 8, SHAPE), ("d", 96, UNSUPPORTED), ("dtype", 2, UNSUPPORTED),
    ("q_stride", 255, SHAPE), ("q_stride", 260, ALIGN), ("k_stride", 64, SHAPE), ("T", 1 << 30, SHAPE)])
def test_norm_rope_shapes(field, value, status):
    assert fwd(qk_shape(**{field: value})) == status
    out = ctypes.c_size_t(0)
    _, lib = _lib()
    assert lib.deltanet_qk_norm_rope_workspace_bytes(qk_shape(**{field: value}), out) == status


@pytest.mark.parametrize("field,value,status", [("rot", -16, SHAPE), ("rot", 80, SHAPE), ("rot", 24, UNSUPPORTED), ("max_pos", 0, SHAPE), ("eps", -1.0, SHAPE),
                                                ("eps", float("nan"), SHAPE), ("eps", float("inf"), SHAPE)])
def test_rotations(field, value, status):
    assert fwd(r=rope(**{field: value})) == status
    _, lib = _lib()
    assert lib.deltanet_paged_norm_rope_append(paged(), rope(**{field: value}), *[FAKE] * 7, cache(), None) == status


def test_norm_rope_pointers():
    _, lib = _lib()
    assert lib.deltanet_qk_norm_rope_fwd(None, rope(), *[FAKE] * 8, None) == NULL
    assert lib.deltanet_qk_norm_rope_fwd(qk_shape(), None, *[FAKE] * 8, None) == NULL
    for name in ("q", "k", "qo", "ko", "cs"):
        assert fwd(ptrs={name: None}) == NULL, name
    for name in ("q", "k", "qw", "kw", "cs", "pos", "qo", "ko"):
        assert fwd(ptrs={name: ODD}) == ALIGN, name
    assert fwd(qk_shape(seq_len=0), ptrs=dict(pos=None)) == SHAPE
    bwd = lambda s, ws, n: lib.deltanet_qk_norm_rope_bwd(s, rope(), *[FAKE] * 12, ws, n, None)  # noqa: E731
    out = ctypes.c_size_t(0)
    assert lib.deltanet_qk_norm_rope_workspace_bytes(qk_shape(), out) == 0 and out.value > 0
    assert lib.deltanet_qk_norm_rope_workspace_bytes(qk_shape(), None) == NULL
    assert bwd(qk_shape(), None, 1 << 30) == WORKSPACE and bwd(qk_shape(), FAKE, out.value - 1) == WORKSPACE and bwd(qk_shape(), ODD, out.value) == ALIGN


@pytest.mark.parametrize("field,value,status", [
    ("T", -1, SHAPE), ("Hkv", 3, SHAPE), ("d", 32, UNSUPPORTED), ("d", 96, UNSUPPORTED), ("dtype", 0, UNSUPPORTED), ("cache_dtype", 0, UNSUPPORTED),
    ("cache_dtype", 3, UNSUPPORTED), ("page_size", 8, UNSUPPORTED), ("page_size", 48, UNSUPPORTED), ("page_size", 512, UNSUPPORTED), ("num_seqs", -1, SHAPE),
    ("num_seqs", 65536, SHAPE), ("max_q", 9, SHAPE), ("max_q", -1, SHAPE), ("max_kv", 65, SHAPE), ("max_kv", -1, SHAPE), ("num_pages", 0, SHAPE),
    ("num_pages", -1, SHAPE), ("max_pages", -1, SHAPE)])
def test_paged_shapes(field, value, status):
    _, lib = _lib()
    s, out = paged(**{field: value}), ctypes.c_size_t(0)
    assert lib.deltanet_paged_append(s, FAKE, FAKE, cache(), None) == status
    assert lib.deltanet_paged_norm_rope_append(s, rope(), *[FAKE] * 7, cache(), None) == status
    assert lib.deltanet_paged_read(s, cache(), FAKE, 8, FAKE, FAKE, None) == status
    assert lib.deltanet_paged_attn_workspace_bytes(s, 0, out) == status
    assert lib.deltanet_paged_attn_fwd(s, FAKE, cache(), 0.125, 0, FAKE, FAKE, 1 << 40, None) == status


def test_fp32_tensors_have_no_eight_bit_cache_and_other_head_sizes():
    _, lib = _lib()
    out = ctypes.c_size_t(0)
    for d, status in ((32, 0), (64, 0), (128, 0), (256, UNSUPPORTED)):
        assert lib.deltanet_paged_attn_workspace_bytes(paged(dtype=0, cache_dtype=0, d=d), 0, out) == status
    assert lib.deltanet_paged_attn_workspace_bytes(paged(dtype=0, cache_dtype=2), 0, out) == UNSUPPORTED
    for d in (64, 128, 256):
        assert lib.deltanet_paged_attn_workspace_bytes(paged(cache_dtype=2, d=d), 0, out) == 0


def test_paged_pointers_strides_and_workspace():
    _, lib = _lib()
    attn = lambda s, q=FAKE, c=None, scale=0.125, window=0, o=FAKE, ws=FAKE, n=1 << 40: lib.deltanet_paged_attn_fwd(  # noqa: E731
        s, q, c if c is not None else cache(), scale, window, o, ws, n, None)
    assert attn(paged(), q=None) == NULL and attn(paged(), o=None) == NULL
    assert attn(paged(), q=ODD) == ALIGN and attn(paged(), o=ODD) == ALIGN and attn(paged(), ws=ODD) == ALIGN
    for name in ("cu_q", "kv_len", "page_table"):
        assert attn(paged(**{name: None})) == NULL and attn(paged(**{name: ODD})) == ALIGN
    for name in ("k_pages", "v_pages"):
        assert attn(paged(), c=cache(**{name: None})) == NULL and attn(paged(), c=cache(**{name: ODD})) == ALIGN
    assert attn(paged(cache_dtype=2)) == NULL and attn(paged(cache_dtype=2), c=cache(k_scale=FAKE)) == NULL
    assert attn(paged(q_stride=128)) == SHAPE and attn(paged(q_stride=257)) == ALIGN
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert attn(paged(), scale=scale) == SHAPE
    assert attn(paged(), window=-1) == SHAPE
    long, out = paged(num_seqs=1, T=1, max_q=1, max_pages=4096, max_kv=65536), ctypes.c_size_t(0)
    assert lib.deltanet_paged_attn_workspace_bytes(long, 0, out) == 0 and out.value > 0
    assert attn(long, ws=None) == WORKSPACE and attn(long, n=out.value - 1) == WORKSPACE
    assert lib.deltanet_paged_attn_workspace_bytes(long, 0, None) == NULL
    for stride in ("k_stride", "v_stride"):
        assert lib.deltanet_paged_append(paged(**{stride: 64}), FAKE, FAKE, cache(), None) == SHAPE
        assert lib.deltanet_paged_append(paged(**{stride: 129}), FAKE, FAKE, cache(), None) == ALIGN
    assert lib.deltanet_paged_append(paged(), None, FAKE, cache(), None) == NULL
    assert lib.deltanet_paged_append(paged(), FAKE, FAKE, None, None) == NULL
    assert lib.deltanet_paged_read(paged(), cache(), FAKE, -1, FAKE, FAKE, None) == SHAPE
    assert lib.deltanet_paged_read(paged(), cache(), None, 8, FAKE, FAKE, None) == NULL
    assert lib.deltanet_paged_read(paged(), cache(), FAKE, 8, None, FAKE, None) == NULL
    assert lib.deltanet_paged_read(paged(), cache(), FAKE, 8, FAKE, ODD, None) == ALIGN


def test_the_binding_refuses_tensors_that_are_not_on_the_device():
    import torch

    import paper_2406_06484_amd as dn
    q, k = torch.zeros(4, 2, 64), torch.zeros(4, 2, 64)
    with pytest.raises(ValueError):
        dn.deltanet_qk_norm_rope_fwd(q, k)
    pages, i32 = torch.zeros(3, 2, 16, 64), dict(dtype=torch.int32)
    with pytest.raises(ValueError):
        dn.deltanet_paged_attn_fwd(q, pages, pages, torch.zeros(1, 2, **i32), torch.zeros(1, **i32), torch.zeros(2, **i32))
