"""Sizes at the ends of the attention operators' 32-bit ranges, refused or taken by the C ABI before any device call (no GPU needed)."""
import ctypes

import pytest

from tests.test_attention_boundary_host import FAKE, SHAPE, _lib, cache, fwd, paged, pytestmark, qk_shape, rope  # noqa: F401

MOST = 1 << 30


@pytest.mark.parametrize("T", [MOST + 1, (1 << 31) - 4, (1 << 31) - 1])
def test_more_rows_than_positions_and_grids_have_room_for(T):
    _, lib = _lib()
    s, out = qk_shape(T=T, Hq=1, Hkv=1), ctypes.c_size_t(0)
    assert lib.deltanet_qk_norm_rope_workspace_bytes(s, out) == SHAPE
    assert fwd(s) == SHAPE
    assert lib.deltanet_qk_norm_rope_bwd(s, rope(), *[FAKE] * 13, 1 << 40, None) == SHAPE
    assert lib.deltanet_paged_read(paged(Hq=1, Hkv=1), cache(), FAKE, T, FAKE, FAKE, None) == SHAPE
    assert lib.deltanet_paged_append(paged(T=T, max_q=1, Hq=1, Hkv=1), FAKE, FAKE, cache(), None) == SHAPE


def test_the_largest_number_of_rows():
    _, lib = _lib()
    out = ctypes.c_size_t(0)
    assert lib.deltanet_qk_norm_rope_workspace_bytes(qk_shape(T=MOST, Hq=1, Hkv=1), out) == 0
    assert out.value == 512 * 2 * 64 * 4


@pytest.mark.parametrize("max_q,status", [((1 << 20) - 1, 0), (1 << 20, SHAPE)])
def test_fp32_chunks_of_more_tiles_than_a_launch_has_room_for(max_q, status):
    _, lib = _lib()
    s, out = paged(dtype=0, cache_dtype=0, T=1 << 20, Hq=64, max_q=max_q, q_stride=64 * 64), ctypes.c_size_t(0)
    assert lib.deltanet_paged_attn_workspace_bytes(s, 0, out) == status
    s.dtype = s.cache_dtype = 1
    assert lib.deltanet_paged_attn_workspace_bytes(s, 0, out) == 0


@pytest.mark.parametrize("field,value", [("Hq", 0), ("Hq", 1), ("Hq", 5), ("T", -1), ("max_q", 9), ("max_kv", 65)])
def test_every_paged_call_checks_the_heads_and_bounds(field, value):
    """also where it does not use them, as the header says"""
    _, lib = _lib()
    s = paged(**{field: value})
    assert lib.deltanet_paged_append(s, FAKE, FAKE, cache(), None) == SHAPE
    assert lib.deltanet_paged_read(s, cache(), FAKE, 8, FAKE, FAKE, None) == SHAPE
    assert lib.deltanet_paged_attn_workspace_bytes(s, 0, ctypes.c_size_t(0)) == SHAPE
