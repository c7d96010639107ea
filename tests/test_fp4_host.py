"""The statement of a 4-bit row on hand-made rows, and what the C ABI says of 4-bit pages (no GPU needed)."""
import ctypes

import torch

from tests import fp4_reference as f4
from tests.test_attention_boundary_host import FAKE, NULL, UNSUPPORTED, _lib, cache, paged, pytestmark, rope  # noqa: F401


def test_numbers_ties_and_factors():
    row = torch.zeros(32, dtype=torch.float64)
    row[:10] = torch.tensor([6.0, -5.0, 5.0001, 3.5, 2.5, 1.75, -1.25, 0.75, 0.25, -0.2])
    codes, factors = f4.quantise(row)
    assert factors.tolist() == [127] and codes[:10].tolist() == [7, 14, 7, 6, 4, 4, 10, 2, 0, 8]
    for top, byte in ((6.0, 127), (6.0001, 128), (12.0, 128), (3.0, 126), (3.1, 127), (2.0 ** -100, 25), (2.0 ** -101, 127), (3.3895e38, 253), (float("inf"), 255), (float("nan"), 255)):
        row = torch.zeros(64, dtype=torch.float64)
        row[40] = top
        assert f4.quantise(row)[1].tolist() == [127, byte], top


def test_values_lie_within_half_a_step_of_what_they_stand_for():
    x = torch.randn(50, 64, generator=torch.Generator().manual_seed(0), dtype=torch.float64)
    codes, factors = f4.quantise(x)
    v, s = f4.values(codes, factors), torch.exp2(factors.double() - 127).repeat_interleave(32, -1)
    assert ((v - x).abs() <= torch.where(x.abs() <= 2 * s, 0.25, torch.where(x.abs() <= 4 * s, 0.5, 1.0)) * s).all()
    assert torch.equal(f4.unpacked(f4.packed(codes)), codes)


def test_what_the_calls_say_of_four_bits():
    _, lib = _lib()
    n = ctypes.c_size_t(0)
    full = dict(k_scale=FAKE, v_scale=FAKE)
    for d, status in ((32, UNSUPPORTED), (64, 0), (128, 0), (256, 0)):
        assert lib.deltanet_paged_attn_workspace_bytes(paged(cache_dtype=4, d=d), 0, n) == status
    assert lib.deltanet_paged_attn_workspace_bytes(paged(cache_dtype=4, dtype=0), 0, n) == UNSUPPORTED
    assert lib.deltanet_paged_attn_workspace_bytes(paged(cache_dtype=5), 0, n) == UNSUPPORTED
    for missing in ("k_scale", "v_scale", "k_pages"):
        c = cache(**{**full, missing: None})
        assert lib.deltanet_paged_append(paged(cache_dtype=4), FAKE, FAKE, c, None) == NULL
        assert lib.deltanet_paged_norm_rope_append(paged(cache_dtype=4), rope(), *[FAKE] * 7, c, None) == NULL
        assert lib.deltanet_paged_read(paged(cache_dtype=4), c, FAKE, 8, FAKE, FAKE, None) == NULL
        assert lib.deltanet_paged_attn_fwd(paged(cache_dtype=4), FAKE, c, 0.125, 0, FAKE, FAKE, 1 << 40, None) == NULL


def test_the_tensors_of_a_cache():
    import pytest

    import paper_2406_06484_amd as dn
    k, v, ks, vs = dn.deltanet_paged_cache(3, 16, 2, 128, torch.float4_e2m1fn_x2, device="cpu")
    assert k.shape == v.shape == (3, 2, 16, 64) and ks.shape == vs.shape == (3, 2, 16, 4) and ks.dtype == torch.float8_e8m0fnu
    with pytest.raises(ValueError):
        dn.deltanet_paged_cache(3, 16, 2, 80, torch.float4_e2m1fn_x2, device="cpu")
