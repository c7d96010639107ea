"""The bound for two-term probabilities tells them from ones that are rounded once, over contexts short enough for single roundings to show (on the CPU)."""
import pytest
import torch

from tests import attention_reference as ref
from tests.attention_roundings import bound, one_term


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("kv", [17, 129])
def test_one_term_is_out_of_bounds(d, kv):
    g = torch.Generator().manual_seed(kv)
    bf16 = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).double()  # noqa: E731
    q, k, v = bf16(4, 4, d), 0.25 * bf16(kv, 2, d), bf16(kv, 2, d)
    args = (q, k, v, kv - 4, d ** -0.5, 0)
    want, size, top = ref.attention(*args)
    most = bound(want, size, top, d, kv)
    assert ((want.to(torch.bfloat16).double() - want).abs() <= most).all()
    assert ((one_term(*args).to(torch.bfloat16).double() - want).abs() > most).any()
