"""The statements that the attention operators' GPU tests are held to, checked on the CPU: the gradient formula against differences, the
8-bit rounding against torch's conversion, and special cases of the attention."""
import math

import pytest
import torch

from tests import attention_reference as ref


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot,weight", [(16, True), (32, True), (32, False), (0, True)])
def test_gradient_formula_against_differences(rot, weight, interleaved):
    g = torch.Generator().manual_seed(3)
    x, dy = (torch.randn(3, 2, 32, generator=g, dtype=torch.float64) for _ in range(2))
    w = 1 + 0.3 * torch.randn(32, generator=g, dtype=torch.float64) if weight else None
    pos, table = torch.tensor([0, 7, 19]), ref.rope_table(20, rot) if rot else None
    f = lambda x, w: float((ref.norm_rope(x, w, table, pos, 1e-3, interleaved) * dy).sum())  # noqa: E731
    dx, dw = ref.norm_rope_grad(x, w, table, pos, 1e-3, interleaved, dy)
    for _ in range(4):
        u = torch.randn(x.shape, generator=g, dtype=torch.float64)
        assert (f(x + 1e-5 * u, w) - f(x - 1e-5 * u, w)) / 2e-5 == pytest.approx(float((dx * u).sum()), rel=1e-7, abs=1e-8)
        if weight:
            u = torch.randn(32, generator=g, dtype=torch.float64)
            assert (f(x, w + 1e-5 * u) - f(x, w - 1e-5 * u)) / 2e-5 == pytest.approx(float((dw * u).sum()), rel=1e-7, abs=1e-8)


def test_rotation_keeps_lengths_and_depends_on_distances():
    g = torch.Generator().manual_seed(4)
    q, k = (torch.randn(1, 1, 64, generator=g, dtype=torch.float64) for _ in range(2))
    table = ref.rope_table(50, 64).double()
    dots = []
    for p in (0, 3, 30):
        a, b = (ref.rotate(t, table, torch.tensor([at]), False) for t, at in ((q, p + 5), (k, p)))
        assert float(a.norm()) == pytest.approx(float(q.norm()), rel=1e-6)
        dots.append(float((a * b).sum()))
    assert dots[0] == pytest.approx(dots[1], abs=1e-5) and dots[0] == pytest.approx(dots[2], abs=1e-5)


def test_eight_bit_rounding_is_torchs():
    x = torch.cat([torch.linspace(-448, 448, 4001, dtype=torch.float64), torch.tensor([448.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 17.0, 19.0])])
    values, scale = ref.e4m3(x[None])
    assert float(scale) == 1.0
    assert torch.equal(values[0], x.float().to(torch.float8_e4m3fn).double())
    values, scale = ref.e4m3(torch.zeros(2, 8, dtype=torch.float64))
    assert not values.any() and not scale.any()


def test_attention_of_one_key_is_its_value_and_windows_hide():
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn(4, 2, 16, generator=g, dtype=torch.float64) for _ in range(3))
    o, _, _ = ref.attention(q, k, v, 0, 0.25, 1)
    assert torch.allclose(o, v)
    o, _, _ = ref.attention(q, k, v, -2, 0.25, 0)     # two rows in front of the context
    assert not o[:2].any() and torch.allclose(o[2], v[0])
    long, _, _ = ref.attention(q, k, v, 0, 0.25, 100)
    assert torch.allclose(long, ref.attention(q, k, v, 0, 0.25, 0)[0])
    assert not math.isclose(float(long[3, 0, 0]), float(ref.attention(q, k, v, 0, 0.25, 2)[0][3, 0, 0]))
