"""The 64-bit statements of the layer operators: their gradients against central differences, on the CPU."""
import pytest
import torch

from tests import layer_reference as ref

EPS = 1e-3


def differences(f, t, step=1e-5):
    """gradient of the number f() with respect to t by central differences"""
    g = torch.zeros_like(t)
    flat, out = t.view(-1), g.view(-1)
    for i in range(flat.numel()):
        was = float(flat[i])
        flat[i] = was + step
        up = float(f())
        flat[i] = was - step
        out[i] = (up - float(f())) / (2 * step)
        flat[i] = was
    return g


def close(a, b):
    assert (a - b).abs().max() <= 1e-7 * (1 + b.abs().max()), (a - b).abs().max()


@pytest.fixture
def rand():
    g = torch.Generator().manual_seed(3)
    return lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)


@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("lens", [[5], [1, 0, 2, 4]])
def test_convolution(rand, W, lens):
    C, T, N = 3, sum(lens), len(lens)
    x, w, b, s = rand(T, C), rand(C, W), rand(C), rand(N, W - 1, C)
    on, dy, ds = torch.tensor([True, False, True]), rand(T, C), rand(N, W - 1, C)

    def total():
        (y, _), last = ref.conv(x, w, b, s, lens, on, "f32")
        return (y * dy).sum() + (last * ds).sum()
    grads = ref.conv_grad(x, w, b, s, lens, on, dy, ds, "f32")
    for (g, _), t in zip(grads, (x, w, b, s)):
        close(g, differences(total, t))


@pytest.mark.parametrize("kind", ["silu", "sigmoid", None])
def test_output_norm(rand, kind):
    o, g, w, dy = rand(3, 2, 4), rand(3, 2, 4) if kind else None, rand(4), rand(3, 2, 4)
    f = lambda: (ref.out_norm(o, g, w, EPS, kind, "f32")[0] * dy).sum()  # noqa: E731
    grads = ref.out_norm_grad(o, g, w, EPS, kind, dy, "f32")
    for got, t in zip(grads, (o, g, w)):
        if t is not None:
            close(got[0], differences(f, t))


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gated", [False, True])
def test_block_norm(rand, post, gated):
    x, res, w, u, dy, dh = rand(3, 5), rand(3, 5), rand(5), rand(5) if gated else None, rand(3, 5), rand(3, 5)

    def total():
        (y, _), (h, _) = ref.block_norm(x, res, w, u, post, 0.7, 0.9, EPS, "f32", "f32")
        return (y * dy).sum() + (h * dh).sum()
    h = ref.block_norm(x, res, w, u, post, 0.7, 0.9, EPS, "f32", "f32")[1][0]
    grads = ref.block_norm_grad(dy, dh, h, x, w, u, post, 0.7, 0.9, EPS, "f32", "f32")
    for (g, _), t in zip(grads, (x, res, w, u)):
        if t is not None:
            close(g, differences(total, t))
