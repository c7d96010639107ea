"""The example's hybrid model against its statement, every layer from the model's own input to it: DeltaNet layers by the oracle, attention layers in 64 bits."""
import numpy as np
import pytest
import torch

import example_hybrid
import oracle
from tests import attention_reference as ref

pytestmark = pytest.mark.gpu


def _bf16(x):
    return x.to(torch.bfloat16).double()


def _statement(model, layers, x):
    """the output of `layers` for one whole sequence x [n, width] (float64, host); operands rounded to bf16 where the model's tensors are"""
    H, Hkv, d, n = model.H, model.Hkv, model.d, x.shape[0]
    pos = torch.arange(n)
    for layer in layers:
        w_in, w_out = (layer[k].double().cpu() for k in ("w_in", "w_out"))
        h = _bf16(x / torch.sqrt((x * x).mean(-1, keepdim=True) + torch.finfo(torch.float32).eps))
        row = _bf16(h @ w_in)
        if layer["kind"] == "delta":
            q, k, v = (t.reshape(1, n, H, d).numpy().astype(np.float32) for t in row[:, :3 * H * d].split(H * d, 1))
            o, _ = oracle.fused_fwd(q, k, v, row[:, 3 * H * d:].reshape(1, n, H).numpy().astype(np.float32), None)
            o = torch.from_numpy(np.asarray(o, dtype=np.float64)).reshape(n, H, d)
        else:
            q, k, v = (t.unflatten(1, (-1, d)) for t in row.split([H * d, Hkv * d, Hkv * d], 1))
            rope = model.rope.cpu()
            q = _bf16(ref.norm_rope(q, layer["q_weight"].double().cpu(), rope, pos, 1e-6, False))
            k = ref.norm_rope(k, layer["k_weight"].double().cpu(), rope, pos, 1e-6, False)
            (kq, ks), (vq, vs) = ref.e4m3(k.float().double()), ref.e4m3(v)
            o = ref.attention(q, kq * ks, vq * vs, 0, d ** -0.5, model.window)[0]
        x = _bf16(x + _bf16(_bf16(o).reshape(n, H * d) @ w_out))
    return x


def _served(model, x, steps):
    """the sequences' outputs (float64, host), served in the given steps"""
    at, out = [0] * len(x), [[] for _ in x]
    for new in steps:
        y = model.step(torch.cat([x[n][a:a + m] for n, (a, m) in enumerate(zip(at, new))]).cuda(), new)
        for n, part in enumerate(y.split(new)):
            out[n].append(part)
        at = [a + m for a, m in zip(at, new)]
    assert at == [len(t) for t in x]
    return [torch.cat(parts).double().cpu() for parts in out]


@pytest.mark.parametrize("layers,heads,head_size,window", [(2, 2, 64, 20), (4, 4, 64, 0), (2, 2, 128, 9)])
def test_chunks_and_single_tokens_compute_every_layer(layers, heads, head_size, window):
    """An attention layer's output differs by roundings to bf16 that a last bit of fp32 tips over, 2^-8 of an element each, and by those of its probabilities, 2^-8 of the
    layer's part of the output: 2^-7 together.  A DeltaNet layer's part is held to what the layer's own tests allow, 2e-2."""
    total, steps = [75, 34, 3], [[40, 31, 0], [33, 1, 1], [1, 1, 1], [1, 1, 1]]
    g = torch.Generator().manual_seed(3)
    x = [torch.randn(n, heads * head_size, generator=g).to(torch.bfloat16) for n in total]
    inputs = [t.double() for t in x]
    for upto in range(1, layers + 1):
        model = example_hybrid.Hybrid(layers, heads, head_size, window, len(total), max(total))
        layer = model.layers[upto - 1]
        model.layers = model.layers[:upto]
        outputs = _served(model, x, steps)
        for n, (a, got) in enumerate(zip(inputs, outputs)):
            want = _statement(model, [layer], a)
            off = float((got - want).norm())
            most = 2e-2 * float((want - a).norm()) if layer["kind"] == "delta" else 2.0 ** -7 * float(want.norm())
            print("layer", upto, layer["kind"], "sequence", n, "difference / bound", off / most, flush=True)
            assert off <= most
        inputs = outputs
