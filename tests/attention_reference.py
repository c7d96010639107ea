"""Plain statements in 64 bits of what the attention operators compute, and the bounds that their arithmetic keeps, on the CPU.  Every
function takes and returns float64 tensors; nothing of the library is used."""
import math

import torch

E32 = 2.0 ** -24                 # largest relative rounding of fp32
HALF = {"f32": E32, "bf16": 2.0 ** -8}   # largest relative rounding of an output: 2^-p with p significant bits
FP8_MAX = 448.0


def rope_table(max_pos, rot, theta=10000.0):
    """fp32 [max_pos, rot]: cosines, then sines"""
    half = rot // 2
    angle = torch.arange(max_pos, dtype=torch.float64)[:, None] * theta ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def pairs(rot, interleaved):
    """index lists (a, b) of the rotated pairs"""
    if interleaved:
        return list(range(0, rot, 2)), list(range(1, rot, 2))
    return list(range(rot // 2)), list(range(rot // 2, rot))


def rotate(z, table, pos, interleaved, back=False):
    if table is None:
        return z.clone()
    rot = table.shape[1]
    a, b = pairs(rot, interleaved)
    t = table.double()[pos.clamp(0, table.shape[0] - 1)]
    cos, sin = t[:, None, : rot // 2], t[:, None, rot // 2:]
    sin = -sin if back else sin
    y = z.clone()
    y[..., a] = z[..., a] * cos - z[..., b] * sin
    y[..., b] = z[..., b] * cos + z[..., a] * sin
    return y


def swapped(z, rot, interleaved):
    """every rotated element's partner in its place, other elements zero"""
    a, b = pairs(rot, interleaved)
    y = torch.zeros_like(z)
    y[..., a], y[..., b] = z[..., b], z[..., a]
    return y


def norm_rope(x, w, table, pos, eps, interleaved):
    z = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return rotate(z * w if w is not None else z, table, pos, interleaved)


def norm_rope_bound(x, w, table, pos, eps, interleaved, dtype):
    """how far y may be off: every sum of d squares is within d E32 of its value, each product and the reciprocal root within a few E32"""
    d = x.shape[-1]
    z = (x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * (w if w is not None else 1.0)).abs()
    spread = z + (swapped(z, table.shape[1], interleaved) if table is not None else 0.0)
    return HALF[dtype] * norm_rope(x, w, table, pos, eps, interleaved).abs() + (d + 16) * E32 * spread


def norm_rope_grad(x, w, table, pos, eps, interleaved, dy):
    """(dx, dw) by the formula"""
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xhat, dz = x * r, rotate(dy, table, pos, interleaved, back=True)
    g = dz * w if w is not None else dz
    return r * (g - xhat * (g * xhat).mean(-1, keepdim=True)), (dz * xhat).sum((0, 1))


def norm_rope_grad_bound(x, w, table, pos, eps, interleaved, dy, dtype):
    d, rows = x.shape[-1], x.shape[0] * x.shape[1]
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    xhat, dz = (x * r).abs(), dy.abs()
    dz = dz + (swapped(dz, table.shape[1], interleaved) if table is not None else 0.0)
    g = dz * w.abs() if w is not None else dz
    size = r * (g + xhat * (g * xhat).mean(-1, keepdim=True))
    dx, _ = norm_rope_grad(x, w, table, pos, eps, interleaved, dy)
    step = (2 * d + 32) * E32
    return HALF[dtype] * dx.abs() + step * size, (dz * xhat).sum((0, 1)) * (step + rows * E32)


def e4m3(x):
    """(numbers that an 8-bit row holds, its factor) of every row of fp32 values: the factor is fp32, and so is the quotient that is
    rounded to the nearest number with four significant bits, ties to even, least step 2^-9"""
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.where(top < 2.0 ** -100, 0.0, top / FP8_MAX).float()
    y = torch.where(scale > 0, x.float() / torch.where(scale > 0, scale, 1.0), 0.0).double()
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, scale.double()


def attention(q, k, v, before, scale, window):
    """q [m, Hq, d] at positions before .., k and v [kv, Hkv, d]: (o, attention of |v|, largest |score| bound); rows that see nothing are 0"""
    m, Hq, d = q.shape
    kv, Hkv = k.shape[:2]
    o, size, top = torch.zeros(m, Hq, d, dtype=torch.float64), torch.zeros(m, Hq, d, dtype=torch.float64), torch.zeros(m, Hq, 1, dtype=torch.float64)
    for i in range(m):
        p = before + i
        lo, hi = (max(0, p - window + 1) if window else 0), min(p + 1, kv)
        if hi <= lo:
            continue
        for h in range(Hq):
            kk, vv = k[lo:hi, h // (Hq // Hkv)], v[lo:hi, h // (Hq // Hkv)]
            w = torch.softmax(scale * (kk @ q[i, h]), 0)
            o[i, h], size[i, h] = w @ vv, w @ vv.abs()
            top[i, h] = scale * (kk.abs() @ q[i, h].abs()).max()
    return o, size, top


def attention_bound(o, size, top, d, kv, dtype):
    """Scores are sums of d products in fp32 ((d + 8) E32 of the sum of their magnitudes, and as much again for the scale and the running
    maximum's rounding); a probability's relative error is the score's, twice (it is in the sum below too), and a few E32 for the
    exponential and the joins; sums run over kv keys; in bf16 each probability is rounded once more, and the output."""
    err = 2 * (2 * (d + 8) * E32 * top + 16 * E32) + (kv + 16) * 2 * E32
    return HALF[dtype] * o.abs() + (err + (HALF["bf16"] if dtype == "bf16" else 0.0)) * size
