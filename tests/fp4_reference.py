"""Rows of a 4-bit cache in 64 bits on the CPU: groups of 32 e2m1 numbers (two significant bits, exponents 0 to 2, a half and zero below one) over a factor that is a power of two."""
import torch

from tests.attention_util import Batch

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
GROUP = 32


def quantise(x):
    """x [.., d] float64: (codes [.., d] of 0 to 15, bytes of the factors [.., d / 32]), by the distances to all numbers there are"""
    g = x.unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1, keepdim=True)
    bad = ~torch.isfinite(g).all(-1, keepdim=True)
    none = top < 2.0 ** -100
    plain = bad | none
    e = torch.zeros_like(top)
    safe = torch.where(plain, 1.0, top)
    # the least e with 6 2^e >= top, from its neighbourhood
    e = torch.floor(torch.log2(safe / 6)) - 1
    for _ in range(4):
        e = torch.where(6 * torch.exp2(e) < safe, e + 1, e)
    s = torch.exp2(e)
    q = torch.where(plain, 0.0, torch.nan_to_num(g).clamp(-1.5 * 2.0 ** 127, 1.5 * 2.0 ** 127) / s)     # (four times the largest factor is past bf16's range)
    away = (q.abs()[..., None] - LEVELS).abs()
    near = away == away.amin(-1, keepdim=True)
    even = near & (torch.arange(8) % 2 == 0)
    code = torch.where(near.sum(-1) > 1, even.int().argmax(-1), near.int().argmax(-1))
    code = torch.where(none, 0, code + 8 * torch.signbit(g).int())
    byte = torch.where(bad, 255, torch.where(none, 127, (e + 127).int()))
    return code.flatten(-2).int(), byte[..., 0].int()


def values(codes, factors):
    v = LEVELS[codes & 7] * torch.where(codes >= 8, -1.0, 1.0)
    f = torch.where(factors == 255, torch.tensor(float("nan"), dtype=torch.float64), torch.exp2(factors.double() - 127))
    return (v.unflatten(-1, (-1, GROUP)) * f[..., None]).flatten(-2)


def packed(codes):
    """two codes a byte, the first in the low half"""
    return (codes[..., 0::2] | codes[..., 1::2] << 4).to(torch.uint8)


def unpacked(b):
    b = b.int()
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


class Batch4(Batch):
    """A batch over a 4-bit cache: places that no context has hold NaN factors over the largest numbers."""

    def __init__(self, qs, kvs, Hkv, d, **kw):
        super().__init__(qs, kvs, Hkv, d, **kw)
        for which, held in (("k", self.k), ("v", self.v)):
            codes, factors = quantise(getattr(self, which + "_pages").double().cpu())
            codes = torch.where((factors == 255).repeat_interleave(GROUP, -1), 15, codes)
            setattr(self, which + "_pages", packed(codes).cuda().view(torch.float4_e2m1fn_x2))
            setattr(self, which + "_scale", factors.to(torch.uint8).cuda().view(torch.float8_e8m0fnu))
            for n, x in enumerate(held):
                held[n] = values(*quantise(x)) if x.numel() else x
        self.cache = "fp4"

    def raw(self, which):
        """(codes, factors) of the pages, on the host"""
        return unpacked(getattr(self, which + "_pages").view(torch.uint8).cpu()), getattr(self, which + "_scale").view(torch.uint8).cpu().int()
