"""Bounds for the attention of few rows, whose probabilities are carried as two bf16 terms."""
import torch

from tests import attention_reference as ref


def bound(want, size, top, d, kv):
    """ref.attention_bound with probabilities of two bf16 terms: what the second one leaves of the first one's rounding is 2^-8 of it, so 2^-16 in all"""
    return ref.attention_bound(want, size, top, d, kv, "f32") + (ref.HALF["bf16"] - ref.HALF["f32"]) * want.abs() + 2.0 ** -16 * size


def one_term(q, k, v, before, scale, window):
    """the same attention with probabilities rounded to bf16 once, relative to the row's largest"""
    o = torch.zeros_like(q)
    for i in range(q.shape[0]):
        lo, hi = (max(0, before + i - window + 1) if window else 0), before + i + 1
        for h in range(q.shape[1]):
            g = h // (q.shape[1] // k.shape[1])
            s = scale * (k[lo:hi, g] @ q[i, h])
            p = torch.exp(s - s.max())
            o[i, h] = p.to(torch.bfloat16).double() @ v[lo:hi, g] / p.sum()
    return o
