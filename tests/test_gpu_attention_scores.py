"""Scores of every size: far above and far below what the running maximum starts from, and so large that a score's last bit is more than the
exponential's range."""
import pytest
import torch

from tests import attention_reference as ref
from tests.attention_util import Batch, near

pytestmark = pytest.mark.gpu

FORMS = [("f32", "f32", 64), ("bf16", "bf16", 128), ("bf16", "bf16", 256), ("bf16", "fp8", 64), ("bf16", "fp8", 128)]
BATCHES = [([1, 4], [70, 300], 0), ([1], [5000], 0), ([1, 50, 130], [70, 300, 260], 0), ([150], [1700], 40), ([140, 140], [3000, 2500], 0)]


def _put(b, n, k):
    """gives sequence n the keys k (float64 [kv, Hkv, d])"""
    held, scale = ref.e4m3(k.float().double()) if b.cache == "fp8" else (k.to(b.k_pages.dtype).double(), None)
    p = torch.arange(b.kvs[n])
    ids = b.table_host[n].long()[p // b.page].cuda()
    pages = b.k_pages.float()       # (8-bit tensors have no indexed store)
    pages[ids, :, (p % b.page).cuda()] = held.float().cuda()
    b.k_pages.copy_(pages.to(b.k_pages.dtype))
    if scale is not None:
        scale = scale.float().double()
        b.k_scale[ids, :, (p % b.page).cuda()] = scale[..., 0].float().cuda()
        held = held * scale
    b.k[n] = held


def _seen(p, kv, window):
    return (max(0, p - window + 1) if window else 0), min(p + 1, kv)


@pytest.mark.parametrize("dtype,cache,d", FORMS)
@pytest.mark.parametrize("qs,kvs,window", BATCHES)
@pytest.mark.parametrize("size,sign", [(18, 1), (18, -1), (54, 1), (54, -1)])
def test_the_largest_score_takes_all(dtype, cache, d, qs, kvs, window, size, sign):
    """queries and keys along one axis: a score is a single product and equals another one or is 2^20 and more apart from it, so that the output is the mean
    of the largest ones' values, whatever the sign (and carries its own rounding alone)"""
    b = Batch(qs, kvs, 2, d, dtype, cache, 16, seed=size, junk=0.0)
    for n, kv in enumerate(kvs):
        k = torch.zeros(kv, 2, d, dtype=torch.float64)
        for h in range(2):
            at = torch.randperm(kv, generator=b.gen)
            k[:, h, 0] = sign * (1 + (at % 128) / 128.0) * torch.exp2(size + (at // 128 % 4).double())
        _put(b, n, k)
    q = torch.zeros(b.T, 4, d, dtype=torch.float64)
    q[..., 0] = 2.0 ** size
    o = b.attend(q.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda(), window=window, max_q=max(qs), max_kv=max(kvs)).double().cpu()
    for n, (m, kv) in enumerate(zip(qs, kvs)):
        for i in range(m):
            lo, hi = _seen(kv - m + i, kv, window)
            for h in range(4):
                k, v = b.k[n][lo:hi, h // 2, 0], b.v[n][lo:hi, h // 2]
                want = v[k == k.max()].mean(0)
                assert ((o[int(b.cu_host[n]) + i, h] - want).abs() <= ref.HALF["bf16"] * v.abs().max()).all(), (n, i, h)


@pytest.mark.parametrize("dtype,cache,d", FORMS)
@pytest.mark.parametrize("qs,kvs,window", BATCHES)
@pytest.mark.parametrize("size,sign", [(18, 1), (54, -1)])
def test_equal_scores_of_any_size_weigh_the_same(dtype, cache, d, qs, kvs, window, size, sign):
    b = Batch(qs, kvs, 2, d, dtype, cache, 16, seed=size, junk=0.0)
    for n, kv in enumerate(kvs):
        k = torch.zeros(kv, 2, d, dtype=torch.float64)
        k[..., 0] = sign * 1.25 * 2.0 ** size
        _put(b, n, k)
    q = torch.zeros(b.T, 4, d, dtype=torch.float64)
    q[..., 0] = 1.125 * 2.0 ** size
    o = b.attend(q.to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda(), window=window, max_q=max(qs), max_kv=max(kvs))
    flat = torch.zeros_like(q)      # (the reference on scores of zero: the same weights)
    b.check(o, flat, d ** -0.5, window, "equal")
