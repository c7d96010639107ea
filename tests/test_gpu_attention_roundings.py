"""Where the attention rounds: sequences of few rows carry their probabilities as two bf16 terms, 8-bit chunks of many rows widen without a rounding."""
import pytest
import torch

from tests import attention_reference as ref
from tests.attention_roundings import bound
from tests.attention_util import Batch, near

pytestmark = pytest.mark.gpu

FORMS = [("bf16", "bf16", 64), ("bf16", "bf16", 128), ("bf16", "bf16", 256), ("bf16", "fp8", 64), ("bf16", "fp8", 128), ("bf16", "fp8", 256)]


@pytest.mark.parametrize("dtype,cache,d", FORMS)
@pytest.mark.parametrize("qs,kvs,window", [([1] * 6, [1, 2, 17, 64, 129, 700], 0), ([1], [4000], 0), ([3, 8, 1], [333, 90, 200], 0), ([1, 5], [600, 300], 77)])
def test_few_rows_carry_two_terms(dtype, cache, d, qs, kvs, window):
    b = Batch(qs, kvs, 2, d, dtype, cache, 16, seed=d + len(qs), k_size=0.25)
    q, qh = b.rows(8)
    o = b.attend(q, window=window, max_q=max(qs), max_kv=max(kvs))
    torch.cuda.synchronize()
    for n, (m, kv) in enumerate(zip(qs, kvs)):
        lo = int(b.cu_host[n])
        want, size, top = ref.attention(qh[lo:lo + m], b.k[n], b.v[n], kv - m, d ** -0.5, window)
        near(o[lo:lo + m], want, bound(want, size, top, d, kv), "seq %d" % n)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("qs,kvs,Hq,Hkv,window", [([128], [128], 4, 2, 0), ([257], [257], 1, 1, 0), ([300], [1000], 2, 1, 0), ([130, 130, 130], [130, 777, 4000], 4, 2, 0), ([64], [3333], 8, 2, 0),
                                                  ([300], [900], 2, 2, 1), ([300], [900], 2, 2, 40), ([512, 512], [512, 1500], 1, 1, 333), ([1000], [1001], 3, 1, 64)])
def test_equal_chunks_of_many_rows_over_eight_bit_pages(qs, kvs, Hq, Hkv, window, d):
    b = Batch(qs, kvs, Hkv, d, "bf16", "fp8", 32, seed=d + len(qs))
    q, qh = b.rows(Hq)
    o = b.attend(q, window=window, max_q=max(qs), max_kv=max(kvs))
    torch.cuda.synchronize()
    b.check(o, qh, d ** -0.5, window, "chunks")
