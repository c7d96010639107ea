"""Batches without a new token over contexts that are there."""
import pytest
import torch

from tests.attention_util import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,cache,d", [("f32", "f32", 64), ("bf16", "bf16", 128), ("bf16", "fp8", 64)])
@pytest.mark.parametrize("kvs", [[9], [5000], [40000, 3]])
def test_a_bound_of_no_tokens(dtype, cache, d, kvs):
    """rows that lie in no sequence become zero, whatever the contexts' length"""
    b = Batch([0] * len(kvs), kvs, 1, d, dtype, cache, 64)
    q, _ = b.rows(4, rows=3)
    o = b.attend(q, max_q=0, max_kv=max(kvs), o=torch.full_like(q, float("nan")))
    assert torch.equal(o, torch.zeros_like(o))


@pytest.mark.parametrize("dtype,d", [("f32", 64), ("bf16", 128)])
@pytest.mark.parametrize("rows", [3, 50])
def test_no_sequences_and_a_wide_table(dtype, d, rows):
    b = Batch([], [], 1, d, dtype, dtype, 64)
    b.table = torch.empty(0, 500, dtype=torch.int32, device="cuda")
    q, _ = b.rows(4, rows=rows)
    o = b.attend(q, o=torch.full_like(q, float("nan")))
    assert torch.equal(o, torch.zeros_like(o))
