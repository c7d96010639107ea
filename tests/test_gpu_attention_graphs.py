"""Captured serving steps: every replay writes its tokens, and follows lengths and tables that advance in place."""
import pytest
import torch

import paper_2406_06484_amd as dn
from tests import attention_reference as ref
from tests.attention_util import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,cache,d", [("f32", "f32", 64), ("bf16", "bf16", 128), ("bf16", "fp8", 64)])
def test_replays_write_the_cache_and_follow_the_lengths(dtype, cache, d):
    b = Batch([1, 1, 7], [30, 200, 40], 2, d, dtype, cache, 16, seed=d)
    b.table = torch.cat([b.table[:, :13], b.table[:, :1]], 1).contiguous()
    q, _ = b.rows(4)
    k, _ = b.rows(2)
    rope = ref.rope_table(256, d).cuda()
    tensors = [t for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale) if t is not None]
    q_out, o, ws = torch.empty_like(q), torch.empty_like(q), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def step():
        dn.deltanet_paged_norm_rope_append(q, k, k, *b.tensors(), b.cu, None, None, rope, **b.scales(), q_out=q_out)
        dn.deltanet_paged_attn_fwd(q_out, *b.tensors(), b.cu, **b.scales(), o=o, workspace=ws, max_q=7, max_kv=208)

    start = [t.clone() for t in tensors]

    def restore(lens, rows):
        b.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
        b.table.copy_(torch.tensor(rows, dtype=torch.int32) if not torch.is_tensor(rows) else rows)
        for t, s in zip(tensors, start):
            t.copy_(s)
        q_out.fill_(float("nan"))
        o.fill_(float("nan"))
        torch.cuda.synchronize()

    table = b.table.clone()
    swapped = table.clone()
    swapped[0, 1], swapped[2, 2] = table[2, 2], table[0, 1]     # two pages change hands
    batches = [([30, 200, 40], table), ([31, 201, 47], table), ([32, 208, 48], table), ([31, 199, 46], swapped), ([30, 200, 40], table)]
    want = []
    for lens, rows in batches:
        restore(lens, rows)
        step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in tensors + [q_out, o]])
    assert torch.isfinite(want[0][-1]).all()
    restore(*batches[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for (lens, rows), expected in zip(batches, want):
        restore(lens, rows)
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(tensors + [q_out, o], expected):
            bits = torch.uint8 if got.element_size() == 1 else torch.int16 if got.element_size() == 2 else torch.int32
            assert torch.equal(got.view(bits), w.view(bits))
        assert not torch.equal(tensors[0].view(torch.uint8), start[0].view(torch.uint8))
