"""Lengths, offsets, tables and positions that are parts of larger arrays, wherever these begin."""
import pytest
import torch

import paper_2406_06484_amd as dn
from tests import attention_reference as ref
from tests.attention_util import Batch, replays

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("skip", [1, 2, 3])
def test_a_part_of_a_batch(cache, skip):
    b = Batch([1, 5, 2, 9, 30], [40, 50, 30, 20, 77], 2, 64, "bf16", cache, 16, seed=skip)
    q, qh = b.rows(4)
    k, _ = b.rows(2)
    first = int(b.cu_host[skip])
    part = (b.table[skip:], b.kv_len[skip:])    # (tables of 6 columns: their rows begin inside 16-byte words)
    cu = (b.cu - first)[skip:]
    own = (part[0].clone(), part[1].clone())
    rope = ref.rope_table(80, 64).cuda()
    dn.deltanet_paged_append(k[first:], k[first:], b.k_pages, b.v_pages, *own, cu.clone(), **b.scales())
    pages = [t.clone() for t in (b.k_pages, b.v_pages)]
    want = (dn.deltanet_paged_norm_rope_append(q[first:], k[first:], k[first:], *pages, *own, cu.clone(), None, None, rope, **b.scales()),
            *dn.deltanet_paged_read(*pages, *own, cu.clone(), b.T - first, **b.scales()),
            dn.deltanet_paged_attn_fwd(q[first:], *pages, *own, cu.clone(), **b.scales()))
    dn.deltanet_paged_append(k[first:], k[first:], b.k_pages, b.v_pages, *part, cu, **b.scales())
    got = (dn.deltanet_paged_norm_rope_append(q[first:], k[first:], k[first:], b.k_pages, b.v_pages, *part, cu, None, None, rope, **b.scales()),
           *dn.deltanet_paged_read(b.k_pages, b.v_pages, *part, cu, b.T - first, **b.scales()),
           dn.deltanet_paged_attn_fwd(q[first:], b.k_pages, b.v_pages, *part, cu, **b.scales()))
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_positions():
    q, k = torch.randn(9, 4, 64, device="cuda"), torch.randn(9, 2, 64, device="cuda")
    pos, rope = torch.arange(20, dtype=torch.int32, device="cuda"), ref.rope_table(20, 64).cuda()
    for at in (1, 2, 7):
        part = pos[at:at + 9]
        for x, y in zip(dn.deltanet_qk_norm_rope_fwd(q, k, None, None, rope, part), dn.deltanet_qk_norm_rope_fwd(q, k, None, None, rope, part.clone())):
            assert torch.equal(x, y)
        for x, y in zip(dn.deltanet_qk_norm_rope_bwd(q, k, q, k, None, None, rope, part), dn.deltanet_qk_norm_rope_bwd(q, k, q, k, None, None, rope, part.clone())):
            assert x is y is None or torch.equal(x, y)


def test_graphs_and_another_stream_follow_the_arrays():
    b = Batch([1, 1, 40], [30, 200, 60], 2, 128, "bf16", "bf16", 16)
    q, _ = b.rows(4)
    lens = torch.cat([b.kv_len[:1], b.kv_len])
    o, ws = torch.empty_like(q), torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    call = lambda **kw: dn.deltanet_paged_attn_fwd(q, b.k_pages, b.v_pages, b.table, lens[1:], b.cu, max_q=40, **kw)  # noqa: E731
    replays(lambda: call(o=o, workspace=ws), [o], lambda: call())
    want = b.attend(q, max_q=40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(stream=side)
    side.synchronize()
    assert torch.equal(got, want)
