"""More tokens than a sequence's table has room for: those with a place keep it, the others are dropped, and nothing moves."""
import pytest
import torch

import paper_2406_06484_amd as dn
from tests import attention_reference as ref
from tests.attention_util import TYPES, Batch, near

pytestmark = pytest.mark.gpu

FORMS = [("f32", "f32", 64), ("bf16", "bf16", 128), ("bf16", "fp8", 64)]


def _full(dtype, cache, d, new, over, pages=3, seed=0):
    """one sequence whose last `over` of `new` tokens have no room in its `pages` pages of 16, and one with room to spare"""
    room = 16 * pages
    b = Batch([new, 2], [room, 20], 2, d, dtype, cache, 16, seed=seed, junk=0.25)
    b.table = b.table[:, :pages].contiguous()      # no spare column
    b.kv_len = torch.tensor([room + over, 20], dtype=torch.int32).cuda()
    return b, room


@pytest.mark.parametrize("dtype,cache,d", FORMS)
@pytest.mark.parametrize("new,over", [(1, 1), (5, 2), (4, 4), (3, 40), (20, 1)])
def test_appends_drop_what_has_no_room(dtype, cache, d, new, over):
    b, room = _full(dtype, cache, d, new, over, seed=new)
    k, kh = b.rows(2)
    dn.deltanet_paged_append(k, k, *b.tensors(), b.cu, **b.scales())
    cu = torch.tensor([0, room, room], dtype=torch.int32).cuda()
    b.kv_len = torch.tensor([room, 0], dtype=torch.int32).cuda()
    got, _ = dn.deltanet_paged_read(*b.tensors(), cu, room, dtype=TYPES[dtype], **b.scales())
    torch.cuda.synchronize()
    kept = max(new - over, 0)
    start = room + over - new
    fresh = kh[:kept]
    if cache == "fp8" and kept:
        values, scale = ref.e4m3(fresh)
        fresh = values * scale.double()
    want = torch.cat([b.k[0][:min(start, room)], fresh])
    if cache == "fp8":
        near(got, want, want.abs() * (2.0 ** -8 + 2.0 ** -22) + 1e-30, "kept")
    else:
        assert torch.equal(got.double().cpu(), want)


@pytest.mark.parametrize("dtype,cache,d", FORMS)
def test_positions_of_rotated_rows_do_not_move(dtype, cache, d):
    b, room = _full(dtype, cache, d, 6, 4)
    table = ref.rope_table(room + 8, d)
    q, qh = b.rows(4)
    k, kh = b.rows(2)
    got = dn.deltanet_paged_norm_rope_append(q, k, k, *b.tensors(), b.cu, None, None, table.cuda(), **b.scales())
    torch.cuda.synchronize()
    pos = torch.cat([torch.arange(room - 2, room + 4), torch.tensor([18, 19])])
    near(got, ref.norm_rope(qh, None, table, pos, 1e-6, False), ref.norm_rope_bound(qh, None, table, pos, 1e-6, False, dtype), "q")


@pytest.mark.parametrize("dtype,cache,d", FORMS)
def test_reading_past_the_table_gives_zeros(dtype, cache, d):
    b, room = _full(dtype, cache, d, 1, 3)
    cu = torch.tensor([0, 10, 12], dtype=torch.int32).cuda()
    got, _ = dn.deltanet_paged_read(*b.tensors(), cu, 12, dtype=TYPES[dtype], **b.scales())
    torch.cuda.synchronize()
    want = torch.cat([b.k[0][room - 7:], torch.zeros(3, 2, d, dtype=torch.float64), b.k[1][18:]])
    near(got, want, want.abs() * (2.0 ** -8 + 2.0 ** -22) + 1e-30, "read")


@pytest.mark.parametrize("dtype,cache,d", FORMS)
@pytest.mark.parametrize("new,over,pages,window", [(1, 1, 3, 0), (6, 2, 3, 0), (6, 2, 3, 9), (40, 5, 3, 0), (40, 5, 3, 13), (3, 30, 3, 8), (2, 1, 200, 0), (100, 60, 20, 33)])
def test_rows_attend_at_their_own_positions(dtype, cache, d, new, over, pages, window):
    b, room = _full(dtype, cache, d, new, over, pages, seed=new + window)
    q, qh = b.rows(4)
    o = b.attend(q, window=window)
    torch.cuda.synchronize()
    for n, before in ((0, room + over - new), (1, 18)):
        lo, m = int(b.cu_host[n]), b.qs[n]
        want, size, top = ref.attention(qh[lo:lo + m], b.k[n], b.v[n], before, d ** -0.5, window)
        near(o[lo:lo + m], want, ref.attention_bound(want, size, top, d, b.kvs[n], dtype), "seq %d" % n)
