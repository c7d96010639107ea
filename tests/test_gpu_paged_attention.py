"""Attention of new tokens over the paged cache against its statement in 64 bits; every place of the cache outside the contexts holds NaN."""
import pytest
import torch

import paper_2406_06484_amd as dn
from tests import attention_reference as ref
from tests.attention_util import Batch, near, replays

pytestmark = pytest.mark.gpu

FORMS = [("f32", "f32", 32), ("f32", "f32", 64), ("f32", "f32", 128), ("bf16", "bf16", 64), ("bf16", "bf16", 128), ("bf16", "bf16", 256), ("bf16", "fp8", 64),
         ("bf16", "fp8", 128), ("bf16", "fp8", 256)]


def _run(b, Hq, label, window=0, scale=None, **kw):
    q, qh = b.rows(Hq)
    o = b.attend(q, window=window, scale=scale, **kw)
    torch.cuda.synchronize()
    b.check(o, qh, scale or b.d ** -0.5, window, label)
    return q, qh, o


@pytest.mark.parametrize("dtype,cache,d", FORMS)
@pytest.mark.parametrize("page", [16, 64])
def test_single_tokens(dtype, cache, d, page):
    b = Batch([1] * 8, [1, 2, 15, 16, 17, 64, 129, 700], 2, d, dtype, cache, page, seed=d)
    _run(b, 6, "single", max_q=1, max_kv=700)


@pytest.mark.parametrize("dtype,cache,d", FORMS)
def test_chunks_of_every_size(dtype, cache, d):
    b = Batch([1, 3, 20, 0, 70, 129], [400, 3, 33, 90, 71, 300], 1, d, dtype, cache, 16, seed=d + 1)
    _run(b, 3, "chunks")


@pytest.mark.parametrize("dtype,cache,d", [("f32", "f32", 64), ("bf16", "bf16", 128), ("bf16", "fp8", 64), ("bf16", "bf16", 256)])
@pytest.mark.parametrize("window", [1, 5, 16, 33, 100])
def test_windows(dtype, cache, d, window):
    b = Batch([1, 40, 150, 7], [333, 40, 260, 60], 2, d, dtype, cache, 16, seed=window)
    _run(b, 4, "window %d" % window, window=window)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (16, 16), (5, 1), (12, 3), (32, 2), (40, 1)])
def test_shared_heads(Hq, Hkv):
    b = Batch([1, 2, 50], [65, 40, 130], Hkv, 64, "bf16", "bf16", 32, seed=Hq)
    _run(b, Hq, "%d of %d" % (Hq, Hkv))


@pytest.mark.parametrize("q", [1, 2, 17, 64])
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_long_contexts_are_split_and_joined(q, cache):
    b = Batch([q, 1], [3001, 5], 1, 128, "bf16", cache, 256, seed=q)
    _run(b, 2, "long", max_kv=3001)
    _run(b, 2, "long, loose bounds")


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_page_sizes(page):
    b = Batch([5, 1, 90], [page, page + 1, 2 * page + 89], 2, 128, "bf16", "fp8", page, seed=page)
    _run(b, 2, "page %d" % page)


def test_rows_in_front_of_their_context_are_zero():
    for dtype, cache, d in (("f32", "f32", 64), ("bf16", "bf16", 128), ("bf16", "fp8", 256)):
        b = Batch([6, 200, 3], [2, 40, 0], 1, d, dtype, cache, 16, seed=3)
        _, _, o = _run(b, 2, "short contexts")
        assert not o[:4].any() and not o[6:6 + 160].any() and not o[-3:].any()


def test_rows_past_the_last_sequence_are_zero():
    for kv in (20, 2000):
        b = Batch([1, 2], [kv, 9], 2, 128, "bf16", "bf16", 16)
        q, qh = b.rows(4, rows=b.T + 5)
        o = b.attend(q, o=torch.full_like(q, float("nan")))
        torch.cuda.synchronize()
        b.check(o, qh, 128 ** -0.5, 0, "padded")
        assert not o[b.T:].any()


def test_nothing_at_all():
    b = Batch([], [], 1, 64)
    q, _ = b.rows(2, rows=3)
    assert not b.attend(q).any()
    q, _ = b.rows(2, rows=0)
    assert b.attend(q).shape == (0, 2, 64)


def test_sharp_and_flat_scores():
    """one key far above the others, scores in the hundreds, and all scores equal"""
    b = Batch([3, 60], [200, 300], 1, 64, "bf16", "bf16", 16, k_size=30.0)
    _run(b, 2, "sharp", scale=1.0)
    b = Batch([3, 60], [200, 300], 1, 64, "bf16", "bf16", 16, k_size=0.0)
    _run(b, 2, "flat")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("qs,kvs,Hq,Hkv,window", [([128], [128], 4, 2, 0), ([257], [257], 1, 1, 0), ([300], [1000], 2, 1, 0), ([130, 130, 130], [130, 777, 4000], 4, 2, 0),
                                                  ([64], [3333], 8, 2, 0), ([300], [900], 2, 2, 1), ([300], [900], 2, 2, 40), ([512, 512], [512, 1500], 1, 1, 333), ([1000], [1001], 3, 1, 64),
                                                  ([256, 256], [256, 200], 1, 1, 0)])
def test_equal_chunks_of_many_rows(qs, kvs, Hq, Hkv, window, d):
    b = Batch(qs, kvs, Hkv, d, "bf16", "bf16", 32, seed=d + len(qs))
    _run(b, Hq, "chunks", window=window, max_q=max(qs), max_kv=max(max(kvs), 1))


@pytest.mark.parametrize("dtype,cache,d", [("bf16", "bf16", 64), ("bf16", "bf16", 256), ("bf16", "fp8", 128), ("f32", "f32", 64)])
def test_what_the_windows_left_behind_reaches_no_result(dtype, cache, d):
    """places in front of a sequence's windows may belong to other sequences by now, or hold nothing that was ever written"""
    window = 21
    b = Batch([1, 70, 5, 2], [333, 170, 90, 22], 2, d, dtype, cache, 16)
    for n, (m, kv) in enumerate(zip(b.qs, b.kvs)):
        at = torch.arange(max(kv - m - window + 1, 0))
        ids, slots = b.table_host[n].long()[at // 16].cuda(), (at % 16).cuda()
        for t in (b.k_pages, b.v_pages, b.k_scale, b.v_scale):
            if t is not None:
                x = t.float()
                x[ids, :, slots] = float("nan")
                t.copy_(x.to(t.dtype))
    _run(b, 4, "windows", window=window)


def test_a_querys_nan_stays_in_its_row():
    b = Batch([4, 50], [100, 90], 1, 128, "bf16", "bf16", 16)
    q, qh = b.rows(2)
    want = b.attend(q)
    q[1, 0, 3] = float("nan")
    q[30, 1, 3] = float("nan")
    got = b.attend(q)
    torch.cuda.synchronize()
    bad = got.isnan().all(-1)
    assert bad[1, 0] and bad[30, 1] and int(bad.sum()) == 2 == int(got.isnan().any(-1).sum())
    keep = ~bad
    assert torch.equal(got[keep], want[keep])


def test_strided_queries_other_streams_and_the_same_bits_again():
    b = Batch([1, 33, 2], [2000, 400, 77], 2, 128, "bf16", "fp8", 64)
    row = torch.randn(b.T, 4 * 128 + 256, generator=b.gen).to(torch.bfloat16).cuda()
    q = row[:, 128:128 + 512].unflatten(1, (4, 128))
    want = b.attend(q.contiguous())
    torch.cuda.synchronize()
    side, o = torch.cuda.Stream(), torch.empty(b.T, 4, 128, dtype=torch.bfloat16, device="cuda")
    b.attend(q, o=o, stream=side)
    side.synchronize()
    assert torch.equal(o, want)
    ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")       # (NaN everywhere)
    assert torch.equal(b.attend(q, workspace=ws), want)
    b.check(want, q.double().cpu(), 128 ** -0.5, 0, "strided")


def test_a_given_stream_owns_what_the_call_allocates():
    """the workspace of a call on another stream is not handed to this stream's tensors while the call is still to run"""
    b = Batch([1], [4000], 2, 128, "bf16", "bf16", 64)
    q, _ = b.rows(8)
    want = b.attend(q)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
    o = b.attend(q, stream=side)
    taken = [torch.zeros(1 << n, dtype=torch.uint8, device="cuda") for n in range(9, 22) for _ in range(3)]
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(o, want) and not any(bool(t.any()) for t in taken)


def test_chunks_in_pieces_equal_one_call():
    """a prompt processed in chunks over the cache gives what one call gives, to rounding"""
    b = Batch([300], [300], 2, 64, "f32", "f32", 16)
    q, qh, whole = _run(b, 4, "whole")
    at = 0
    for m in (1, 100, 16, 183):
        b.cu = torch.tensor([0, m], dtype=torch.int32).cuda()
        b.kv_len = torch.tensor([at + m], dtype=torch.int32).cuda()
        o = b.attend(q[at:at + m])
        assert torch.allclose(o, whole[at:at + m], rtol=1e-5, atol=1e-5)
        at += m


def test_tables_with_anything_in_them_stay_inside_the_cache():
    b = Batch([1, 40], [50, 90], 1, 64, "bf16", "bf16", 16, junk=0.5)
    q, _ = b.rows(2)
    b.table = torch.full_like(b.table, 2 ** 30)
    b.kv_len = torch.tensor([10 ** 9, -5], dtype=torch.int32).cuda()
    o = b.attend(q)
    torch.cuda.synchronize()
    assert torch.isfinite(o[0]).all() and not o[1:].any()


def test_graphs():
    b = Batch([1, 1, 40, 1], [2000, 30, 60, 1], 2, 128, "bf16", "fp8", 16)
    q, _ = b.rows(4)
    o = torch.empty_like(q)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    replays(lambda: b.attend(q, o=o, workspace=ws, max_q=40, max_kv=2000), [o], lambda: b.attend(q))


def test_refusals():
    b = Batch([2], [2000], 2, 64, "bf16", "bf16", 16)
    q, _ = b.rows(4)
    for kw in (dict(q=q.float()), dict(q=q[..., :32]), dict(q=q[:, :, None])):
        with pytest.raises((TypeError, ValueError)):
            b.attend(**kw)
    for kw, status in ((dict(q=q[:, :3].contiguous()), -2), (dict(scale=0.0), -2), (dict(window=-1), -2), (dict(max_q=3), -2), (dict(max_kv=10 ** 6), -2),
                       (dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), -5)):
        with pytest.raises(dn.DeltaNetError) as e:
            b.attend(**{**dict(q=q), **kw})
        assert e.value.status == status, kw
    with pytest.raises(ValueError):
        b.attend(q, o=torch.empty_like(q)[:1])


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_many_sequences_of_every_kind(cache):
    """more sequences than the search for a workgroup's tile looks at together, chunks beside single tokens and empty ones"""
    qs = [(0, 1, 40, 3, 17, 90)[(7 * n) % 6] for n in range(150)]
    kvs = [q + (5 * n) % 37 for n, q in enumerate(qs)]
    b = Batch(qs, kvs, 1, 64, "bf16", cache, 16, seed=4)
    _run(b, 2, "many", max_q=90, max_kv=max(kvs))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_bounds_that_promise_equal_chunks_and_padded_rows(d):
    """as many rows as sequences times max_q, but shorter sequences and rows that lie in none"""
    b = Batch([40, 1, 0, 33], [70, 9, 5, 33], 2, d, "bf16", "bf16", 16, seed=d)
    q, qh = b.rows(4, rows=4 * 40)
    o = b.attend(q, max_q=40, o=torch.full_like(q, float("nan")))
    torch.cuda.synchronize()
    b.check(o, qh, d ** -0.5, 0, "padded")
    assert not o[b.T:].any()


def test_a_window_longer_than_the_context_is_none():
    b = Batch([3, 50], [80, 60], 1, 128, "bf16", "bf16", 16)
    q, _ = b.rows(2)
    want = b.attend(q)
    for window in (b.table.shape[1] * 16, 2 ** 31 - 1):
        assert torch.equal(b.attend(q, window=window), want)
