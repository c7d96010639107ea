"""The paged cache: rows written (quantised, or normalised and rotated first) and read back."""
import pytest
import torch

import paper_2406_06484_amd as dn
from tests import attention_reference as ref
from tests.attention_util import TYPES, Batch, near, replays

pytestmark = pytest.mark.gpu

FORMS = [("f32", "f32", 32), ("f32", "f32", 64), ("f32", "f32", 128), ("bf16", "bf16", 64), ("bf16", "bf16", 128), ("bf16", "bf16", 256), ("bf16", "fp8", 64),
         ("bf16", "fp8", 128), ("bf16", "fp8", 256)]


def _read(b, lens):
    cu = torch.tensor([0] + list(torch.tensor(lens).cumsum(0)), dtype=torch.int32).cuda()
    return dn.deltanet_paged_read(*b.tensors(), cu, int(cu[-1]), dtype=TYPES[b.dtype], **b.scales())


def _expected(b, n, held, new):
    """sequence n's context, its last rows replaced by the new ones (those in front of the context's start dropped)"""
    kept = max(b.kvs[n] - new.shape[0], 0)
    return torch.cat([held[n][:kept], new[new.shape[0] - (b.kvs[n] - kept):]])


@pytest.mark.parametrize("dtype,cache,d", FORMS)
@pytest.mark.parametrize("page", [16, 64, 256])
def test_written_rows_read_back(dtype, cache, d, page):
    b = Batch([1, 5, 0, 40, 33], [1, 70, 20, 40, 300], 3, d, dtype, cache, page, seed=d + page)
    k, kh = b.rows(3)
    v, vh = b.rows(3)
    v[2, 1] = 0
    vh[2, 1] = 0
    dn.deltanet_paged_append(k, v, *b.tensors(), b.cu, **b.scales())
    rk, rv = _read(b, b.kvs)
    torch.cuda.synchronize()
    at = 0
    for n in range(len(b.qs)):
        lo = int(b.cu_host[n])
        for got, held, new in ((rk, b.k, kh), (rv, b.v, vh)):
            new = new[lo:lo + b.qs[n]]
            if cache == "fp8" and len(new):
                values, scale = ref.e4m3(new)
                new = values * scale.float().double()
            want = _expected(b, n, held, new)
            if cache == "fp8":   # the products with the factor are rounded to bf16: equal to what fp32 gives, half a step of bf16 at most from the definition
                near(got[at:at + b.kvs[n]], want, want.abs() * (2.0 ** -8 + 2.0 ** -22) + 1e-30, "seq %d" % n)
            else:
                assert torch.equal(got[at:at + b.kvs[n]].double().cpu(), want)
        at += b.kvs[n]


@pytest.mark.parametrize("dtype,cache,d", FORMS)
@pytest.mark.parametrize("inter,rot", [(False, 32), (True, 16)])
def test_norm_and_rotation_on_the_way_in(dtype, cache, d, inter, rot):
    Hq, Hkv = 6, 2
    b = Batch([1, 9, 0, 30, 3], [1, 9, 7, 77, 500], Hkv, d, dtype, cache, 32, seed=d + rot)
    g = b.gen
    row = torch.randn(b.T, (Hq + 2 * Hkv) * d, generator=g).to(TYPES[dtype])
    parts = [x.unflatten(1, (-1, d)) for x in row.split([Hq * d, Hkv * d, Hkv * d], 1)]
    dev = [x.unflatten(1, (-1, d)) for x in row.cuda().split([Hq * d, Hkv * d, Hkv * d], 1)]       # rows of one projection's output
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(TYPES[dtype]) for _ in range(2)]
    rope = ref.rope_table(500, rot)
    q_out = dn.deltanet_paged_norm_rope_append(*dev, *b.tensors(), b.cu, w[0].cuda(), w[1].cuda(), rope.cuda(), **b.scales(), eps=1e-5, interleaved=inter)
    rk, rv = _read(b, b.qs)
    torch.cuda.synchronize()
    pos = torch.cat([torch.arange(kv - q, kv) for q, kv in zip(b.qs, b.kvs)])
    qh, kh, vh = (x.double() for x in parts)
    args = (rope, pos, 1e-5, inter)
    near(q_out, ref.norm_rope(qh, w[0].double(), *args), ref.norm_rope_bound(qh, w[0].double(), *args, dtype), "q")
    k = ref.norm_rope(kh, w[1].double(), *args)
    bound = ref.norm_rope_bound(kh, w[1].double(), *args, dtype)
    if cache == "fp8":
        # half a step of the row's 8-bit numbers (2^-4 of an element, or of the factor times 2^-6), the result's rounding to bf16, and the
        # norm's own error, which may move a number by a step
        for got, x, err in ((rk, k, bound), (rv, vh, torch.zeros_like(vh))):
            scale = ref.e4m3(x)[1]
            near(got, x, torch.maximum(x.abs() * 2.0 ** -4, scale * 2.0 ** -10) * (1 + 2.0 ** -6) + x.abs() * 2.0 ** -8 + 2 * err + 1e-30, "8 bits")
        values, scale = ref.e4m3(vh)
        near(rv, values * scale, (values * scale).abs() * (2.0 ** -8 + 2.0 ** -22) + 1e-30, "v")
    else:
        near(rk, k, bound, "k")
        assert torch.equal(rv.double().cpu(), vh)


def test_eight_bits_keep_signs_zeros_tiny_rows_and_mark_infinities():
    b = Batch([6], [6], 1, 64, "bf16", "fp8", 16)
    k = torch.randn(6, 1, 64, generator=b.gen).to(torch.bfloat16)
    k[1] = 0
    k[2] *= 2.0 ** -120
    k[3, 0, 5] = float("inf")
    k[4, 0, 6] = float("nan")
    k[5] *= 2.0 ** 100
    v = -k
    dn.deltanet_paged_append(k.cuda(), v.cuda(), *b.tensors(), b.cu, **b.scales())
    rk, rv = (t.double().cpu() for t in _read(b, [6]))
    assert torch.equal(rk[:3].isfinite(), torch.ones(3, 1, 64, dtype=torch.bool)) and torch.equal(rv[0], -rk[0])
    assert not rk[1].any() and not rk[2].any()
    assert rk[3].isnan().all() and rk[4, 0, 6].isnan() and int(rk[4].isnan().sum()) == 1
    values, scale = ref.e4m3(k[5:].double())
    near(rk[5:], values * scale, (values * scale).abs() * (2.0 ** -8 + 2.0 ** -22), "large")


def test_only_the_new_tokens_places_change():
    for cache in ("bf16", "fp8"):
        b = Batch([3, 17], [20, 50], 2, 64, "bf16", cache, 16, seed=5, junk=3.0)
        before = [t.clone().view(torch.uint8) for t in (b.k_pages, b.v_pages)]
        k, _ = b.rows(2)
        dn.deltanet_paged_append(k, k, *b.tensors(), b.cu, **b.scales())
        torch.cuda.synchronize()
        places = torch.zeros(b.k_pages.shape[:3], dtype=torch.bool)
        for n in range(2):
            p = torch.arange(b.kvs[n] - b.qs[n], b.kvs[n])
            places[b.table_host[n].long()[p // 16], :, p % 16] = True
        for old, new in zip(before, (b.k_pages, b.v_pages)):
            same = (old == new.view(torch.uint8)).all(-1).cpu()
            assert same[~places].all()


def test_rows_without_a_place_are_dropped():
    """a context shorter than its chunk, rows past the last sequence, page numbers outside the cache, more tokens than the table has room for"""
    b = Batch([5, 2, 2, 2], [2, 16, 16, 32], 1, 64, "bf16", "bf16", 16, junk=1.0)
    table = b.table_host.clone()
    table[1, 0], table[2, 0] = -1, b.k_pages.shape[0]
    b.table = table.cuda()
    b.kv_len[3] = 1000
    k, kh = b.rows(1, rows=b.T + 3)
    before = b.k_pages.clone()
    dn.deltanet_paged_append(k, k, *b.tensors(), b.cu, **b.scales())
    torch.cuda.synchronize()
    changed = (b.k_pages != before).any(-1).cpu()
    want = torch.zeros_like(changed)
    want[table[0, 0].long(), 0, :2] = True
    assert torch.equal(changed & ~want, torch.zeros_like(changed))
    assert torch.equal(b.k_pages[table[0, 0].long(), 0, :2].double().cpu(), kh[3:5, 0])


def test_reading_more_than_the_context_gives_zeros_in_front():
    b = Batch([1, 1], [3, 20], 2, 64, "bf16", "fp8", 16)
    cu = torch.tensor([0, 5, 5 + 4], dtype=torch.int32).cuda()
    k, v = dn.deltanet_paged_read(*b.tensors(), cu, 12, **b.scales())
    torch.cuda.synchronize()
    assert k.shape == (12, 2, 64) and k.dtype == torch.bfloat16
    for got, held in ((k, b.k), (v, b.v)):
        assert not got[:2].any() and not got[9:].any()
        near(got[2:5], held[0], held[0].abs() * (2.0 ** -8 + 2.0 ** -22) + 1e-30, "short")
        near(got[5:9], held[1][16:], held[1][16:].abs() * (2.0 ** -8 + 2.0 ** -22) + 1e-30, "last four")


def test_many_sequences():
    """more sequences than one probe of a wave covers, some of them empty"""
    qs = [(n * 7) % 4 for n in range(300)]
    kvs = [q + (n % 5) for n, q in enumerate(qs)]
    b = Batch(qs, kvs, 1, 64, "bf16", "bf16", 16, seed=9)
    k, kh = b.rows(1)
    dn.deltanet_paged_append(k, k, *b.tensors(), b.cu)
    rk, _ = _read(b, b.qs)
    assert torch.equal(rk.double().cpu(), kh)


def test_offsets_past_32_bits():
    """a cache of over 2^31 elements: its last pages are reached"""
    page, d = 256, 256
    pages = (1 << 31) // (page * d) + 3
    k_pages = torch.empty(pages, 1, page, d, dtype=torch.bfloat16, device="cuda")
    v_pages = torch.empty_like(k_pages)
    table = torch.tensor([[pages - 1, 0]], dtype=torch.int32, device="cuda")
    kv_len, cu = torch.tensor([256 + 7], dtype=torch.int32, device="cuda"), torch.tensor([0, 263], dtype=torch.int32, device="cuda")
    x = torch.randn(263, 1, d, device="cuda").to(torch.bfloat16)
    dn.deltanet_paged_append(x, -x, k_pages, v_pages, table, kv_len, cu)
    k, v = dn.deltanet_paged_read(k_pages, v_pages, table, kv_len, cu, 263)
    assert torch.equal(k, x) and torch.equal(v, -x)
    assert torch.equal(k_pages[-1, 0], x[:256, 0]) and torch.equal(k_pages[0, 0, :7], x[256:, 0])
    o = dn.deltanet_paged_attn_fwd(x[-1:], k_pages, v_pages, table, kv_len, torch.tensor([0, 1], dtype=torch.int32, device="cuda"))
    want, size, top = ref.attention(x[-1:].double().cpu(), x.double().cpu(), -x.double().cpu(), 262, d ** -0.5, 0)
    near(o, want, ref.attention_bound(want, size, top, d, 263, "bf16"), "attention at the far end")


def test_no_rows_no_sequences_and_graphs():
    b = Batch([0, 0], [0, 5], 2, 64, "bf16", "fp8", 16)
    k, _ = b.rows(2)
    dn.deltanet_paged_append(k, k, *b.tensors(), b.cu, **b.scales())
    rk, _ = dn.deltanet_paged_read(*b.tensors(), torch.zeros(3, dtype=torch.int32, device="cuda"), 0, **b.scales())
    assert rk.shape == (0, 2, 64)
    b = Batch([1] * 5, [9, 1, 33, 16, 17], 2, 128, "bf16", "fp8", 16, junk=0.0)
    q, _ = b.rows(4)
    k, _ = b.rows(2)
    rope = ref.rope_table(40, 128).cuda()
    q_out, ko, vo = torch.empty_like(q), torch.empty_like(k), torch.empty_like(k)

    def step():
        dn.deltanet_paged_norm_rope_append(q, k, k, *b.tensors(), b.cu, None, None, rope, **b.scales(), q_out=q_out)
        dn.deltanet_paged_read(*b.tensors(), b.cu, 5, **b.scales(), k_out=ko, v_out=vo)

    replays(step, [q_out, ko, vo, b.k_pages.view(torch.uint8)[b.table_host[0, 0].long()]][:3], lambda: b.attend(q, max_kv=33))


def test_refusals():
    b = Batch([2], [9], 2, 64, "bf16", "fp8", 16)
    k, _ = b.rows(2)
    t = b.tensors()
    ok = dict(k=k, v=k, kp=t[0], vp=t[1], table=t[2], kv=t[3], cu=b.cu, ks=b.k_scale, vs=b.v_scale)
    for bad in (dict(k=k.float()), dict(v=k[:1]), dict(v=k[:, :1]), dict(kp=t[0][:1]), dict(kp=t[0].float()), dict(vp=t[1].transpose(1, 2)), dict(table=t[2].long()),
                dict(table=t[2][0]), dict(kv=t[3].long()), dict(kv=torch.cat([t[3], t[3]])), dict(cu=b.cu[:1]), dict(cu=b.cu.long()), dict(ks=None),
                dict(vs=b.v_scale[..., :8]), dict(ks=b.k_scale.double())):
        a = {**ok, **bad}
        with pytest.raises((TypeError, ValueError)):
            dn.deltanet_paged_append(a["k"], a["v"], a["kp"], a["vp"], a["table"], a["kv"], a["cu"], k_scale=a["ks"], v_scale=a["vs"])
    with pytest.raises(TypeError):
        dn.deltanet_paged_read(*t, b.cu, 2, dtype=torch.float16, **b.scales())
    with pytest.raises(dn.DeltaNetError) as e:
        dn.deltanet_paged_read(*t, b.cu, 2, dtype=torch.float32, **b.scales())
    assert e.value.status == -3
    assert [x is None for x in dn.deltanet_paged_cache(2, 16, 1, 64)] == [False, False, True, True]
    with pytest.raises(TypeError):
        dn.deltanet_paged_cache(2, 16, 1, 64, torch.float16)
