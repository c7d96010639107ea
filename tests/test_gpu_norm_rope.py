"""The norm and rotation of queries and keys, and its gradient, against their statement in 64 bits."""
import pytest
import torch

import paper_2406_06484_amd as dn
from tests import attention_reference as ref
from tests.attention_util import TYPES, near, replays

pytestmark = pytest.mark.gpu


def _inputs(T, Hq, Hkv, d, dtype, seed, fused=True, weight=True):
    g = torch.Generator().manual_seed(seed)
    row = torch.randn(T, (Hq + 2 * Hkv) * d, generator=g).to(TYPES[dtype]).cuda()
    q, k = row[:, :Hq * d].unflatten(1, (Hq, d)), row[:, Hq * d:(Hq + Hkv) * d].unflatten(1, (Hkv, d))
    if not fused:
        q, k = q.contiguous(), k.contiguous()
    w = [(1 + 0.3 * torch.randn(d, generator=g)).to(TYPES[dtype]).cuda() if weight else None for _ in range(2)]
    dy = [torch.randn(T, H, d, generator=g).to(TYPES[dtype]).cuda() for H in (Hq, Hkv)]
    return q, k, w, dy, g


def _host(t):
    return None if t is None else t.double().cpu()


def _check(q, k, w, dy, rope, pos, eps, inter, dtype, label):
    T = q.shape[0]
    kw = dict(eps=eps, interleaved=inter)
    dpos = None if pos is None else pos.int().cuda()
    drope = None if rope is None else rope.cuda()
    outs = dn.deltanet_qk_norm_rope_fwd(q, k, *w, drope, dpos, **kw)
    grads = dn.deltanet_qk_norm_rope_bwd(q, k, *dy, *w, drope, dpos, **kw)
    torch.cuda.synchronize()
    pos = torch.arange(T) if pos is None else pos
    for i, (x, name) in enumerate(((q, "q"), (k, "k"))):
        x, wt, g = _host(x), _host(w[i]), _host(dy[i])
        near(outs[i], ref.norm_rope(x, wt, rope, pos, eps, inter), ref.norm_rope_bound(x, wt, rope, pos, eps, inter, dtype), "%s %s" % (label, name))
        dx, dw = ref.norm_rope_grad(x, wt, rope, pos, eps, inter, g)
        bx, bw = ref.norm_rope_grad_bound(x, wt, rope, pos, eps, inter, g, dtype)
        near(grads[i], dx, bx, "%s d%s" % (label, name))
        if wt is None:
            assert grads[2 + i] is None
        else:
            assert grads[2 + i].dtype == torch.float32
            near(grads[2 + i], dw, bw, "%s d%s_weight" % (label, name))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("inter", [False, True])
def test_head_sizes_types_and_pairs(dtype, d, inter):
    q, k, w, dy, _ = _inputs(37, 6, 3, d, dtype, d)
    _check(q, k, w, dy, ref.rope_table(64, d), None, 1e-6, inter, dtype, "d %d" % d)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("inter", [False, True])
def test_more_tokens_than_one_workgroup_takes(dtype, d, inter):
    q, k, w, dy, _ = _inputs(701, 6, 3, d, dtype, d + 1)
    _check(q, k, w, dy, ref.rope_table(701, d), None, 1e-6, inter, dtype, "d %d" % d)


@pytest.mark.parametrize("T,Hq,Hkv,d", [(9, 3, 1, 128), (64, 8, 8, 64), (128, 4, 2, 64), (500, 1, 1, 64), (33, 7, 1, 256)])
def test_few_tokens_in_place_and_with_one_weight(T, Hq, Hkv, d):
    q, k, w, dy, _ = _inputs(T, Hq, Hkv, d, "bf16", T)
    rope, pos = ref.rope_table(T, d), torch.arange(T).flip(0)
    _check(q, k, w, dy, rope, pos, 1e-6, False, "bf16", "both weights")
    _check(q, k, [w[0], None], dy, rope, pos, 1e-6, False, "bf16", "q's weight")
    _check(q, k, [None, w[1]], dy, rope, pos, 1e-6, True, "bf16", "k's weight")
    want = dn.deltanet_qk_norm_rope_bwd(q, k, *dy, *w, rope.cuda())
    a, b = (t.clone() for t in dy)
    got = dn.deltanet_qk_norm_rope_bwd(q, k, a, b, *w, rope.cuda(), dq=a, dk=b)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


@pytest.mark.parametrize("T,Hq,Hkv,d,rot", [(1, 1, 1, 64, 64), (1, 16, 16, 128, 64), (3, 5, 1, 128, 16), (4, 33, 11, 64, 48), (2050, 4, 2, 128, 128), (301, 2, 2, 256, 112),
                                            (65, 7, 7, 32, 32), (9, 3, 1, 64, 0)])
def test_sizes_and_partial_rotations(T, Hq, Hkv, d, rot):
    for dtype in ("f32", "bf16"):
        q, k, w, dy, g = _inputs(T, Hq, Hkv, d, dtype, T + rot)
        pos = torch.randint(0, 500, (T,), generator=g)
        _check(q, k, w, dy, ref.rope_table(500, rot) if rot else None, pos, 1e-5, rot % 32 == 16, dtype, "T %d rot %d" % (T, rot))


def test_many_rows_reach_every_loop():
    """more rows than the launches have waves, so that each takes several"""
    q, k, w, dy, _ = _inputs(20000, 2, 1, 32, "f32", 6)
    _check(q, k, w, dy, ref.rope_table(20000, 32), None, 1e-6, False, "f32", "20000 rows")


def test_without_weights_and_with_large_small_and_zero_rows():
    q, k, w, dy, _ = _inputs(12, 4, 4, 64, "f32", 8, weight=False)
    q[1] *= 1e15
    q[2] *= 1e-15
    q[3] = 0
    k[4] = 0
    _check(q, k, w, dy, ref.rope_table(12, 64), None, 1e-6, False, "f32", "extremes")
    out = dn.deltanet_qk_norm_rope_fwd(q, k)[0]
    assert not out[3].any()


def test_dense_batches_restart_their_positions():
    q, k, w, dy, _ = _inputs(3 * 17, 4, 2, 64, "bf16", 9)
    rope = ref.rope_table(17, 64).cuda()
    pos = torch.arange(17, dtype=torch.int32).repeat(3).cuda()
    want = dn.deltanet_qk_norm_rope_fwd(q, k, *w, rope, pos)
    got = dn.deltanet_qk_norm_rope_fwd(q.unflatten(0, (3, 17)), k.unflatten(0, (3, 17)), *w, rope)
    assert got[0].shape == (3, 17, 4, 64)
    for a, b in zip(got, want):
        assert torch.equal(a.flatten(0, 1), b)
    grads = dn.deltanet_qk_norm_rope_bwd(q, k, *dy, *w, rope, pos)
    again = dn.deltanet_qk_norm_rope_bwd(q.unflatten(0, (3, 17)), k.unflatten(0, (3, 17)), *(t.unflatten(0, (3, 17)) for t in dy), *w, rope)
    for a, b in zip(again, grads):
        assert torch.equal(a.reshape(b.shape), b)


def test_positions_outside_the_table_read_its_nearest_row():
    q, k, w, dy, _ = _inputs(4, 2, 2, 64, "f32", 10)
    _check(q, k, w, dy, ref.rope_table(5, 64), torch.tensor([-3, 4, 5, 1000000]), 1e-6, False, "f32", "table's ends")


def test_gradients_may_replace_what_they_came_from_and_are_the_same_every_time():
    q, k, w, dy, _ = _inputs(300, 8, 2, 128, "bf16", 11)
    rope = ref.rope_table(300, 128).cuda()
    want = dn.deltanet_qk_norm_rope_bwd(q, k, *dy, *w, rope)
    a, b = (t.clone() for t in dy)
    got = dn.deltanet_qk_norm_rope_bwd(q, k, a, b, *w, rope, dq=a, dk=b)
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_kernel_gradients_against_differences():
    q, k, w, dy, g = _inputs(5, 2, 1, 64, "f32", 12)
    table, pos = ref.rope_table(5, 64), torch.arange(5)
    grads = dn.deltanet_qk_norm_rope_bwd(q, k, *dy, *w, table.cuda())
    for i, x in enumerate((q, k)):
        x, wt, d = _host(x), _host(w[i]), _host(dy[i])
        f = lambda x, wt: float((ref.norm_rope(x, wt, table, pos, 1e-6, False) * d).sum())  # noqa: E731
        u, uw = torch.randn(x.shape, generator=g, dtype=torch.float64), torch.randn(64, generator=g, dtype=torch.float64)
        assert float((_host(grads[i]) * u).sum()) == pytest.approx((f(x + 1e-5 * u, wt) - f(x - 1e-5 * u, wt)) / 2e-5, rel=1e-4, abs=1e-4)
        assert float((_host(grads[2 + i]) * uw).sum()) == pytest.approx((f(x, wt + 1e-5 * uw) - f(x, wt - 1e-5 * uw)) / 2e-5, rel=1e-4, abs=1e-4)


def test_no_rows():
    q, k = torch.empty(0, 4, 64, device="cuda"), torch.empty(0, 2, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    a, b = dn.deltanet_qk_norm_rope_fwd(q, k, w, w)
    assert a.shape == (0, 4, 64) and b.shape == (0, 2, 64)
    grads = dn.deltanet_qk_norm_rope_bwd(q, k, a, b, w, w, dq_weight=torch.full((64,), 5.0, device="cuda"))
    torch.cuda.synchronize()
    assert not grads[2].any() and not grads[3].any()


def test_another_stream_and_graphs():
    q, k, w, dy, _ = _inputs(129, 4, 4, 128, "bf16", 13)
    rope = ref.rope_table(129, 128).cuda()
    want = dn.deltanet_qk_norm_rope_fwd(q, k, *w, rope) + dn.deltanet_qk_norm_rope_bwd(q, k, *dy, *w, rope)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    qo, ko = torch.empty_like(want[0]), torch.empty_like(want[1])
    dn.deltanet_qk_norm_rope_fwd(q, k, *w, rope, q_out=qo, k_out=ko, stream=side)
    side.synchronize()
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    dq, dk = torch.empty_like(qo), torch.empty_like(ko)
    dqw, dkw = (torch.empty(128, device="cuda") for _ in range(2))

    def step():
        dn.deltanet_qk_norm_rope_fwd(q, k, *w, rope, q_out=qo, k_out=ko)
        dn.deltanet_qk_norm_rope_bwd(q, k, *dy, *w, rope, dq=dq, dk=dk, dq_weight=dqw, dk_weight=dkw)

    replays(step, [qo, ko, dq, dk, dqw, dkw], lambda: dn.deltanet_qk_norm_rope_fwd(q[:7], k[:7], *w, rope))


def test_refusals():
    q, k, w, dy, _ = _inputs(4, 4, 2, 64, "bf16", 14)
    rope = ref.rope_table(4, 64).cuda()
    for bad in (dict(q=q.float()), dict(k=k[:3]), dict(k=k[..., :32]), dict(w=[w[0].float(), w[1]]), dict(w=[w[0][:32], w[1]]), dict(rope=rope.double()),
                dict(rope=rope[0]), dict(pos=torch.zeros(4, dtype=torch.int64, device="cuda")), dict(pos=torch.zeros(3, dtype=torch.int32, device="cuda")),
                dict(q=q.transpose(0, 1)), dict(q=q.half(), k=k.half())):
        a = {**dict(q=q, k=k, w=w, rope=rope, pos=None), **bad}
        with pytest.raises((TypeError, ValueError)):
            dn.deltanet_qk_norm_rope_fwd(a["q"], a["k"], *a["w"], a["rope"], a["pos"])
    with pytest.raises((TypeError, ValueError)):
        dn.deltanet_qk_norm_rope_bwd(q, k, dy[0].float(), dy[1], *w, rope)
    with pytest.raises(dn.DeltaNetError) as e:
        dn.deltanet_qk_norm_rope_bwd(q, k, *dy, *w, rope, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == -5
    with pytest.raises(dn.DeltaNetError) as e:
        dn.deltanet_qk_norm_rope_fwd(q, k, *w, ref.rope_table(4, 24).cuda())
    assert e.value.status == -3
