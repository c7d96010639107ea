"""The output norm and the block norm on the GPU, with their gradients, against the 64-bit statements."""
import pytest
import torch

import paper_2406_06484_amd as dn
from tests import layer_reference as ref
from tests.attention_util import near, replays

pytestmark = pytest.mark.gpu
EPS = 1e-6


def rng(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda td, *s, size=1.0: (torch.randn(*s, generator=g, dtype=torch.float64) * size).to(td)


def wide(t):
    return None if t is None else t.double()


def column_block(t):
    """t's values as rows apart inside a larger tensor of NaN"""
    T = t.shape[0]
    row = t.shape[1:].numel()
    room = torch.full((T, row + 32), float("nan"), dtype=t.dtype, device="cuda")
    room[:, 16:16 + row] = t.reshape(T, row).cuda()
    return room[:, 16:16 + row].unflatten(1, t.shape[1:]) if t.dim() > 2 else room[:, 16:16 + row]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,d", [(1, 1, 32), (5, 3, 64), (33, 16, 128), (7, 2, 256), (1030, 5, 64), (300, 7, 32), (0, 2, 64)])
@pytest.mark.parametrize("kind", ["silu", "sigmoid", None])
def test_output_norm(dtype, T, H, d, kind):
    rand, td = rng(T * 1000 + H + d), ref.TYPES[dtype]
    o, g, w, dy = rand(td, T, H, d, size=0.5), rand(td, T, H, d, size=3.0) if kind else None, rand(td, d), rand(td, T, H, d)
    if T > 4:
        o[2] = 0.0
    od, gd, wd, dyd = column_block(o), None if g is None else column_block(g), w.cuda(), dy.cuda()
    act = kind or "silu"
    label = "%s %dx%dx%d %s" % (dtype, T, H, d, kind)
    want, bound = ref.out_norm(wide(o), wide(g), wide(w), EPS, kind, dtype)
    near(dn.deltanet_out_norm_fwd(od, gd, wd, act=act), want, bound, label)
    (do, edo), dg, (dw, edw) = ref.out_norm_grad(wide(o), wide(g), wide(w), EPS, kind, wide(dy), dtype)
    got = dn.deltanet_out_norm_bwd(od, dyd, gd, wd, act=act)
    near(got[0], do, edo, label + " do")
    near(got[2], dw, edw, label + " dw")
    if dg is None:
        assert got[1] is None
    else:
        near(got[1], *dg, label + " dgate")
    # without a weight; d_o over dy, the gate's gradient into a column block
    want, bound = ref.out_norm(wide(o), wide(g), None, EPS, kind, dtype)
    near(dn.deltanet_out_norm_fwd(od, gd, act=act), want, bound, label + " no weight")
    (do, edo), dg, _ = ref.out_norm_grad(wide(o), wide(g), None, EPS, kind, wide(dy), dtype)
    room = torch.full((T, H * d + 16), 3.0, dtype=td, device="cuda")
    block = room[:, 16:].unflatten(1, (H, d)) if kind else None
    got = dn.deltanet_out_norm_bwd(od, dyd, gd, act=act, d_o=dyd, dgate=block)
    assert got[0].data_ptr() == dyd.data_ptr() and got[2] is None and (room[:, :16] == 3).all()
    near(dyd, do, edo, label + " do in place")
    if kind:
        near(block, *dg, label + " dgate in a block")


def test_output_norm_dense_rows_and_gates_of_every_size():
    rand = rng(1)
    o, dy = (rand(torch.float32, 2, 9, 3, 64).cuda() for _ in range(2))
    g = torch.linspace(-120, 120, 2 * 9 * 3 * 64).view(2, 9, 3, 64).cuda()
    y = dn.deltanet_out_norm_fwd(o, g)
    do, dg, _ = dn.deltanet_out_norm_bwd(o, dy, g)
    flat = lambda t: t.flatten(0, 1).double().cpu()  # noqa: E731
    near(y.flatten(0, 1), *ref.out_norm(flat(o), flat(g), None, EPS, "silu", "f32"), "y")
    (v, e), gg, _ = ref.out_norm_grad(flat(o), flat(g), None, EPS, "silu", flat(dy), "f32")
    near(do.flatten(0, 1), v, e, "do")
    near(dg.flatten(0, 1), *gg, "dgate")


WIDTHS = [(1, 8), (3, 64), (9, 504), (130, 512), (6, 520), (5, 1024), (17, 1032), (33, 2048), (4, 2056), (3, 4096), (7, 4104), (5, 8192), (0, 64), (70, 24), (77, 128), (1030, 136), (35, 256), (1, 200), (4099, 32)]


@pytest.mark.parametrize("dtype,stream", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("T,D", WIDTHS)
@pytest.mark.parametrize("post,gated", [(False, False), (True, True), (True, False), (False, True)])
def test_block_norm(dtype, stream, T, D, post, gated):
    rand, td, ts = rng(T * 10000 + D), ref.TYPES[dtype], ref.TYPES[stream]
    x, res, w, u = rand(td, T, D), rand(ts, T, D, size=2.0), rand(td, D), rand(td, D) if gated else None
    dy, dh = rand(td, T, D), rand(ts, T, D)
    scale, keep = (1.0, 1.0) if not (post or gated) else (0.37, 0.9)
    # the call rounds them to fp32
    scale, keep = (float(torch.tensor(v, dtype=torch.float32)) for v in (scale, keep))
    kw = dict(gate=None if u is None else u.cuda(), post_norm=post, scale=scale, residual_scale=keep)
    label = "%s %s %dx%d post %d gate %d" % (dtype, stream, T, D, post, gated)
    xd, rd, wd = column_block(x), column_block(res), w.cuda()
    y, h = dn.deltanet_block_norm_fwd(xd, rd, wd, **kw)
    (yw, ye), (hw, he) = ref.block_norm(wide(x), wide(res), wide(w), wide(u), post, scale, keep, EPS, dtype, stream)
    near(y, yw, ye, label + " y")
    near(h, hw, he, label + " h")
    assert h.dtype == ts and y.dtype == td
    got = dn.deltanet_block_norm_bwd(dy.cuda(), h, xd, wd, dh.cuda(), **kw)
    want = ref.block_norm_grad(wide(dy), wide(dh), h.double().cpu(), wide(x), wide(w), wide(u), post, scale, keep, EPS, dtype, stream)
    for name, a, (v, e) in zip(("dx", "dresidual", "dw", "dgate"), got, want):
        if name == "dgate" and not gated:
            assert a is None
        else:
            near(a, v, e, "%s %s" % (label, name))
    assert (got[0].data_ptr() == got[1].data_ptr()) == (T == 0 or (dtype == stream and not post and not gated))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_block_norm_parts_left_out(dtype):
    rand, td = rng(5), ref.TYPES[dtype]
    x, w, dy = rand(td, 11, 256), rand(td, 256), rand(td, 11, 256)
    # the first norm of a model: no residual, the stream is x
    y, h = dn.deltanet_block_norm_fwd(x.cuda().view(1, 11, 256), None, w.cuda())
    near(y[0], *ref.block_norm(wide(x), None, wide(w), None, False, 1.0, 1.0, EPS, dtype, dtype)[0], "first")
    assert h.shape == (1, 11, 256) and torch.equal(h[0].cpu(), x)
    dx, dr, dw, dg = dn.deltanet_block_norm_bwd(dy.cuda(), x.cuda(), None, w.cuda(), want_dresidual=False)
    want = ref.block_norm_grad(wide(dy), None, wide(x), None, wide(w), None, False, 1.0, 1.0, EPS, dtype, dtype)
    near(dx, *want[0], "dx")
    near(dw, *want[2], "dw")
    assert dr is None and dg is None
    # a stream in fp32 begun by a given h, a scaled branch, no weight
    room = torch.empty(11, 256, device="cuda")
    half = float(torch.tensor(0.3, dtype=torch.float32))
    y, h = dn.deltanet_block_norm_fwd(x.cuda(), scale=half, post_norm=True, h=room)
    (yw, ye), (hw, he) = ref.block_norm(wide(x), None, None, None, True, half, 1.0, EPS, dtype, "f32")
    near(y, yw, ye, "begun y")
    near(h, hw, he, "begun h")
    dx, dr, dw, dg = dn.deltanet_block_norm_bwd(dy.cuda(), h, x.cuda(), scale=half, post_norm=True)
    want = ref.block_norm_grad(wide(dy), None, h.double().cpu(), wide(x), None, None, True, half, 1.0, EPS, dtype, "f32")
    near(dx, *want[0], "begun dx")
    near(dr, *want[1], "begun dresidual")
    assert dw is None and dg is None


def test_block_norm_in_place():
    rand = rng(6)
    for D in (512, 2048, 4096):
        x, res, w, dy, dh = (rand(torch.bfloat16, *s).cuda() for s in ((19, D), (19, D), (D,), (19, D), (19, D)))
        y, h = dn.deltanet_block_norm_fwd(x, res, w, post_norm=True, scale=0.5)
        y2, h2 = x.clone(), res.clone()
        dn.deltanet_block_norm_fwd(y2, h2, w, post_norm=True, scale=0.5, y=y2, h=h2)
        assert torch.equal(y, y2) and torch.equal(h, h2)
        want = dn.deltanet_block_norm_bwd(dy, h, x, w, dh, post_norm=True, scale=0.5)
        a, b = dy.clone(), dh.clone()
        got = dn.deltanet_block_norm_bwd(a, h, x, w, b, post_norm=True, scale=0.5, dx=a, dresidual=b)
        assert all(torch.equal(p, q) for p, q in zip(want[:3], got[:3]))


def test_first_norm_in_place_of_the_branch_keeps_the_stream():
    x = rng(9)(torch.bfloat16, 19, 512).cuda()
    want, h = dn.deltanet_block_norm_fwd(x)
    assert h.data_ptr() == x.data_ptr()
    y = x.clone()
    got, h = dn.deltanet_block_norm_fwd(y, y=y)
    assert got.data_ptr() == y.data_ptr() and h.data_ptr() != y.data_ptr()
    assert torch.equal(got, want) and torch.equal(h, x)


@pytest.mark.parametrize("T,D", [(16, 512), (17, 512), (128, 64), (129, 64), (4, 4096), (5, 4096)])
def test_block_norm_where_one_workgroup_ends_to_have_all_rows(T, D):
    rand = rng(T + D)
    h, w, dy, u, x = rand(torch.bfloat16, T, D), rand(torch.bfloat16, D), rand(torch.bfloat16, T, D), rand(torch.bfloat16, D), rand(torch.bfloat16, T, D)
    got = dn.deltanet_block_norm_bwd(dy.cuda(), h.cuda(), x.cuda(), w.cuda(), gate=u.cuda())
    want = ref.block_norm_grad(wide(dy), None, wide(h), wide(x), wide(w), wide(u), False, 1.0, 1.0, EPS, "bf16", "bf16")
    for name, a, (v, e) in zip(("dx", "dresidual", "dw", "dgate"), got, want):
        near(a, v, e, "%dx%d %s" % (T, D, name))


@pytest.mark.parametrize("T", [32, 33])
def test_output_norm_where_one_workgroup_ends_to_have_all_rows(T):
    rand = rng(T)
    o, g, w, dy = rand(torch.bfloat16, T, 4, 128), rand(torch.bfloat16, T, 4, 128), rand(torch.bfloat16, 128), rand(torch.bfloat16, T, 4, 128)
    got = dn.deltanet_out_norm_bwd(o.cuda(), dy.cuda(), g.cuda(), w.cuda())
    for name, a, (v, e) in zip(("do", "dgate", "dw"), got, ref.out_norm_grad(wide(o), wide(g), wide(w), EPS, "silu", wide(dy), "bf16")):
        near(a, v, e, name)


def test_norms_on_another_stream():
    rand = rng(10)
    o, g, w = (rand(torch.bfloat16, *s).cuda() for s in ((300, 4, 64), (300, 4, 64), (64,)))
    x, res = (rand(torch.bfloat16, 300, 256).cuda() for _ in range(2))
    calls = [lambda **k: [dn.deltanet_out_norm_fwd(o, g, w, **k)], lambda **k: dn.deltanet_out_norm_bwd(o, g, g, w, **k),
             lambda **k: dn.deltanet_block_norm_fwd(x, res, post_norm=True, **k), lambda **k: dn.deltanet_block_norm_bwd(x, res, x, post_norm=True, **k)]
    side = torch.cuda.Stream()
    for call in calls:
        want = call()
        side.wait_stream(torch.cuda.current_stream())
        got = call(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(want, got))


def test_a_row_of_nan_or_infinity_stays_in_its_row():
    rand = rng(7)
    for D in (64, 1024, 2048, 8192):
        x, res = rand(torch.bfloat16, 9, D).cuda(), rand(torch.bfloat16, 9, D).cuda()
        x[4, 3], res[6, 5] = float("nan"), float("inf")
        y, h = dn.deltanet_block_norm_fwd(x, res)
        rest = [i for i in range(9) if i not in (4, 6)]
        assert torch.isfinite(y[rest]).all() and torch.isnan(y[4]).all() and torch.isnan(y[6, 5])
        assert torch.isnan(h[4, 3]) and torch.isinf(h[6, 5]) and torch.isfinite(h[rest]).all()


def test_same_bits_every_time_and_replayed():
    rand = rng(8)
    o, g, dy, w = (rand(torch.bfloat16, *s).cuda() for s in ((700, 4, 64), (700, 4, 64), (700, 4, 64), (64,)))
    x, res, u, dh = (rand(torch.bfloat16, *s).cuda() for s in ((700, 256), (700, 256), (256,), (700, 256)))
    ww = rand(torch.bfloat16, 256).cuda()
    dyb = dy.view(700, 256)
    outs = [torch.empty_like(o), torch.empty_like(o), torch.empty_like(o), torch.empty(64, device="cuda"), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x), torch.empty_like(x),
            torch.empty(256, device="cuda"), torch.empty(256, device="cuda")]
    ws = [torch.empty(1 << 22, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def step():
        dn.deltanet_out_norm_fwd(o, g, w, y=outs[0])
        dn.deltanet_out_norm_bwd(o, dy, g, w, d_o=outs[1], dgate=outs[2], dweight=outs[3], workspace=ws[0])
        dn.deltanet_block_norm_fwd(x, res, ww, gate=u, post_norm=True, y=outs[4], h=outs[5])
        dn.deltanet_block_norm_bwd(dyb, outs[5], x, ww, dh, gate=u, post_norm=True, dx=outs[6], dresidual=outs[7], dweight=outs[8], dgate=outs[9], workspace=ws[1])
    replays(step, outs, lambda: [t.fill_(0x7f) for t in ws])


def test_more_elements_than_31_bits_count():
    T, D = (1 << 18) + 96, 8192      # 2^31 elements and some rows
    g = torch.Generator(device="cuda").manual_seed(0)
    tail = torch.randn(64, D, generator=g, device="cuda").to(torch.bfloat16)
    x = torch.ones(T, D, dtype=torch.bfloat16, device="cuda")
    x[-64:] = tail
    y, h = dn.deltanet_block_norm_fwd(x, x)
    y1, h1 = dn.deltanet_block_norm_fwd(tail, tail)
    assert torch.equal(y[-64:], y1) and torch.equal(h[-64:], h1)
    dx, _, _, _ = dn.deltanet_block_norm_bwd(y, h)
    dx1, _, _, _ = dn.deltanet_block_norm_bwd(y1, h1)
    assert torch.equal(dx[-64:], dx1)
    del dx, h
    heads = (T * D // 256) // 16
    o = x.view(-1)[:heads * 16 * 256].view(heads, 16, 256)
    a = dn.deltanet_out_norm_fwd(o, o)
    assert torch.equal(a[-8:], dn.deltanet_out_norm_fwd(o[-8:].clone(), o[-8:].clone()))
    b, c, _ = dn.deltanet_out_norm_bwd(o, a, o)
    b1, c1, _ = dn.deltanet_out_norm_bwd(o[-8:].clone(), a[-8:].clone(), o[-8:].clone())
    assert torch.equal(b[-8:], b1) and torch.equal(c[-8:], c1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,D", [(1, 64), (11, 256), (300, 1032)])
@pytest.mark.parametrize("weighted", [True, False])
def test_first_norm_of_a_column_block_and_its_gradient(dtype, T, D, weighted):
    """A model's first norm on rows apart: the stream that the forward call returns is what the backward call takes."""
    rand, td = rng(T + D), ref.TYPES[dtype]
    x, w, dy, dh = rand(td, T, D), rand(td, D) if weighted else None, rand(td, T, D), rand(td, T, D)
    wd = None if w is None else w.cuda()
    y, h = dn.deltanet_block_norm_fwd(column_block(x), None, wd)
    near(y, *ref.block_norm(wide(x), None, wide(w), None, False, 1.0, 1.0, EPS, dtype, dtype)[0], "y")
    assert h.is_contiguous() and torch.equal(h.cpu(), x)
    dx, dr, dw, dg = dn.deltanet_block_norm_bwd(dy.cuda(), h, None, wd, dh.cuda(), want_dresidual=False)
    want = ref.block_norm_grad(wide(dy), wide(dh), wide(x), None, wide(w), None, False, 1.0, 1.0, EPS, dtype, dtype)
    near(dx, *want[0], "dx")
    assert dr is None and dg is None
    if weighted:
        near(dw, *want[2], "dw")
    dense = dn.deltanet_block_norm_fwd(column_block(x).unsqueeze(0), None, wd)
    assert all(t.shape == (1, T, D) and torch.equal(t[0], s) for t, s in zip(dense, (y, h)))


@pytest.mark.parametrize("dtype,stream", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("T,D", [(13, 32), (1031, 32), (131, 64), (7, 136), (333, 136), (21, 512), (6, 1024), (5, 2056), (3, 8192), (67, 8192)])
@pytest.mark.parametrize("post,gated", [(False, False), (True, True)])
def test_block_norm_in_place_at_every_width(dtype, stream, T, D, post, gated):
    """Rows that share a wave, whose lanes past the last row read it again while its owner stores; rows of some waves; one workgroup and several."""
    rand, td, ts = rng(T + D), ref.TYPES[dtype], ref.TYPES[stream]
    x, res, w, u, dy, dh = (rand(t, *s).cuda() for t, s in ((td, (T, D)), (ts, (T, D)), (td, (D,)), (td, (D,)), (td, (T, D)), (ts, (T, D))))
    kw = dict(gate=u if gated else None, post_norm=post, scale=0.5)
    y, h = dn.deltanet_block_norm_fwd(x, res, w, **kw)
    y2, h2 = x.clone(), res.clone()
    dn.deltanet_block_norm_fwd(y2, h2, w, y=y2, h=h2, **kw)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    want = dn.deltanet_block_norm_bwd(dy, h, x, w, dh, **kw)
    a, b = dy.clone(), dh.clone()
    got = dn.deltanet_block_norm_bwd(a, h, x, w, b, dx=a, dresidual=b, **kw)
    assert got[0].data_ptr() == a.data_ptr() and got[1].data_ptr() == b.data_ptr()
    assert all((p is None and q is None) or torch.equal(p, q) for p, q in zip(want, got))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,d", [(1, 1, 32), (37, 3, 32), (1031, 3, 32), (7, 5, 64), (333, 4, 128), (3, 2, 256), (129, 3, 256)])
def test_output_norm_in_place(dtype, T, H, d):
    rand, td = rng(T + d), ref.TYPES[dtype]
    o, g, w, dy = (rand(td, *s).cuda() for s in ((T, H, d), (T, H, d), (d,), (T, H, d)))
    y = o.clone()
    want, got = dn.deltanet_out_norm_fwd(o, g, w), dn.deltanet_out_norm_fwd(y, g, w, y=y)
    assert got.data_ptr() == y.data_ptr() and torch.equal(got, want)
    want, a = dn.deltanet_out_norm_bwd(o, dy, g, w), dy.clone()
    got = dn.deltanet_out_norm_bwd(o, a, g, w, d_o=a)
    assert got[0].data_ptr() == a.data_ptr() and all(torch.equal(p, q) for p, q in zip(want, got))
