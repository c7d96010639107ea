"""The operators around a mixer together, as a model uses them: a DeltaNet block's training step against 64 bits, and the hybrid example served with all of them."""
import pytest
import torch

import example_hybrid
import paper_2406_06484_amd as dn
from tests.attention_util import Batch, replays
from tests.gpu_util import TOL

pytestmark = pytest.mark.gpu
EPS, KEEP, SCALE = 1e-5, 0.875, 0.5


def rms(x):
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS)


def statement(p, lens, H, d):
    """(y, h) of the block in 64 bits: residual sum and norm, projection, convolution, feature map, delta rule token by token, gated norm, projection, normed and gated
    branch, sum and norm"""
    D = H * d
    h0 = p["residual"] + p["x"]
    y0 = rms(h0) * p["w0"]
    row, gate = y0 @ p["w_in"], y0 @ p["w_gate"]
    outs, at = [], 0
    for n in lens:
        r = torch.nn.functional.pad(row[at:at + n, :3 * D], (0, 0, 3, 0))
        z = sum(p["conv"][:, j] * r[j:j + n] for j in range(4)) + p["bias"]
        q, k = (torch.nn.functional.normalize(torch.nn.functional.silu(t.view(n, H, d)), dim=-1) for t in z[:, :2 * D].split(D, 1))
        v, beta = torch.nn.functional.silu(z[:, 2 * D:]).view(n, H, d), torch.sigmoid(row[at:at + n, 3 * D:])
        S = torch.zeros(H, d, d, dtype=torch.float64)
        for t in range(n):
            new = v[t] - (S * k[t][:, :, None]).sum(1)
            S = S + beta[t][:, None, None] * k[t][:, :, None] * new[:, None, :]
            outs.append((S * q[t][:, :, None]).sum(1))
        at += n
    o = rms(torch.stack(outs)) * p["w_o"] * torch.nn.functional.silu(gate.view(-1, H, d))
    h1 = KEEP * h0 + SCALE * p["u"] * rms(o.reshape(-1, D) @ p["w_out"])
    return rms(h1) * p["w1"], h1


def step(p, lens, H, d, dy, dh):
    """the same by the library's calls, forward and backward: (y, h, gradients by name)"""
    D = H * d
    host = [sum(lens[:i]) for i in range(len(lens) + 1)]
    cu = torch.tensor(host, dtype=torch.int32, device="cuda")
    seq = dict(cu_seqlens=cu, cu_seqlens_host=host)
    conv = dict(splits=(D, D, D), silu=(False, False, True), **seq)
    y0, h0 = dn.deltanet_block_norm_fwd(p["x"], p["residual"], p["w0"], eps=EPS)
    row, gate = y0 @ p["w_in"], y0 @ p["w_gate"]
    qkv = row[:, :3 * D].contiguous()
    heads = lambda t: t.view(-1, H, d)  # noqa: E731
    (q, k, v), _ = dn.deltanet_short_conv_fwd(qkv, p["conv"], p["bias"], **conv)
    q, k, v, beta = heads(q), heads(k), heads(v), row[:, 3 * D:].contiguous()
    o, _, saved = dn.deltanet_fused_fwd_save(q, k, v, beta, **seq)
    on = dn.deltanet_out_norm_fwd(o, heads(gate), p["w_o"], eps=EPS)
    br = on.view(-1, D) @ p["w_out"]
    mix = dict(gate=p["u"], post_norm=True, scale=SCALE, residual_scale=KEEP, eps=EPS)
    y1, h1 = dn.deltanet_block_norm_fwd(br, h0, p["w1"], **mix)
    g = {}
    dbr, dh0, g["w1"], g["u"] = dn.deltanet_block_norm_bwd(dy, h1, br, p["w1"], dh, **mix)
    don = dbr @ p["w_out"].t()
    g["w_out"] = on.view(-1, D).t() @ dbr
    do, dgate, g["w_o"] = dn.deltanet_out_norm_bwd(o, heads(don), heads(gate), p["w_o"], eps=EPS)
    dq, dk, dv, dbeta, _ = dn.deltanet_fused_bwd_saved(q, k, v, beta, do, saved, **seq)
    dqkv, g["conv"], g["bias"], _ = dn.deltanet_short_conv_bwd(qkv, p["conv"], tuple(t.reshape(-1, D) for t in (dq, dk, dv)), p["bias"], **conv)
    drow = torch.cat([dqkv, dbeta], 1)
    g["w_in"], g["w_gate"] = y0.t() @ drow, y0.t() @ dgate.view(-1, D)
    dy0 = drow @ p["w_in"].t() + dgate.view(-1, D) @ p["w_gate"].t()
    g["x"], g["residual"], g["w0"], _ = dn.deltanet_block_norm_bwd(dy0, h0, None, p["w0"], dh0, eps=EPS)
    return y1, h1, g


@pytest.mark.parametrize("lens", [[70], [1, 40, 0, 67]])
def test_training_step_of_a_block(lens):
    """Normalised largest errors within what the library's fp32 passes are held to; every part's own roundings are far below."""
    H, d, T = 2, 64, sum(lens)
    D = H * d
    g = torch.Generator().manual_seed(len(lens))
    rand = lambda *s, size=1.0: size * torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    p = dict(x=rand(T, D), residual=rand(T, D), w0=1 + rand(D, size=0.1), w_in=rand(D, 3 * D + H, size=D ** -0.5), w_gate=rand(D, D, size=D ** -0.5), conv=rand(3 * D, 4, size=0.5),
             bias=rand(3 * D, size=0.1), w_o=1 + rand(d, size=0.1), w_out=rand(D, D, size=D ** -0.5), u=1 + rand(D, size=0.3), w1=1 + rand(D, size=0.1))
    p = {k: v.float().double().requires_grad_() for k, v in p.items()}
    dy, dh = (rand(T, D).float().double() for _ in range(2))
    y, h = statement(p, lens, H, d)
    want = dict(zip(p, torch.autograd.grad((y * dy).sum() + (h * dh).sum(), list(p.values()))))
    dev = {k: v.detach().float().cuda() for k, v in p.items()}
    y1, h1, got = step(dev, lens, H, d, dy.float().cuda(), dh.float().cuda())
    assert set(got) == set(want)
    for name, a, b in [("y", y1, y), ("h", h1, h)] + [(n, got[n], want[n]) for n in want]:
        off = float((a.double().cpu() - b.detach()).abs().max() / b.detach().abs().max())
        print(name, "%.1e" % off, flush=True)
        assert off <= TOL["f32"], (name, off)


@pytest.mark.parametrize("layers,heads,head_size,window,more", [(4, 4, 64, 256, dict(taps=4, gated=True, fused=True)), (2, 2, 128, 0, dict(taps=2, gated=True, cache="bf16", fused=True)), (4, 2, 128, 100, dict(taps=3)),
                                                               (4, 4, 64, 256, dict(taps=4, gated=True, cache="fp4", fused=True)), (2, 2, 128, 0, dict(gated=True, cache="fp4"))])
def test_served_in_chunks_and_in_one_piece(layers, heads, head_size, window, more):
    """As the example's own test: half a per cent per layer.  With a 4-bit cache a rounding to bf16 in front of it, 2^-8 of a number, tips over up to 3 * 2^-8 of the numbers (neighbours are a third of a number
    apart, or more), by up to their own size: sqrt(3 * 2^-8), a tenth, of the keys and as much of the values of an attention layer, every second one."""
    off, _ = example_hybrid.run(layers, heads, head_size, window, tokens=6, **more)
    print("relative difference", off)
    assert off <= (0.1 * layers / 2 if more.get("cache") == "fp4" else 5e-3 * layers)


def test_a_captured_generation_step():
    """A DeltaNet layer's and an attention layer's single-token step in one graph, states and pages written in place on every replay."""
    N, H, d, Hkv = 5, 4, 64, 2
    D = H * d
    g = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    x, conv, rows0, w, gate = rand(N, 1, 3 * D), rand(3 * D, 4), rand(N, 3, 3 * D), rand(D), rand(N, 1, H, d)
    S0 = torch.randn(N, H, d, d, generator=g, device="cuda")
    b = Batch([1] * N, [1, 20, 64, 65, 300], Hkv, d, cache="bf16", junk=0.0)
    k4, v4, ks, vs = dn.deltanet_paged_cache(b.k_pages.shape[0], b.page, Hkv, d, torch.float4_e2m1fn_x2)
    for t in (k4, v4, ks, vs):
        t.view(torch.uint8).zero_()
    q, k, v, beta = rand(N, H, d), rand(N, Hkv, d), rand(N, Hkv, d), rand(N, 1, H)
    rows, S = rows0.clone(), S0.clone()
    y = tuple(torch.empty(N, 1, D, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    o, on, a = (torch.empty(N, 1, H, d, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    nxt, stream = (torch.empty(N, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    cache = (k4, v4, b.table, b.kv_len)

    def step():
        rows.copy_(rows0)
        S.copy_(S0)
        dn.deltanet_short_conv_fwd(x, conv, None, rows, splits=(D, D, D), silu=(True, True, True), y=y, final_state=rows)
        dn.deltanet_recurrent_fwd(*(t.view(N, 1, H, d) for t in y), beta, S, o=o, final_state=S)
        dn.deltanet_out_norm_fwd(o, gate, y=on)
        dn.deltanet_block_norm_fwd(on.view(N, D), x[:, 0, :D], w, y=nxt, h=stream)
        dn.deltanet_paged_append(k, v, *cache, b.cu, k_scale=ks, v_scale=vs)
        dn.deltanet_paged_attn_fwd(q, *cache, b.cu, k_scale=ks, v_scale=vs, o=a.view(N, H, d), workspace=ws)
    replays(step, [*y, rows, S, o, on, a, nxt, stream], lambda: ws.fill_(0x7f))
