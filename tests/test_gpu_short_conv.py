"""The short convolution and its gradient on the GPU against the 64-bit statement."""
import pytest
import torch

import paper_2406_06484_amd as dn
from tests import layer_reference as ref
from tests.attention_util import near, replays

pytestmark = pytest.mark.gpu


class Case:
    """Sequences of `lens` rows; widths of the parts and whether they are activated; x a column block of a wider tensor."""

    def __init__(self, lens, widths, silu, W, dtype, bias, states, packed=True, seed=0, size=1.0):
        g = torch.Generator().manual_seed(seed)
        self.td, self.dtype, self.lens, self.widths, self.silu, self.W = ref.TYPES[dtype], dtype, lens, widths, silu, W
        rand = lambda *s: (torch.randn(*s, generator=g, dtype=torch.float64) * size).to(self.td)  # noqa: E731
        T, C, N = sum(lens), sum(widths), len(lens)
        self.T, self.C, self.N = T, C, N
        self.host = dict(x=rand(T, C), w=rand(C, W), b=rand(C) if bias else None, s=rand(N, W - 1, C) if states else None, ds=rand(N, W - 1, C) if states else None,
                         dy=rand(T, C))
        dev = {k: None if v is None else v.cuda() for k, v in self.host.items()}
        wide = torch.full((T, C + 24), float("nan"), dtype=self.td, device="cuda")
        wide[:, 8:8 + C] = dev["x"]
        self.x, self.w, self.b, self.s, self.ds = wide[:, 8:8 + C], dev["w"], dev["b"], dev["s"], dev["ds"]
        self.dy = tuple(t.contiguous() for t in dev["dy"].split(widths, 1))
        self.offsets = [sum(lens[:i]) for i in range(N + 1)]
        self.cu = torch.tensor(self.offsets, dtype=torch.int32, device="cuda") if packed else None
        if not packed:
            self.x = self.x.unflatten(0, (N, lens[0] if N else 0))
            self.dy = tuple(t.unflatten(0, self.x.shape[:2]) for t in self.dy)
        self.on = torch.cat([torch.full((n,), bool(s)) for n, s in zip(widths, silu)])
        self.kw = dict(splits=widths, silu=silu, cu_seqlens=self.cu)
        self.wide64 = {k: None if v is None else v.double() for k, v in self.host.items()}

    def check_forward(self, y, last, label):
        h = self.wide64
        (want, bound), final = ref.conv(h["x"], h["w"], h["b"], h["s"], self.lens, self.on, self.dtype)
        near(torch.cat([t.reshape(self.T, n) for t, n in zip(y, self.widths)], 1), want, bound, label + " y")
        assert torch.equal(last.double().cpu(), final), label

    def check_backward(self, got, label):
        h = self.wide64
        want = ref.conv_grad(h["x"], h["w"], h["b"], h["s"], self.lens, self.on, h["dy"], h["ds"], self.dtype)
        for name, g, (v, bound) in zip(("dx", "dw", "db", "ds"), got, want):
            if g is not None:
                near(g.reshape(v.shape), v, bound, "%s %s" % (label, name))
        assert (got[2] is None) == (self.b is None) and (got[3] is None) == (self.s is None)


CASES = [
    # lens, widths, silu, W, type, bias, states, packed
    ([1], [8], [True], 4, "bf16", False, False, False),
    ([16, 16], [8, 16, 8], [True, False, True], 4, "bf16", True, True, False),
    ([1, 1, 1, 1, 1], [264], [True], 4, "bf16", False, True, False),
    ([3, 3], [520], [False], 2, "bf16", True, False, False),
    ([1, 0, 2, 3, 17, 0, 64, 65, 5], [24, 512, 16], [False, True, False], 4, "bf16", True, True, True),
    ([1, 0, 2, 3, 17, 0, 64, 65, 5], [24, 128, 16], [False, True, True], 3, "f32", True, True, True),
    ([0, 0, 33], [12], [True], 2, "f32", False, True, True),
    ([200, 1, 130], [4, 4, 260], [True, True, False], 4, "f32", False, False, True),
    ([700], [1048], [True], 3, "bf16", False, True, True),
    ([1] * 70 + [0] * 70 + [4, 1], [40], [True], 4, "bf16", True, True, True),
    ([0, 0], [16], [True], 4, "bf16", True, True, True),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_forward_and_backward(case):
    c = Case(*CASES[case], seed=case)
    y, last = dn.deltanet_short_conv_fwd(c.x, c.w, c.b, c.s, **c.kw)
    c.check_forward(y, last, "case %d" % case)
    c.check_backward(dn.deltanet_short_conv_bwd(c.x, c.w, c.dy, c.b, c.s, c.ds, **c.kw), "case %d" % case)


def test_long_sequences_of_many_strips_and_workgroups():
    for dtype in ("bf16", "f32"):
        c = Case([5000, 77, 3000], [16, 8], [True, False], 4, dtype, True, True)
        y, last = dn.deltanet_short_conv_fwd(c.x, c.w, c.b, c.s, cu_seqlens_host=c.offsets, **c.kw)
        c.check_forward(y, last, dtype)
        c.check_backward(dn.deltanet_short_conv_bwd(c.x, c.w, c.dy, c.b, c.s, c.ds, **c.kw), dtype)


def test_one_part_is_a_tensor_and_values_of_every_size():
    c = Case([40, 9], [64], [True], 4, "f32", True, True, size=30.0)
    y, last = dn.deltanet_short_conv_fwd(c.x, c.w, c.b, c.s, cu_seqlens=c.cu)
    assert isinstance(y, torch.Tensor)
    c.check_forward((y,), last, "large")
    c.check_backward(dn.deltanet_short_conv_bwd(c.x, c.w, c.dy[0], c.b, c.s, c.ds, cu_seqlens=c.cu), "large")


@pytest.mark.parametrize("T", [0, 2])
def test_dense_sequences_of_fewer_rows_than_taps(T):
    c = Case([T, T, T], [16], [True], 4, "bf16", True, True, packed=False)
    y, last = dn.deltanet_short_conv_fwd(c.x, c.w, c.b, c.s, **c.kw)
    c.check_forward(y, last, "T %d" % T)
    c.check_backward(dn.deltanet_short_conv_bwd(c.x, c.w, c.dy, c.b, c.s, c.ds, **c.kw), "T %d" % T)


@pytest.mark.parametrize("W", [2, 3, 4])
def test_chunks_and_single_tokens_continue_a_sequence_with_states_in_place(W):
    c = Case([37, 37], [96], [True], W, "bf16", False, True, packed=False)
    whole, last = dn.deltanet_short_conv_fwd(c.x, c.w, None, c.s)
    state, at, parts = c.s.clone(), 0, []
    with pytest.raises(ValueError, match="evenly spaced"):
        dn.deltanet_short_conv_fwd(c.x[:, :2], c.w)
    for m in (1, 1, 2, 3, 1, 16, 5, 1, 7):
        y, same = dn.deltanet_short_conv_fwd(c.x[:, at:at + m].contiguous(), c.w, None, state, final_state=state)
        assert same.data_ptr() == state.data_ptr()
        parts.append(y)
        at += m
    assert at == 37 and torch.equal(torch.cat(parts, 1), whole) and torch.equal(state, last)


def test_rows_in_no_sequence_become_zero_and_neighbours_do_not_mix():
    c = Case([20, 13, 31], [32], [True], 4, "bf16", False, False)
    cu = torch.tensor([20, 20, 33], dtype=torch.int32, device="cuda")       # the first 20 and the last 31 rows lie in none
    y, last = dn.deltanet_short_conv_fwd(c.x, c.w, cu_seqlens=cu)
    alone, _ = dn.deltanet_short_conv_fwd(c.x[20:33].unsqueeze(0), c.w)
    assert torch.equal(y[20:33], alone[0]) and not y[:20].any() and not y[33:].any() and not last[0].any()
    dx, dw, _, _ = dn.deltanet_short_conv_bwd(c.x, c.w, c.dy[0], cu_seqlens=cu)
    dx1, dw1, _, _ = dn.deltanet_short_conv_bwd(c.x[20:33].unsqueeze(0), c.w, c.dy[0][20:33].unsqueeze(0))
    assert torch.equal(dx[20:33], dx1[0]) and not dx[:20].any() and not dx[33:].any()
    near(dw, dw1.double().cpu(), 100 * 2.0 ** -24 * (dw1.abs().double().cpu() + 100), "dw")
    x = c.x.clone()
    x[20:33] = float("nan")
    y, _ = dn.deltanet_short_conv_fwd(x, c.w, **{**c.kw, "splits": None, "silu": True})
    assert torch.isfinite(y[:20]).all() and torch.isnan(y[20:33]).all() and torch.isfinite(y[33:]).all()


@pytest.mark.parametrize("cu", [[0, -5, 90], [64, 3, 17, 99, -1], [1 << 30, -(1 << 30), 5], [7]])
def test_malformed_offsets_stay_inside(cu):
    c = Case([64], [32], [True], 4, "bf16", False, False)
    cu = torch.tensor(cu, dtype=torch.int32, device="cuda")
    room = torch.full((3, 64, 32), 7.0, dtype=torch.bfloat16, device="cuda")
    y, _ = dn.deltanet_short_conv_fwd(c.x, c.w, cu_seqlens=cu, y=room[1])
    dn.deltanet_short_conv_bwd(c.x, c.w, c.dy[0], cu_seqlens=cu)
    torch.cuda.synchronize()
    assert (room[0] == 7).all() and (room[2] == 7).all()


def test_gradient_into_a_column_block_and_given_outputs():
    c = Case([50, 9], [16, 32], [True, False], 4, "bf16", True, True)
    block = torch.full((59, 80), 5.0, dtype=torch.bfloat16, device="cuda")
    given = dict(dx=block[:, 16:64], dweight=torch.empty(48, 4, device="cuda"), dbias=torch.empty(48, device="cuda"), dinitial_state=torch.empty_like(c.s),
                 workspace=torch.empty(1 << 22, dtype=torch.uint8, device="cuda"))
    got = dn.deltanet_short_conv_bwd(c.x, c.w, c.dy, c.b, c.s, c.ds, **c.kw, **given)
    c.check_backward(got, "given")
    assert all(got[i].data_ptr() == t.data_ptr() for i, t in enumerate(list(given.values())[:4]))
    assert (block[:, :16] == 5).all() and (block[:, 64:] == 5).all()


def test_offsets_that_begin_anywhere_and_another_stream():
    c = Case([9, 30], [32], [True], 4, "bf16", False, False)
    cu = torch.tensor([77] + c.offsets, dtype=torch.int32, device="cuda")[1:]
    want, _ = dn.deltanet_short_conv_fwd(c.x, c.w, cu_seqlens=c.cu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, _ = dn.deltanet_short_conv_fwd(c.x, c.w, cu_seqlens=cu, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)


def test_captured_and_replayed():
    c = Case([900, 3, 41], [64, 32], [True, False], 4, "bf16", True, True)
    y = tuple(torch.empty_like(t) for t in c.dy)
    last, outs = torch.empty_like(c.s), [torch.empty(c.T, c.C, dtype=c.td, device="cuda"), torch.empty(c.C, 4, device="cuda"), torch.empty(c.C, device="cuda"), torch.empty_like(c.s)]
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")

    def step():
        dn.deltanet_short_conv_fwd(c.x, c.w, c.b, c.s, y=y, final_state=last, **c.kw)
        dn.deltanet_short_conv_bwd(c.x, c.w, c.dy, c.b, c.s, c.ds, dx=outs[0], dweight=outs[1], dbias=outs[2], dinitial_state=outs[3], workspace=ws, **c.kw)
    replays(step, [*y, last, *outs], lambda: ws.fill_(0x7f))


def test_more_elements_than_31_bits_count():
    T, C = 1 << 17, 16392        # 2^31 + 2^20 elements
    x = torch.zeros(1, T, C, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    x[0, -40:] = torch.randn(40, C, generator=g, device="cuda").to(torch.bfloat16)
    w = torch.randn(C, 4, generator=g, device="cuda").to(torch.bfloat16)
    y, last = dn.deltanet_short_conv_fwd(x, w)
    tail, last1 = dn.deltanet_short_conv_fwd(x[:, -40:], w)
    assert torch.equal(y[:, -40:], tail) and torch.equal(last, last1) and not y[:, :-40].any()
    dx, dw, _, _ = dn.deltanet_short_conv_bwd(x, w, y)
    dx1, dw1, _, _ = dn.deltanet_short_conv_bwd(x[:, -40:], w, tail)
    assert torch.equal(dx[:, -40:], dx1)
    near(dw, dw1.double().cpu(), 64 * 2.0 ** -24 * (dw1.abs().double().cpu() + 40), "dw")
