"""Calls of more workgroups than one row of a grid has room for (2^32 threads): every part of the work is done."""
import pytest
import torch

import paper_2406_06484_amd as dn

pytestmark = pytest.mark.gpu


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("N,per", [(64, 64), (256, 256)])
def test_fp32_chunks_under_the_loosest_bound(N, per):
    """max_q is the whole batch's number of tokens where the caller names none"""
    H, d = 16, 32
    g = torch.Generator(device="cuda").manual_seed(N)
    q = torch.randn(N * per, H, d, generator=g, device="cuda")
    k, v = (torch.randn(N * per // 16, 1, 16, d, generator=g, device="cuda") for _ in range(2))
    table = torch.arange(N * per // 16, dtype=torch.int32, device="cuda").view(N, -1)
    cu, kv = torch.arange(0, N * per + 1, per, dtype=torch.int32, device="cuda"), torch.full((N,), per, dtype=torch.int32, device="cuda")
    want = dn.deltanet_paged_attn_fwd(q, k, v, table, kv, cu, max_q=per)
    got = dn.deltanet_paged_attn_fwd(q, k, v, table, kv, cu, o=torch.full_like(q, float("nan")))
    assert torch.isfinite(want).all() and torch.equal(got, want)


def test_fp32_chunks_among_many_sequences_without_one():
    N, m, Hq, d = 16384, 20, 64, 32
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(m, Hq, d, generator=g, device="cuda")
    k, v = (torch.randn(2, 1, 16, d, generator=g, device="cuda") for _ in range(2))
    table, kv = torch.zeros(N, 2, dtype=torch.int32, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")
    table[:, 1], kv[777] = 1, 25
    cu = torch.zeros(N + 1, dtype=torch.int32, device="cuda")
    cu[778:] = m
    want = dn.deltanet_paged_attn_fwd(q, k, v, table[:1], _i32([25]), _i32([0, m]))
    got = dn.deltanet_paged_attn_fwd(q, k, v, table, kv, cu, o=torch.full_like(q, float("nan")))
    assert torch.isfinite(want).all() and torch.equal(got, want)


@pytest.mark.parametrize("max_q", [1, None])
def test_many_sequences_of_many_heads(max_q):
    """one token each, over one key: its value"""
    N, H, d = 65535, 257, 64
    q = torch.ones(N, H, d, dtype=torch.bfloat16, device="cuda")
    k = torch.ones(1, H, 16, d, dtype=torch.bfloat16, device="cuda")
    v = torch.randn(1, H, 16, d, device="cuda").to(torch.bfloat16)
    o = dn.deltanet_paged_attn_fwd(q, k, v, torch.zeros(N, 1, dtype=torch.int32, device="cuda"), torch.ones(N, dtype=torch.int32, device="cuda"),
                                   torch.arange(N + 1, dtype=torch.int32, device="cuda"), max_q=max_q, o=torch.full_like(q, float("nan")))
    assert (o == v[:, :, 0]).all()


def test_many_tokens_written_and_read():
    """the last tokens of a chunk far longer than its context"""
    T, d, held = (1 << 26) + 4, 64, 40
    k = torch.zeros(T, 1, d, dtype=torch.bfloat16, device="cuda")
    k[-held:] = torch.randn(held, 1, d, device="cuda").to(torch.bfloat16)
    pages = [torch.zeros(3, 1, 16, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    batch = (_i32([[2, 0, 1]]), _i32([held]), _i32([0, T]))
    dn.deltanet_paged_append(k, k, *pages, *batch)
    for p in pages:
        assert torch.equal(p[[2, 0, 1], 0].flatten(0, 1)[:held], k[-held:, 0])
    out = [torch.full_like(k, 1.0) for _ in range(2)]
    dn.deltanet_paged_read(*pages, *batch, T, k_out=out[0], v_out=out[1])
    for t in out:
        assert torch.equal(t[-held:], k[-held:]) and not t[:-held].any()
