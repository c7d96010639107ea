"""Helpers of the attention operators' GPU tests: batches over a paged cache, and the element-wise check against a bound."""
import numpy as np
import torch

import paper_2406_06484_amd as dn
from tests import attention_reference as ref

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}


def near(got, want, bound, label):
    """every element of `got` (device) within `bound` of `want` (float64, host)"""
    got = got.double().cpu()
    assert got.shape == want.shape, (label, got.shape, want.shape)
    assert torch.isfinite(got).all(), "%s: not finite" % label
    off = (got - want).abs()
    worst = float((off / bound.clamp(min=1e-300)).max()) if off.numel() else 0.0
    print("%s: largest error / bound %.3f" % (label, worst), flush=True)
    assert (off <= bound).all(), "%s: error / bound %.3f" % (label, worst)


class Batch:
    """Sequences with `qs` new tokens at the end of contexts of `kvs` tokens, in a cache of pages in random order.  `k`, `v` are the
    contexts' values as the cache holds them (float64, host); every other place of the cache holds `junk`."""

    def __init__(self, qs, kvs, Hkv, d, dtype="bf16", cache="bf16", page=16, seed=0, junk=float("nan"), spare=2, k_size=1.0):
        g = torch.Generator().manual_seed(seed)
        self.qs, self.kvs, self.Hkv, self.d, self.dtype, self.cache, self.page = qs, kvs, Hkv, d, dtype, cache, page
        counts = [-(-n // page) for n in kvs]
        total = sum(counts) + spare
        order = torch.randperm(total, generator=g).int()
        width = max(counts + [1]) + 1
        table = torch.full((len(kvs), width), -7, dtype=torch.int32)     # entries past a sequence's pages are not read
        at = 0
        for n, c in enumerate(counts):
            table[n, :c] = order[at:at + c]
            at += c
        self.table_host = table
        kp = torch.full((total, Hkv, page, d), junk, dtype=torch.float64)
        vp = kp.clone()
        ks, vs = (torch.full((total, Hkv, page), junk, dtype=torch.float64) for _ in range(2))
        self.k, self.v = [], []
        for n, kv in enumerate(kvs):
            for which, pages, scales, held in ((0, kp, ks, self.k), (1, vp, vs, self.v)):
                x = torch.randn(kv, Hkv, d, generator=g, dtype=torch.float64) * (k_size if which == 0 else 1.0)
                if cache == "fp8":
                    values, scale = ref.e4m3(x.float().double())
                    scale = scale.float().double()
                else:
                    values, scale = x.to(TYPES[cache]).double(), torch.ones(kv, Hkv, 1, dtype=torch.float64)
                p = torch.arange(kv)
                ids = table[n].long()[p // page] if kv else p
                pages[ids, :, p % page] = values
                scales[ids, :, p % page] = scale[..., 0]
                held.append(values * scale)
        self.k_pages, self.v_pages = (t.float().to(TYPES[cache]).cuda() for t in (kp, vp))
        self.k_scale, self.v_scale = ((t.float().cuda() for t in (ks, vs)) if cache == "fp8" else (None, None))
        self.cu_host = np.concatenate([[0], np.cumsum(qs)]).astype(np.int32)
        self.cu = torch.from_numpy(self.cu_host).cuda()
        self.kv_len = torch.tensor(kvs, dtype=torch.int32).cuda()
        self.table = table.cuda()
        self.T, self.gen = int(self.cu_host[-1]), g

    def tensors(self):
        return (self.k_pages, self.v_pages, self.table, self.kv_len)

    def scales(self):
        return dict(k_scale=self.k_scale, v_scale=self.v_scale)

    def rows(self, heads, rows=None):
        """random rows of the tensors' type: (device, float64)"""
        x = torch.randn(self.T if rows is None else rows, heads, self.d, generator=self.gen, dtype=torch.float64).to(TYPES[self.dtype])
        return x.cuda(), x.double()

    def attend(self, q, **kw):
        return dn.deltanet_paged_attn_fwd(q, *self.tensors(), self.cu, **self.scales(), **kw)

    def check(self, o, q, scale, window, label):
        for n, (m, kv) in enumerate(zip(self.qs, self.kvs)):
            lo = int(self.cu_host[n])
            want, size, top = ref.attention(q[lo:lo + m], self.k[n], self.v[n], kv - m, scale, window)
            near(o[lo:lo + m], want, ref.attention_bound(want, size, top, self.d, kv, self.dtype), "%s seq %d (%d of %d)" % (label, n, m, kv))


def replays(step, outs, disturb, times=3):
    """captures step() into a graph and checks that every replay writes what the eager run wrote; eager work between the replays"""
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(times):
        for t in outs:
            t.zero_()
        disturb()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), i
