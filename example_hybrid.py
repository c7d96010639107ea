#!/usr/bin/env python3
"""A small hybrid model served in chunks: DeltaNet layers and sliding-window attention layers in turn, as the paper's hybrids have them,
with random weights.  Prompts of different lengths are processed in chunks and continued token by token; DeltaNet layers
carry a state of fixed size per sequence, attention layers a paged cache (8-bit here), into which queries' and keys' norm and rotation lead.
The same tokens in one piece give the same outputs, to rounding, which the script checks and reports.

    python example_hybrid.py [--layers 4] [--heads 4] [--head-size 64] [--window 256] [--tokens 40]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))


class Hybrid:
    """Layers of width heads x head_size; every second one attends (query heads in pairs over a key/value head)."""

    def __init__(self, layers, heads, head_size, window, sequences, max_len, page=64, seed=0):
        import torch
        self.torch, self.H, self.Hkv, self.d, self.window = torch, heads, max(1, heads // 2), head_size, window
        g = torch.Generator(device="cuda").manual_seed(seed)
        width, bf = heads * head_size, torch.bfloat16
        weight = lambda rows, cols: (torch.randn(rows, cols, generator=g, device="cuda") * rows ** -0.5).to(bf)  # noqa: E731
        self.layers = []
        for i in range(layers):
            if i % 2 == 0:      # q, k, v and the writing strength's logit
                self.layers.append(dict(kind="delta", w_in=weight(width, 3 * width + heads), w_out=weight(width, width)))
            else:
                self.layers.append(dict(kind="attn", w_in=weight(width, width + 2 * self.Hkv * head_size), w_out=weight(width, width),
                                        q_weight=torch.ones(head_size, dtype=bf, device="cuda"), k_weight=torch.ones(head_size, dtype=bf, device="cuda")))
        half = head_size // 2
        angle = torch.arange(max_len, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, device="cuda") / half)
        self.rope = torch.cat([angle.cos(), angle.sin()], 1).float()
        self.reset(sequences, max_len, page)

    def reset(self, sequences, max_len, page=64):
        import paper_2406_06484_amd as dn
        torch = self.torch
        pages = -(-max_len // page)
        for layer in self.layers:
            if layer["kind"] == "delta":
                layer["state"] = torch.zeros(sequences, self.H, self.d, self.d, device="cuda")
            else:
                layer["cache"] = dn.deltanet_paged_cache(sequences * pages, page, self.Hkv, self.d, torch.float8_e4m3fn)
        # every layer's cache has the same pages; a server would hand them out as sequences grow
        self.table = torch.randperm(sequences * pages, device="cuda").to(torch.int32).view(sequences, pages)
        self.lengths = [0] * sequences

    def step(self, x, new):
        """x [sum(new), width]: the next new[n] tokens of every sequence n; returns the layers' output for them."""
        import paper_2406_06484_amd as dn
        torch, H, Hkv, d = self.torch, self.H, self.Hkv, self.d
        self.lengths = [a + b for a, b in zip(self.lengths, new)]
        offsets = [0]
        for n in new:
            offsets.append(offsets[-1] + n)
        cu, kv_len = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in (offsets, self.lengths))
        T = x.shape[0]
        for layer in self.layers:
            h = torch.nn.functional.rms_norm(x.float(), (x.shape[1],)).to(x.dtype)
            row = h @ layer["w_in"]
            if layer["kind"] == "delta":
                q, k, v = (t.reshape(T, H, d).contiguous() for t in row[:, :3 * H * d].split(H * d, 1))
                o, layer["state"] = dn.deltanet_fused_fwd(q, k, v, row[:, 3 * H * d:].contiguous(), layer["state"], cu_seqlens=cu,
                                                          cu_seqlens_host=offsets)
            else:
                q, k, v = (t.unflatten(1, (-1, d)) for t in row.split([H * d, Hkv * d, Hkv * d], 1))   # rows of the projection: no copies
                k_pages, v_pages, k_scale, v_scale = layer["cache"]
                held = dict(k_scale=k_scale, v_scale=v_scale)
                q = dn.deltanet_paged_norm_rope_append(q, k, v, k_pages, v_pages, self.table, kv_len, cu, layer["q_weight"], layer["k_weight"],
                                                       self.rope, **held)
                o = dn.deltanet_paged_attn_fwd(q, k_pages, v_pages, self.table, kv_len, cu, window=self.window, max_q=max(new),
                                               max_kv=max(self.lengths), **held)
            x = x + o.reshape(T, H * d) @ layer["w_out"]
        return x


def run(layers=4, heads=4, head_size=64, window=256, prompts=(700, 130, 1, 333), chunk=256, tokens=40):
    """Serves the prompts in chunks and `tokens` single steps; returns (largest difference to one piece, relative; us per single step)."""
    import torch
    total = [p + tokens for p in prompts]
    model = Hybrid(layers, heads, head_size, window, len(prompts), max(total))
    g = torch.Generator(device="cuda").manual_seed(1)
    x = [torch.randn(n, heads * head_size, generator=g, device="cuda").to(torch.bfloat16) for n in total]
    out, at = [[] for _ in prompts], [0] * len(prompts)
    while any(a < p for a, p in zip(at, prompts)):
        new = [min(chunk, p - a) for a, p in zip(at, prompts)]     # sequences whose prompt is done wait with no new token
        y = model.step(torch.cat([x[n][a:a + m] for n, (a, m) in enumerate(zip(at, new))]), new)
        for n, part in enumerate(y.split(new)):
            out[n].append(part)
        at = [a + m for a, m in zip(at, new)]
    torch.cuda.synchronize()
    began = time.perf_counter()
    for _ in range(tokens):
        y = model.step(torch.stack([x[n][a] for n, a in enumerate(at)]), [1] * len(prompts))
        for n in range(len(prompts)):
            out[n].append(y[n:n + 1])
        at = [a + 1 for a in at]
    torch.cuda.synchronize()
    each = (time.perf_counter() - began) / max(tokens, 1) * 1e6
    model.reset(len(prompts), max(total))
    want = model.step(torch.cat(x), total)
    got = torch.cat([torch.cat(parts) for parts in out])
    return float((got.float() - want.float()).norm() / want.float().norm()), each


def main() -> int:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--heads", type=int, default=4)
    ap.add_argument("--head-size", type=int, default=64)
    ap.add_argument("--window", type=int, default=256)
    ap.add_argument("--tokens", type=int, default=40)
    args = ap.parse_args()
    import torch
    if not torch.cuda.is_available():
        print("example_hybrid: no GPU visible; there is no CPU fallback", file=sys.stderr)
        return 2
    off, each = run(args.layers, args.heads, args.head_size, args.window, tokens=args.tokens)
    print("chunks and single tokens against one piece: relative difference %.2e; %.0f us per step of %d layers" % (off, each, args.layers))
    return 0


if __name__ == "__main__":
    sys.exit(main())
