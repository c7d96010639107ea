"""The work of the attention layers that stand between DeltaNet layers in a hybrid model, as plain cases: what is called, on
which sizes, and the same results from elementary torch operations and from the definitions in 64 bits.

    op      "norm_rope"  training: RMS norm of every head's query and key with the position rotation, forward and backward
                         (deltanet_qk_norm_rope_fwd + deltanet_qk_norm_rope_bwd)
            "cache"      serving: that pass on the new tokens of a batch, with k and v quantised and written to the paged cache
                         as they leave it, and the cache read back (deltanet_paged_norm_rope_append + deltanet_paged_read)
            "attn"       serving: attention of the new tokens over the paged cache (deltanet_paged_attn_fwd)
    dtype   element type of q, k, v and of the outputs; cache: of the pages ("fp8": e4m3 with a scale per token and head)
    N       sequences; q: new tokens of the longest; kv: tokens of the longest context, the new ones included
    lens    "same": every sequence has q and kv tokens; "ragged": contexts from a quarter of kv up, chunks of 1 to q tokens;
            "mixed": the same, and every second sequence has one new token
    page    tokens of a page; window: how many tokens a query sees (0: its whole past); back: how many tokens "cache" reads back
            ("new": those just written, "all": the sequences)

Sizes are those of ``synth.CONFIGS``, ``bench.py`` and ``perf/cases.py`` (model width 2048 in heads of 64, 128 or 256, batches of 8 x 2048
tokens, sequences to 32768) or generic.
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-6
FP8_MAX = 448.0           # largest e4m3 value: a row's largest magnitude is scaled to it
THETA = 10000.0


def _nr(name=None, *, N, q, Hq, Hkv, d, dtype="bf16", rot=0, pairs="halves", lens="same"):
    c = dict(op="norm_rope", dtype=dtype, N=N, q=q, Hq=Hq, Hkv=Hkv, d=d, rot=rot or d, pairs=pairs, lens=lens)
    return dict(c, name=name) if name else c


def _cache(name=None, *, N, q, kv, Hq, Hkv, d, dtype="bf16", cache="fp8", page=64, back="new", rot=0, pairs="halves", lens="same"):
    c = dict(op="cache", dtype=dtype, cache=cache, N=N, q=q, kv=kv, Hq=Hq, Hkv=Hkv, d=d, page=page, back=back, rot=rot or d, pairs=pairs, lens=lens)
    return dict(c, name=name) if name else c


def _attn(name=None, *, N, q, kv, Hq, Hkv, d, dtype="bf16", cache="bf16", page=64, window=0, lens="same"):
    c = dict(op="attn", dtype=dtype, cache=cache, N=N, q=q, kv=kv, Hq=Hq, Hkv=Hkv, d=d, page=page, window=window, lens=lens)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest training step, fp32 heads of 64 over one short sequence: launches and latency
        _nr("norm_rope_f32_small", N=1, q=256, Hq=2, Hkv=2, d=64, dtype="f32"),
        # the training step of an attention layer of the 1.3B width on the benchmark's batch
        _nr("norm_rope_train", N=8, q=2048, Hq=16, Hkv=16, d=128),
        # a packed batch of odd lengths, double-size heads shared in pairs, half of each head rotated in neighbouring pairs
        _nr("norm_rope_packed_d256", N=5, q=1501, Hq=8, Hkv=4, d=256, rot=128, pairs="neighbours", lens="ragged"),
        # one generated token for each of 32 sequences into an 8-bit cache
        _cache("cache_decode_b32", N=32, q=1, kv=2048, Hq=16, Hkv=16, d=128, lens="ragged"),
        # prompts written to an 8-bit cache and handed on whole (to another server, or to a layer that wants them contiguous)
        _cache("cache_prompts_fp8", N=4, q=2048, kv=2048, Hq=16, Hkv=4, d=128, back="all"),
        # chunks of mixed sizes into a 16-bit cache of small pages, half-size heads
        _cache("cache_mixed_bf16", N=9, q=300, kv=1500, Hq=32, Hkv=8, d=64, cache="bf16", page=16, back="all", lens="mixed"),
        # the precision mode's small calls: a few tokens of two short sequences in fp32
        _attn("attn_f32_small", N=2, q=5, kv=120, Hq=2, Hkv=2, d=64, dtype="f32", cache="f32", page=16, lens="ragged"),
        # one generated token for each of 32 sequences, every head with a cache of its own
        _attn("attn_decode_b32", N=32, q=1, kv=2048, Hq=16, Hkv=16, d=128, lens="ragged"),
        # generation over one long document in an 8-bit cache that four query heads share
        _attn("attn_decode_long_fp8", N=1, q=1, kv=32768, Hq=16, Hkv=4, d=128, cache="fp8", page=128),
        # prefill: whole prompts at once
        _attn("attn_prompts", N=4, q=2048, kv=2048, Hq=16, Hkv=16, d=128),
        # one chunk of a long prompt
        _attn("attn_chunk_long", N=1, q=512, kv=16384, Hq=16, Hkv=4, d=128),
        # continuous batching in a sliding-window layer: chunks beside single tokens, small pages, 8 bits, half-size heads
        _attn("attn_mixed_window_fp8", N=24, q=256, kv=4096, Hq=32, Hkv=8, d=64, cache="fp8", page=16, window=1024, lens="mixed"),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _heads(rng, d):
    Hkv = rng.choice([1, 2, 3, 4, 4, 8, 16])
    return min(2048 // d, Hkv) * rng.choice([1, 1, 2, 4]), min(2048 // d, Hkv)


def draw(rng: random.Random):
    op = rng.choice(["norm_rope", "norm_rope", "cache", "cache", "cache", "attn", "attn", "attn", "attn", "attn"])
    f32 = rng.random() < 0.15
    dtype = "f32" if f32 else "bf16"
    d = rng.choice([32, 64, 64, 128]) if f32 else rng.choice([64, 128, 128, 256])
    Hq, Hkv = _heads(rng, d)
    page = rng.choice([16, 16, 32, 64, 64, 128, 256])
    if op == "norm_rope":
        most = 8 * 2048 * 32 * 128 // ((Hq + Hkv) * d * (2 if f32 else 1))  # rows that cost what the largest listed case costs
        T = _log_int(rng, 1, min(most, 16384))
        N = rng.choice([1, 1, 2, 5, 8])
        return _nr(N=min(N, T), q=max(1, T // min(N, T)), Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, rot=max(16, d // rng.choice([1, 1, 2])),
                   pairs=rng.choice(["halves", "halves", "neighbours"]), lens=rng.choice(["same", "ragged"]))
    cache = "f32" if f32 else rng.choice(["bf16", "fp8"])
    if op == "cache":
        N = _log_int(rng, 1, 64)
        q = 1 if rng.random() < 0.4 else _log_int(rng, 2, max(2, 8192 // N))
        kv = max(q, _log_int(rng, q, 4096))
        return _cache(N=N, q=q, kv=kv, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, cache=cache, page=page, rot=max(16, d // rng.choice([1, 1, 2])),
                      back="all" if N * kv * Hkv * d <= 1 << 25 and rng.random() < 0.5 else "new",
                      pairs=rng.choice(["halves", "halves", "neighbours"]), lens=rng.choice(["same", "ragged", "mixed"]))
    window = rng.choice([0, 0, 0, _log_int(rng, 16, 4096)])
    if rng.random() < 0.5:  # generation: one token or a few
        q, N = rng.choice([1, 1, 1, 2, 4, 7]), _log_int(rng, 1, 64)
        kv = _log_int(rng, max(q, 30), max(64, min(32768, (1 << 27) // (N * Hkv * d))))
    else:                   # chunks: at most the products of the largest listed case
        q = _log_int(rng, 8, 2048) if not f32 else _log_int(rng, 8, 300)
        kv = max(q, _log_int(rng, q, 16384 if not f32 else 2000))
        N = max(1, min(16, int(4 * 16 * 2048 * 2048 * 128 / (Hq * q * kv * d))))
        kv = min(kv, max(q, 4 * 16 * 2048 * 2048 * 128 // (Hq * q * N * d)))
        N = rng.randint(1, N)
    return _attn(N=N, q=q, kv=kv, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype, cache=cache, page=page, window=window,
                 lens=rng.choice(["same", "ragged", "ragged", "mixed"]))


# --- the plan of a case: lengths and pages go by the case, values by the seed

def _lens(case):
    """(new tokens, context) of every sequence"""
    N, q, kv = case["N"], case["q"], case.get("kv", case["q"])
    rng = random.Random(N * 1000003 + q * 1009 + kv)
    if case["lens"] == "same":
        return [q] * N, [kv] * N
    qs = [q if n == 0 else 1 if case["lens"] == "mixed" and n % 2 else rng.randint(1, q) for n in range(N)]
    return qs, [kv if n == 0 else max(qs[n], rng.randint(max(1, kv // 4), kv)) for n in range(N)]


def _back(case):
    """how many of its last tokens are read back of every sequence"""
    qs, kvs = _lens(case)
    return kvs if case["back"] == "all" else qs


def _prefix(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _torch_type(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}[name]


def _e4m3(x):
    """a row's values and scale as an 8-bit cache holds them"""
    amax = x.abs().amax(-1)
    scale = amax / FP8_MAX
    return (x / torch.where(scale > 0, scale, 1.0)[..., None]).to(torch.float8_e4m3fn), scale


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device=dev)  # noqa: E731
    whole = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    td, d, Hq, Hkv = _torch_type(case["dtype"]), case["d"], case["Hq"], case["Hkv"]
    qs, kvs = _lens(case)
    T = sum(qs)
    st = dict(case=case, cu_q=whole(_prefix(qs)), max_q=max(qs), max_kv=max(kvs))
    if case["op"] != "attn":
        # the projections' output, q, k and v side by side in one row per token; RMS weights near 1; the rotation's table
        row = rand(T, (Hq + 2 * Hkv) * d).to(td)
        st["q"], st["k"], st["v"] = (x.unflatten(1, (-1, d)) for x in row.split([Hq * d, Hkv * d, Hkv * d], 1))
        st["q_weight"], st["k_weight"] = (1 + 0.1 * rand(d)).to(td), (1 + 0.1 * rand(d)).to(td)
        half = case["rot"] // 2
        freq = THETA ** (-torch.arange(half, device=dev, dtype=torch.float64) / half)
        angle = torch.arange(max(kvs), device=dev, dtype=torch.float64)[:, None] * freq
        st["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    if case["op"] == "norm_rope":
        st["positions"] = torch.cat([torch.arange(n, dtype=torch.int32, device=dev) for n in qs])
        st["dq_out"], st["dk_out"] = rand(T, Hq, d).to(td), rand(T, Hkv, d).to(td)
        return st
    # the cache: every sequence's pages anywhere in it
    page = case["page"]
    pages = [-(-n // page) for n in kvs]
    total = sum(pages) + 3
    order = torch.randperm(total, generator=g, device=dev, dtype=torch.int32)
    table = torch.full((case["N"], max(pages)), -1, dtype=torch.int32, device=dev)
    own_page = torch.arange(max(pages), device=dev)[None, :] < whole(pages)[:, None]
    table[own_page] = order[:sum(pages)]
    st["page_table"], st["kv_len"] = table, whole(kvs)
    for name in ("k", "v"):
        x = rand(total, Hkv, page, d)
        if case["cache"] == "fp8":
            st[name + "_pages"], st[name + "_scale"] = _e4m3(x)
        else:
            st[name + "_pages"], st[name + "_scale"] = x.to(_torch_type(case["cache"])), None
    if case["op"] == "cache":
        back = _back(case)
        st["cu_back"], st["back_rows"] = whole(_prefix(back)), sum(back)
    else:
        st["q"] = rand(T, Hq, d).to(td)
    return st


# --- the plain forms, in 32 bits

def _norm_rope_plain(st, x, weight, positions):
    """(unrounded result, normalised rows, 1 / RMS)"""
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    xhat = x * r
    return _rotate(st, xhat * weight.float(), positions, 1.0), xhat, r


def _rotate(st, y, positions, sign):
    rot = st["case"]["rot"]
    cos, sin = (t[:, None, :] for t in st["rope"][positions.long()].split(rot // 2, 1))
    head, rest = y[..., :rot], y[..., rot:]
    if st["case"]["pairs"] == "halves":
        a, b = head.split(rot // 2, -1)
        return torch.cat([a * cos - sign * b * sin, b * cos + sign * a * sin, rest], -1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat([torch.stack([a * cos - sign * b * sin, b * cos + sign * a * sin], -1).flatten(-2), rest], -1)


def _norm_rope_grad_plain(st, dy, xhat, r, weight, positions, td):
    dz = _rotate(st, dy.float(), positions, -1.0)
    dw = (dz * xhat).sum((0, 1))
    dxhat = dz * weight.float()
    return (r * (dxhat - xhat * (dxhat * xhat).mean(-1, keepdim=True))).to(td), dw


def _tokens(st, cu, rows):
    """(sequence, position in it) of every row of a packed tensor whose sequences end where the contexts end"""
    row = torch.arange(rows, device=cu.device)
    seq = torch.searchsorted(cu[1:].contiguous(), row, right=True)
    return seq, st["kv_len"].long()[seq] - cu.long()[seq + 1] + row


def _write_plain(st, name, x, seq, pos):
    page = st["case"]["page"]
    at = st["page_table"].long()[seq, pos // page]
    pages = st[name + "_pages"]
    if st["case"]["cache"] == "fp8":
        values, scale = _e4m3(x)
        pages.view(torch.uint8)[at, :, pos % page] = values.view(torch.uint8)
        st[name + "_scale"][at, :, pos % page] = scale
    else:
        pages[at, :, pos % page] = x.to(pages.dtype)


def _read_plain(st, name, at, slot):
    x = st[name + "_pages"][at, :, slot].float() if st["case"]["cache"] != "fp8" else st[name + "_pages"].view(torch.uint8)[at, :, slot].view(torch.float8_e4m3fn).float()
    return x * st[name + "_scale"][at, :, slot][..., None] if st["case"]["cache"] == "fp8" else x


def _plain(st):
    case, td = st["case"], _torch_type(st["case"]["dtype"])
    if case["op"] == "norm_rope":
        q, qhat, qr = _norm_rope_plain(st, st["q"], st["q_weight"], st["positions"])
        k, khat, kr = _norm_rope_plain(st, st["k"], st["k_weight"], st["positions"])
        dq, dwq = _norm_rope_grad_plain(st, st["dq_out"], qhat, qr, st["q_weight"], st["positions"], td)
        dk, dwk = _norm_rope_grad_plain(st, st["dk_out"], khat, kr, st["k_weight"], st["positions"], td)
        return q.to(td), k.to(td), dq, dk, dwq, dwk
    if case["op"] == "cache":
        seq, pos = _tokens(st, st["cu_q"], st["q"].shape[0])
        q = _norm_rope_plain(st, st["q"], st["q_weight"], pos)[0].to(td)
        _write_plain(st, "k", _norm_rope_plain(st, st["k"], st["k_weight"], pos)[0], seq, pos)
        _write_plain(st, "v", st["v"].float(), seq, pos)
        seq, pos = _tokens(st, st["cu_back"], st["back_rows"])
        at, slot = st["page_table"].long()[seq, pos // case["page"]], pos % case["page"]
        return q, _read_plain(st, "k", at, slot).to(td), _read_plain(st, "v", at, slot).to(td)
    # attention: sequences padded to the longest chunk and the longest context
    N, Q, K, Hq, Hkv, d, dev = case["N"], st["max_q"], st["max_kv"], case["Hq"], case["Hkv"], case["d"], st["q"].device
    seq, pos = _tokens(st, st["cu_q"], st["q"].shape[0])
    place = torch.arange(st["q"].shape[0], device=dev) - st["cu_q"].long()[seq]
    q = torch.zeros(N, Q, Hq, d, device=dev)
    q[seq, place] = st["q"].float()
    qpos = torch.full((N, Q), -1, dtype=torch.int64, device=dev)
    qpos[seq, place] = pos
    q = q.view(N, Q, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(N, Hkv, -1, d)
    at = st["page_table"].clamp(min=0).long()
    kv = []
    for name in ("k", "v"):
        x = (st[name + "_pages"].view(torch.uint8)[at].view(torch.float8_e4m3fn) if case["cache"] == "fp8" else st[name + "_pages"][at]).float()
        if case["cache"] == "fp8":
            x = x * st[name + "_scale"][at][..., None]
        kv.append(x.permute(0, 2, 1, 3, 4).reshape(N, Hkv, -1, d)[:, :, :K])
    j = torch.arange(K, device=dev)
    live = (j < st["kv_len"].long()[:, None])
    v = torch.where(live[:, None, :, None], kv[1], 0.0)
    s = torch.matmul(q, kv[0].transpose(2, 3)) / math.sqrt(d)
    seen = live[:, None, :] & (j <= qpos[..., None])
    if case["window"]:
        seen &= j > qpos[..., None] - case["window"]
    s = s.view(N, Hkv, Hq // Hkv, Q, K).masked_fill_(~seen[:, None, None], -torch.inf)
    s = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
    o = torch.matmul((s / s.sum(-1, keepdim=True).clamp(min=1e-30)).view(N, Hkv, -1, K), v)
    return o.view(N, Hq, Q, d)[seq, :, place].to(td)


# --- the framework's calls

def _calls(st):
    import paper_2406_06484_amd as dn
    case = st["case"]
    if case["op"] == "attn":
        return dn.deltanet_paged_attn_fwd(st["q"], st["k_pages"], st["v_pages"], st["page_table"], st["kv_len"], st["cu_q"], k_scale=st["k_scale"],
                                          v_scale=st["v_scale"], window=case["window"], max_q=st["max_q"], max_kv=st["max_kv"])
    rope = dict(eps=EPS, interleaved=case["pairs"] == "neighbours")
    w = (st["q_weight"], st["k_weight"], st["rope"])
    if case["op"] == "norm_rope":
        q, k = dn.deltanet_qk_norm_rope_fwd(st["q"], st["k"], *w, st["positions"], **rope)
        return (q, k) + dn.deltanet_qk_norm_rope_bwd(st["q"], st["k"], st["dq_out"], st["dk_out"], *w, st["positions"], **rope)
    cache = (st["k_pages"], st["v_pages"], st["page_table"], st["kv_len"])
    scales = dict(k_scale=st["k_scale"], v_scale=st["v_scale"])
    q = dn.deltanet_paged_norm_rope_append(st["q"], st["k"], st["v"], *cache, st["cu_q"], *w, **scales, **rope)
    return (q,) + dn.deltanet_paged_read(*cache, st["cu_back"], st["back_rows"], dtype=st["q"].dtype, **scales)


def run(st):
    return _calls(st) if own else _plain(st)


# --- the definitions in 64 bits

def _exact_norm_rope(st, x, weight, positions):
    rot = st["case"]["rot"]
    y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight
    t = st["rope"].double()[positions.long()]
    turn = torch.complex(t[:, :rot // 2], t[:, rot // 2:])[:, None, :]
    head = y[..., :rot]
    if st["case"]["pairs"] == "halves":
        z = torch.complex(head[..., :rot // 2], head[..., rot // 2:]) * turn
        return torch.cat([z.real, z.imag, y[..., rot:]], -1)
    z = torch.view_as_complex(head.unflatten(-1, (-1, 2)).contiguous()) * turn
    return torch.cat([torch.view_as_real(z).flatten(-2), y[..., rot:]], -1)


def exact(case, seed):
    st = prepare(case, seed)
    qs, kvs = _lens(case)
    wide = lambda t: t.double()  # noqa: E731
    if case["op"] == "norm_rope":
        out, grads, weights = [], [], []
        for n, dy in (("q", st["dq_out"]), ("k", st["dk_out"])):
            x, w = wide(st[n]).clone().requires_grad_(), wide(st[n + "_weight"]).clone().requires_grad_()
            y = _exact_norm_rope(st, x, w, st["positions"])
            dx, dw = torch.autograd.grad(y, (x, w), wide(dy))
            out.append(y.detach()), grads.append(dx), weights.append(dw)
        return tuple(out + grads + weights)
    held = {}
    for name in ("k", "v"):
        x = wide(st[name + "_pages"].float())
        held[name] = x * wide(st[name + "_scale"])[..., None] if case["cache"] == "fp8" else x

    def past(name, n):  # [kv, Hkv, d] of sequence n
        ids = st["page_table"][n, :-(-kvs[n] // case["page"])].long()
        return held[name][ids].transpose(1, 2).reshape(-1, case["Hkv"], case["d"])[:kvs[n]]

    if case["op"] == "cache":
        pos = torch.cat([torch.arange(kv - q, kv, device=st["q"].device) for q, kv in zip(qs, kvs)])
        q = _exact_norm_rope(st, wide(st["q"]), wide(st["q_weight"]), pos)
        new = dict(k=_exact_norm_rope(st, wide(st["k"]), wide(st["k_weight"]), pos), v=wide(st["v"]))
        read = []
        for name in ("k", "v"):
            rows = []  # (what the cache held before, and the new rows as they would be without the rounding to the pages' type)
            for n, (lo, m) in enumerate(zip(_prefix(qs), _back(case))):
                rows.append(torch.cat([past(name, n)[:kvs[n] - qs[n]], new[name][lo:lo + qs[n]]])[kvs[n] - m:])
            read.append(torch.cat(rows))
        return (q,) + tuple(read)
    G, rows = case["Hq"] // case["Hkv"], []
    for n, (lo, m) in enumerate(zip(_prefix(qs), qs)):
        k, v = (past(name, n).permute(1, 2, 0) for name in ("k", "v"))                       # [Hkv, d, kv]
        q = wide(st["q"][lo:lo + m]).unflatten(1, (-1, G)).permute(1, 2, 0, 3).flatten(1, 2)     # [Hkv, G m, d]
        dist = torch.arange(kvs[n] - m, kvs[n], device=q.device)[:, None] - torch.arange(kvs[n], device=q.device)
        hide = (dist < 0) | (dist >= case["window"] if case["window"] else dist < 0)
        s = (q @ k.contiguous() * case["d"] ** -0.5).unflatten(1, (G, m)).masked_fill(hide, -math.inf)
        p = torch.softmax(s, -1).flatten(1, 2)
        rows.append((p @ v.transpose(1, 2).contiguous()).unflatten(1, (G, m)).permute(2, 0, 1, 3).flatten(1, 2))
    return torch.cat(rows)


# --- what a pass cannot do without

def work(case):
    qs, kvs = _lens(case)
    T, d, Hq, Hkv = sum(qs), case["d"], case["Hq"], case["Hkv"]
    es = 4 if case["dtype"] == "f32" else 2
    row = T * (Hq + Hkv) * d * es
    if case["op"] == "norm_rope":
        # q, k in and out, then q, k and the gradients in and out; weights, table and positions
        return {"bytes": 5 * row + 2 * (4 * T + 4 * max(qs) * case["rot"]) + 4 * d * es + 8 * d, "flops": 30 * T * (Hq + Hkv) * d}
    held = d * {"f32": 4, "bf16": 2, "fp8": 1}[case["cache"]] + (4 if case["cache"] == "fp8" else 0)  # bytes of a token and head in the cache
    if case["op"] == "cache":
        back = sum(_back(case))
        by = T * (Hq + 2 * Hkv) * d * es + T * Hq * d * es + 2 * T * Hkv * held + 4 * min(T, max(kvs)) * case["rot"]
        return {"bytes": by + 2 * back * Hkv * (held + d * es), "flops": 12 * T * (Hq + 2 * Hkv) * d}
    keys = pairs = 0
    for q, kv in zip(qs, kvs):
        w = case["window"] or kv
        keys += min(kv, w + q - 1)
        pairs += sum(min(p + 1, w) for p in range(kv - q, kv))
    return {"bytes": 2 * T * Hq * d * es + 2 * keys * Hkv * held, "flops": 4 * pairs * Hq * d}
