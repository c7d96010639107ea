"""The work between the matrix products of a hybrid model's step that ``perf/operators.py`` does not hold, as plain cases: what is
called, on which sizes, and the same results from elementary torch operations and from the definitions in 64 bits.

    op      "conv"        the short causal convolution of q, k and v in front of a DeltaNet mixer (deltanet_short_conv_fwd, _bwd)
            "out_norm"    RMS norm of every head's output with its gate, behind the mixer (deltanet_out_norm_fwd, _bwd)
            "block_norm"  what stands between two blocks: the branch's norm, gate and scale, the residual sum, the norm in front of the next
                          block (deltanet_block_norm_fwd, _bwd)
            "kv4"         serving: new keys and values appended to a paged cache of 4-bit numbers, and attention over it or the cache read back
                          (deltanet_paged_append, deltanet_paged_attn_fwd, deltanet_paged_read)
    mode    "train": forward and backward; "serve": forward, with the states that generation carries
    dtype   element type of the tensors; stream: of the residual stream
    N, q    sequences and tokens of the longest; lens: "same", "ragged" (packed, 1 to q tokens) or, for "kv4", as in ``perf/operators.py``
    kv      tokens of the longest context, the new ones included; page: tokens of a page; window: how many tokens a query sees (0: its whole past)
    back    how much of the cache is read back: "none", "new" (the tokens just written) or "all"

Sizes are those of ``synth.CONFIGS``, ``bench.py`` and ``perf/cases.py`` (model width 2048 in heads of 64, 128 or 256, batches of 8 x 2048
tokens) or generic.
"""
from __future__ import annotations

import math
import random

import torch

own = False

EPS = 1e-6
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # magnitudes of a 4-bit number (e2m1), by their code
GROUP = 32                                          # numbers that share a factor


def _conv(name=None, *, N, q, parts, W=4, dtype="bf16", mode="train", lens="same", bias=False, states=False):
    """parts: widths of q, k and v, each followed by s where SiLU is applied ("2048,2048,2048s")"""
    c = dict(op="conv", mode=mode, dtype=dtype, N=N, q=q, parts=parts, W=W, lens=lens, bias=bias, states=states)
    return dict(c, name=name) if name else c


def _out(name=None, *, N, q, H, d, dtype="bf16", mode="train", act="silu"):
    c = dict(op="out_norm", mode=mode, dtype=dtype, N=N, q=q, H=H, d=d, act=act)
    return dict(c, name=name) if name else c


def _block(name=None, *, N, q, D, dtype="bf16", stream="bf16", mode="train", gate=False, post=False, scale=1.0, keep=1.0):
    c = dict(op="block_norm", mode=mode, dtype=dtype, stream=stream, N=N, q=q, D=D, gate=gate, post=post, scale=scale, keep=keep)
    return dict(c, name=name) if name else c


def _kv4(name=None, *, N, q, kv, Hq, Hkv, d, page=64, window=0, lens="same", attend=True, back="none"):
    c = dict(op="kv4", N=N, q=q, kv=kv, Hq=Hq, Hkv=Hkv, d=d, page=page, window=window, lens=lens, attend=attend, back=back)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest training step: fp32, a narrow layer over short packed sequences, three taps, bias and states; launches and latency
        _conv("conv_f32_small", N=3, q=100, parts="128,128,136s", W=3, dtype="f32", lens="ragged", bias=True, states=True),
        # the training step of a DeltaNet layer of the 1.3B width on the benchmark's batch, q, k and v side by side
        _conv("conv_train", N=8, q=2048, parts="2048,2048,2048s"),
        # one generated token for each of 32 sequences, the last inputs carried along
        _conv("conv_decode_b32", N=32, q=1, parts="2048,2048,2048s", mode="serve", states=True),
        # the mixer's output on the benchmark's batch
        _out("out_norm_train", N=8, q=2048, H=16, d=128),
        # ... and for one generated token of 32 sequences
        _out("out_norm_decode_b32", N=32, q=1, H=16, d=128, mode="serve"),
        # between two blocks on the benchmark's batch, the stream in the tensors' type
        _block("block_norm_train", N=8, q=2048, D=2048),
        # a wider model with normed and gated branches over a scaled stream in fp32, an odd number of rows
        _block("block_norm_post_f32", N=3, q=1367, D=4104, stream="f32", gate=True, post=True, scale=0.5, keep=0.875),
        # one generated token of 32 sequences
        _block("block_norm_decode_b32", N=32, q=1, D=2048, mode="serve"),
        # one generated token for each of 32 sequences over contexts of up to 8192, four query heads to a key head
        _kv4("kv4_decode_b32", N=32, q=1, kv=8192, Hq=16, Hkv=4, d=128, lens="ragged"),
        # generation behind one very long document
        _kv4("kv4_decode_long", N=1, q=1, kv=131072, Hq=16, Hkv=4, d=128, page=128),
        # whole prompts, and the cache handed on (to another server, or to a layer that wants it contiguous)
        _kv4("kv4_prompts", N=4, q=2048, kv=2048, Hq=16, Hkv=4, d=128, back="all"),
        # continuous batching in a sliding-window layer: chunks beside single tokens, small pages, half-size heads
        _kv4("kv4_mixed_window", N=24, q=256, kv=4096, Hq=32, Hkv=8, d=64, page=16, window=1024, lens="mixed"),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng: random.Random):
    op = rng.choice(["conv", "conv", "out_norm", "block_norm", "block_norm", "kv4", "kv4", "kv4"])
    f32 = rng.random() < 0.2
    dtype = "f32" if f32 else "bf16"
    serve = rng.random() < 0.35
    mode = "serve" if serve else "train"
    most = 1 << (24 if f32 else 25)     # elements of a tensor
    if op == "conv":
        count = rng.choice([1, 2, 3, 3])
        parts = [8 * _log_int(rng, 4, 256) for _ in range(count)]
        C = sum(parts)
        T = _log_int(rng, 1, 128) if serve else _log_int(rng, 16, min(16384, 2 * most // C))
        N = min(T, rng.choice([1, 2, 5, 8, T]) if serve else rng.choice([1, 2, 5, 8]))
        return _conv(N=N, q=max(1, T // N), parts=",".join("%d%s" % (p, rng.choice(["", "s"])) for p in parts), W=rng.choice([2, 3, 4, 4]), dtype=dtype,
                     mode=mode, lens=rng.choice(["same", "ragged"]), bias=rng.random() < 0.4, states=serve or rng.random() < 0.3)
    if op == "out_norm":
        d, H = rng.choice([32, 64, 64, 128, 128, 256]), _log_int(rng, 1, 32)
        T = _log_int(rng, 1, 64 if serve else min(16384, most // (H * d)))
        N = min(T, rng.choice([1, 2, 5]))
        return _out(N=N, q=max(1, T // N), H=H, d=d, dtype=dtype, mode=mode, act=rng.choice(["silu", "silu", "sigmoid", "none"]))
    if op == "block_norm":
        D = 8 * _log_int(rng, 8, 1024)
        T = _log_int(rng, 1, 64 if serve else min(16384, most // D))
        N = min(T, rng.choice([1, 2, 5]))
        plain = rng.random() < 0.4
        return _block(N=N, q=max(1, T // N), D=D, dtype=dtype, stream="f32" if f32 else rng.choice(["bf16", "f32"]), mode=mode, gate=not plain and rng.random() < 0.6,
                      post=not plain and rng.random() < 0.6, scale=1.0 if plain else rng.choice([1.0, 0.5, 0.22]), keep=1.0 if plain else rng.choice([1.0, 0.875]))
    d = rng.choice([64, 128, 128, 256])
    Hkv = min(2048 // d, rng.choice([1, 2, 3, 4, 4, 8, 16]))
    Hq = Hkv * rng.choice([1, 1, 2, 4])
    page = rng.choice([16, 16, 32, 64, 64, 128, 256])
    window = rng.choice([0, 0, 0, _log_int(rng, 16, 4096)])
    if rng.random() < 0.55:     # generation: one token or a few
        q, N = rng.choice([1, 1, 1, 2, 4, 7]), _log_int(rng, 1, 64)
        kv = _log_int(rng, max(q, 30), max(64, min(131072, (1 << 27) // (N * Hkv * d))))
    else:                       # chunks: at most the products of the largest listed case
        q = _log_int(rng, 8, 2048)
        kv = max(q, _log_int(rng, q, 16384))
        kv = min(kv, max(q, 4 * 16 * 2048 * 2048 * 128 // (Hq * q * d)))
        N = rng.randint(1, max(1, min(16, int(4 * 16 * 2048 * 2048 * 128 / (Hq * q * kv * d)))))
    attend = rng.random() < 0.85
    back = rng.choice(["none", "none", "new", "all"]) if N * kv * Hkv * d <= 1 << 25 else rng.choice(["none", "new"])
    return _kv4(N=N, q=q, kv=kv, Hq=Hq, Hkv=Hkv, d=d, page=page, window=window, lens=rng.choice(["same", "ragged", "ragged", "mixed"]),
                attend=attend or back == "none", back=back)


# --- the plan of a case: lengths and pages go by the case, values by the seed

def _lens(case):
    """(new tokens, context) of every sequence"""
    N, q, kv = case["N"], case["q"], case.get("kv", case["q"])
    rng = random.Random(N * 1000003 + q * 1009 + kv)
    if case.get("lens", "same") == "same":
        return [q] * N, [kv] * N
    qs = [q if n == 0 else 1 if case["lens"] == "mixed" and n % 2 else rng.randint(1, q) for n in range(N)]
    return qs, [kv if n == 0 else max(qs[n], rng.randint(max(1, kv // 4), kv)) for n in range(N)]


def _prefix(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _parts(case):
    """(widths, whether SiLU is applied) of the convolution's outputs"""
    names = case["parts"].split(",")
    return tuple(int(p.rstrip("s")) for p in names), tuple(p.endswith("s") for p in names)


def _torch_type(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _to_4_bits(x):
    """x [.., d] as a 4-bit cache holds it: (codes [.., d / 2], the first of two in the low half of a byte; factors' exponents [.., d / 32], 127 more)"""
    g = x.unflatten(-1, (-1, GROUP)).float()
    m, e = torch.frexp(g.abs().amax(-1))                # amax = m 2^e, 0.5 <= m < 1
    e = torch.where(m > 0.75, e - 2, e - 3)             # the least power of two of which six are enough
    e = torch.where(m > 0, e, 0)
    a = torch.ldexp(g.abs(), -e[..., None])             # (exact: a power of two)
    # the nearest level, halfway ones to the even code
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = (code + 8 * torch.signbit(g).int()).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).to(torch.uint8)


def _from_4_bits(codes, exponents):
    """the values that codes and exponents stand for, in fp32 (exact)"""
    level = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float32, device=codes.device)
    x = torch.stack([level[(codes & 15).int()], level[(codes >> 4).int()]], -1).flatten(-2)
    return torch.ldexp(x.unflatten(-1, (-1, GROUP)), exponents.int()[..., None] - 127).flatten(-2)


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device=dev)  # noqa: E731
    whole = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    qs, kvs = _lens(case)
    T, N = sum(qs), case["N"]
    st = dict(case=case)
    if case["op"] == "conv":
        td, W = _torch_type(case["dtype"]), case["W"]
        widths, _ = _parts(case)
        C = sum(widths)
        # the projections' output: q, k, v and the writing strengths' logits side by side in one row per token
        rows = rand(T, C + 16).to(td)[:, :C]
        dense = case["lens"] == "same"
        shape = (N, case["q"]) if dense else (T,)
        st["x"] = rows.unflatten(0, shape)
        st["cu"] = None if dense else whole(_prefix(qs))
        st["cu_host"] = None if dense else _prefix(qs)
        st["weight"] = (W ** -0.5 * rand(C, W)).to(td)
        st["bias"] = (0.1 * rand(C)).to(td) if case["bias"] else None
        st["initial"] = rand(N, W - 1, C).to(td) if case["states"] else None
        if case["mode"] == "train":
            st["dfinal"] = rand(N, W - 1, C).to(td) if case["states"] else None
            st["dy"] = tuple(rand(*shape, w).to(td) for w in widths)
        return st
    if case["op"] == "out_norm":
        td, H, d = _torch_type(case["dtype"]), case["H"], case["d"]
        st["o"] = (0.3 * rand(T, H, d)).to(td)
        # the gate: a column block of a projection's output
        st["gate"] = None if case["act"] == "none" else rand(T, 2 * H * d).to(td)[:, H * d:].unflatten(1, (H, d))
        st["weight"] = (1 + 0.1 * rand(d)).to(td)
        st["dy"] = rand(T, H, d).to(td) if case["mode"] == "train" else None
        return st
    if case["op"] == "block_norm":
        td, ts, D = _torch_type(case["dtype"]), _torch_type(case["stream"]), case["D"]
        st["x"], st["residual"] = rand(T, D).to(td), (2 * rand(T, D)).to(ts)
        st["weight"] = (1 + 0.1 * rand(D)).to(td)
        st["gate"] = (1 + 0.3 * rand(D)).to(td) if case["gate"] else None
        if case["mode"] == "train":
            st["dy"], st["dh"] = rand(T, D).to(td), rand(T, D).to(ts)
            st["h"] = _block_sum(st)[0].to(ts)      # the stream as the forward pass of the step left it
        return st
    # the cache: every sequence's pages anywhere in it, holding numbers that came from bf16 values
    page, Hq, Hkv, d = case["page"], case["Hq"], case["Hkv"], case["d"]
    pages = [-(-n // page) for n in kvs]
    total = sum(pages) + 3
    order = torch.randperm(total, generator=g, device=dev, dtype=torch.int32)
    table = torch.full((N, max(pages)), -1, dtype=torch.int32, device=dev)
    own_page = torch.arange(max(pages), device=dev)[None, :] < whole(pages)[:, None]
    table[own_page] = order[:sum(pages)]
    st.update(page_table=table, kv_len=whole(kvs), cu_q=whole(_prefix(qs)), max_q=max(qs), max_kv=max(kvs))
    for name in ("k", "v"):
        codes = torch.empty(total, Hkv, page, d // 2, dtype=torch.uint8, device=dev)
        exponents = torch.empty(total, Hkv, page, d // GROUP, dtype=torch.uint8, device=dev)
        some = max(1, (1 << 24) // (Hkv * page * d))
        for i in range(0, total, some):
            codes[i:i + some], exponents[i:i + some] = _to_4_bits(rand(min(some, total - i), Hkv, page, d).to(torch.bfloat16))
        st[name + "_pages"], st[name + "_scale"] = codes.view(torch.float4_e2m1fn_x2), exponents.view(torch.float8_e8m0fnu)
    row = rand(T, (Hq + 2 * Hkv) * d).to(torch.bfloat16)
    st["q"], st["k"], st["v"] = (x.unflatten(1, (-1, d)) for x in row.split([Hq * d, Hkv * d, Hkv * d], 1))
    back = kvs if case["back"] == "all" else qs
    st["cu_back"], st["back_rows"] = whole(_prefix(back)), sum(back)
    return st


# --- the plain forms, in 32 bits

def _tokens(cu, rows):
    """sequence of every row of a packed tensor"""
    return torch.searchsorted(cu[1:].long().contiguous(), torch.arange(rows, device=cu.device), right=True)


def _activate(z, widths, silu):
    return torch.cat([p * torch.sigmoid(p) if s else p for p, s in zip(z.split(widths, -1), silu)], -1)


def _conv_plain(st):
    case = st["case"]
    td, W, N = _torch_type(case["dtype"]), case["W"], case["N"]
    widths, silu = _parts(case)
    x = st["x"].float().flatten(0, -2)
    T, C = x.shape
    dev = x.device
    # every sequence's rows behind the W - 1 rows of its state
    cu = st["cu"].long() if st["cu"] is not None else torch.arange(N + 1, device=dev) * case["q"]
    at = torch.arange(T, device=dev) + (_tokens(cu, T) + 1) * (W - 1)
    front = (cu[:-1] + torch.arange(N, device=dev) * (W - 1))[:, None] + torch.arange(W - 1, device=dev)
    last = (cu[1:] + torch.arange(1, N + 1, device=dev) * (W - 1))[:, None] - torch.arange(W - 1, 0, -1, device=dev)
    ext = torch.zeros(T + N * (W - 1), C, device=dev)
    ext[at] = x
    if st["initial"] is not None:
        ext[front.flatten()] = st["initial"].float().flatten(0, 1)
    w = st["weight"].float()
    z = sum(w[:, j] * ext[j:len(ext) - (W - 1) + j] for j in range(W))[at - (W - 1)]
    if st["bias"] is not None:
        z = z + st["bias"].float()
    y = _activate(z, widths, silu)
    out = tuple(p.contiguous() for p in y.to(td).unflatten(0, st["x"].shape[:-1]).split(widths, -1))
    if case["mode"] == "serve":
        return out, ext[last].to(td)
    dy = torch.cat(st["dy"], -1).float().flatten(0, -2)
    g = torch.sigmoid(z)
    on = torch.cat([torch.full((n,), float(s), device=dev) for n, s in zip(widths, silu)])
    dz = dy * (1 + on * (g * (1 + z * (1 - g)) - 1))
    dext = torch.zeros(len(ext) + W - 1, C, device=dev)
    dext[at] = dz
    dw = torch.stack([(dext[W - 1:len(ext)] * ext[j:len(ext) - (W - 1) + j]).sum(0) for j in range(W)], 1)
    db = dz.sum(0) if st["bias"] is not None else None
    de = sum(w[:, j] * dext[W - 1 - j:len(ext) + W - 1 - j] for j in range(W))
    if st["dfinal"] is not None:
        de[last.flatten()] += st["dfinal"].float().flatten(0, 1)
    dx = de[at].to(td).view(st["x"].shape)
    return out, ext[last].to(td), dx, dw, db, de[front].to(td) if st["initial"] is not None else None


def _gate_plain(act, g):
    """(the gate's factor, its derivative)"""
    s = torch.sigmoid(g)
    return (s, s * (1 - s)) if act == "sigmoid" else (g * s, s * (1 + g * (1 - s)))


def _out_norm_plain(st):
    td, act = _torch_type(st["case"]["dtype"]), st["case"]["act"]
    o, w = st["o"].float(), st["weight"].float()
    r = torch.rsqrt((o * o).mean(-1, keepdim=True) + EPS)
    n = o * r
    f, df = (1.0, None) if act == "none" else _gate_plain(act, st["gate"].float())
    y = (n * w * f).to(td)
    if st["case"]["mode"] == "serve":
        return y
    a = st["dy"].float() * f
    dn = a * w
    do = (r * (dn - n * (dn * n).mean(-1, keepdim=True))).to(td)
    return y, do, None if act == "none" else (st["dy"].float() * n * w * df).to(td), (a * n).sum((0, 1))


def _block_sum(st):
    """(the new stream unrounded, the branch as it enters, 1 / RMS of the branch or None, the branch's factors)"""
    case, x = st["case"], st["x"].float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) if case["post"] else None
    n = x * r if case["post"] else x
    f = case["scale"] * (st["gate"].float() if case["gate"] else 1.0)
    return case["keep"] * st["residual"].float() + f * n, n, r, f


def _block_norm_plain(st):
    case = st["case"]
    td, ts = _torch_type(case["dtype"]), _torch_type(case["stream"])
    h, n, rx, f = _block_sum(st)
    w = st["weight"].float()
    y = (h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * w).to(td)
    if case["mode"] == "serve":
        return y, h.to(ts)
    kept, dy = st["h"].float(), st["dy"].float()
    r = torch.rsqrt((kept * kept).mean(-1, keepdim=True) + EPS)
    hhat = kept * r
    dz = dy * w
    dh = st["dh"].float() + r * (dz - hhat * (dz * hhat).mean(-1, keepdim=True))
    b = f * dh
    dx = (rx * (b - n * (b * n).mean(-1, keepdim=True)) if case["post"] else b).to(td)
    return y, h.to(ts), dx, (case["keep"] * dh).to(ts), (dy * hhat).sum(0), case["scale"] * (dh * n).sum(0) if case["gate"] else None


def _places(st, cu, rows):
    """(page, slot) of every row of a packed tensor whose sequences end where the contexts end; its sequence and position"""
    seq = _tokens(cu, rows)
    pos = st["kv_len"].long()[seq] - cu.long()[seq + 1] + torch.arange(rows, device=cu.device)
    page = st["case"]["page"]
    return st["page_table"].long()[seq, pos // page], pos % page, seq, pos


def _held(st, name):
    return st[name + "_pages"].view(torch.uint8), st[name + "_scale"].view(torch.uint8)


def _kv4_plain(st):
    case = st["case"]
    at, slot, seq, pos = _places(st, st["cu_q"], st["q"].shape[0])
    for name in ("k", "v"):
        codes, exponents = _held(st, name)
        codes[at, :, slot], exponents[at, :, slot] = _to_4_bits(st[name])
    out = ()
    if case["attend"]:
        # sequences padded to the longest chunk and the longest context
        N, Q, K, Hq, Hkv, d, dev = case["N"], st["max_q"], st["max_kv"], case["Hq"], case["Hkv"], case["d"], st["q"].device
        place = torch.arange(st["q"].shape[0], device=dev) - st["cu_q"].long()[seq]
        q = torch.zeros(N, Q, Hq, d, device=dev)
        q[seq, place] = st["q"].float()
        qpos = torch.full((N, Q), -1, dtype=torch.int64, device=dev)
        qpos[seq, place] = pos
        q = q.view(N, Q, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(N, Hkv, -1, d)
        table = st["page_table"].clamp(min=0).long()
        k, v = (_from_4_bits(*(t[table] for t in _held(st, name))).permute(0, 2, 1, 3, 4).reshape(N, Hkv, -1, d)[:, :, :K] for name in ("k", "v"))
        j = torch.arange(K, device=dev)
        live = j < st["kv_len"].long()[:, None]
        s = torch.matmul(q, k.transpose(2, 3)) / math.sqrt(d)
        seen = live[:, None, :] & (j <= qpos[..., None])
        if case["window"]:
            seen &= j > qpos[..., None] - case["window"]
        s = s.view(N, Hkv, Hq // Hkv, Q, K).masked_fill_(~seen[:, None, None], -torch.inf)
        s = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min))
        o = torch.matmul((s / s.sum(-1, keepdim=True).clamp(min=1e-30)).view(N, Hkv, -1, K), v)
        out += (o.view(N, Hq, Q, d)[seq, :, place].to(torch.bfloat16),)
    if case["back"] != "none":
        at, slot, _, _ = _places(st, st["cu_back"], st["back_rows"])
        out += tuple(_from_4_bits(*(t[at, :, slot] for t in _held(st, name))).to(torch.bfloat16) for name in ("k", "v"))
    return out


def _plain(st):
    return {"conv": _conv_plain, "out_norm": _out_norm_plain, "block_norm": _block_norm_plain, "kv4": _kv4_plain}[st["case"]["op"]](st)


# --- the framework's calls

def _calls(st):
    import paper_2406_06484_amd as dn
    case = st["case"]
    train = case.get("mode") == "train"
    if case["op"] == "conv":
        widths, silu = _parts(case)
        kw = dict(splits=widths, silu=silu, cu_seqlens=st["cu"], cu_seqlens_host=st["cu_host"])
        y, final = dn.deltanet_short_conv_fwd(st["x"], st["weight"], st["bias"], st["initial"], **kw)
        if not train:
            return y, final
        return (y, final) + dn.deltanet_short_conv_bwd(st["x"], st["weight"], st["dy"], st["bias"], st["initial"], st["dfinal"], **kw)
    if case["op"] == "out_norm":
        kw = dict(eps=EPS, act="silu" if case["act"] == "none" else case["act"])
        y = dn.deltanet_out_norm_fwd(st["o"], st["gate"], st["weight"], **kw)
        return (y,) + dn.deltanet_out_norm_bwd(st["o"], st["dy"], st["gate"], st["weight"], **kw) if train else y
    if case["op"] == "block_norm":
        kw = dict(gate=st["gate"], post_norm=case["post"], scale=case["scale"], residual_scale=case["keep"], eps=EPS)
        y, h = dn.deltanet_block_norm_fwd(st["x"], st["residual"], st["weight"], **kw)
        return (y, h) + dn.deltanet_block_norm_bwd(st["dy"], st["h"], st["x"], st["weight"], st["dh"], **kw) if train else (y, h)
    cache = (st["k_pages"], st["v_pages"], st["page_table"], st["kv_len"])
    scales = dict(k_scale=st["k_scale"], v_scale=st["v_scale"])
    dn.deltanet_paged_append(st["k"], st["v"], *cache, st["cu_q"], **scales)
    out = ()
    if case["attend"]:
        out += (dn.deltanet_paged_attn_fwd(st["q"], *cache, st["cu_q"], **scales, window=case["window"], max_q=st["max_q"], max_kv=st["max_kv"]),)
    if case["back"] != "none":
        out += tuple(dn.deltanet_paged_read(*cache, st["cu_back"], st["back_rows"], **scales))
    return out


def run(st):
    return _calls(st) if own else _plain(st)


# --- the definitions in 64 bits

def _exact_conv(st):
    case = st["case"]
    W, qs = case["W"], _lens(case)[0]
    widths, silu = _parts(case)
    leaf = lambda t: None if t is None else t.double().clone().requires_grad_()  # noqa: E731
    x, w, b, s0 = leaf(st["x"].flatten(0, -2)), leaf(st["weight"]), leaf(st["bias"]), leaf(st["initial"])
    ys, finals = [], []
    for n, rows in enumerate(x.split(qs)):
        past = s0[n] if s0 is not None else torch.zeros(W - 1, x.shape[1], dtype=torch.float64, device=x.device)
        line = torch.cat([past, rows])
        z = (line.unfold(0, W, 1) * w).sum(-1)                  # windows [rows, C, W]
        if b is not None:
            z = z + b
        ys.append(torch.cat([torch.nn.functional.silu(p) if s else p for p, s in zip(z.split(widths, 1), silu)], 1))
        finals.append(line[len(line) - (W - 1):])
    y, final = torch.cat(ys), torch.stack(finals)
    out = tuple(p.detach().unflatten(0, st["x"].shape[:-1]) for p in y.split(widths, 1))
    if case["mode"] == "serve":
        return out, final.detach()
    total = (y * torch.cat([d.flatten(0, -2) for d in st["dy"]], 1).double()).sum()
    if st["dfinal"] is not None:
        total = total + (final * st["dfinal"].double()).sum()
    leaves = [t for t in (x, w, b, s0) if t is not None]
    grads = dict(zip(map(id, leaves), torch.autograd.grad(total, leaves)))
    dx, dw, db, ds = (None if t is None else grads[id(t)] for t in (x, w, b, s0))
    return out, final.detach(), dx.view(st["x"].shape), dw, db, ds


def _rms(x):
    return x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS)


def _exact_out_norm(st):
    act = {"silu": torch.nn.functional.silu, "sigmoid": torch.sigmoid}.get(st["case"]["act"])
    o, w = st["o"].double().requires_grad_(), st["weight"].double().requires_grad_()
    g = None if act is None else st["gate"].double().requires_grad_()
    y = _rms(o) * w
    y = y if g is None else y * act(g)
    if st["case"]["mode"] == "serve":
        return y.detach()
    leaves = [t for t in (o, g, w) if t is not None]
    grads = torch.autograd.grad(y, leaves, st["dy"].double())
    return (y.detach(), grads[0], grads[1] if g is not None else None, grads[-1])


def _exact_block_norm(st):
    case = st["case"]
    x, w = st["x"].double().requires_grad_(), st["weight"].double().requires_grad_()
    u = st["gate"].double().requires_grad_() if case["gate"] else None
    branch = case["scale"] * (_rms(x) if case["post"] else x)
    branch = branch if u is None else branch * u
    h = case["keep"] * st["residual"].double() + branch.detach()
    y = _rms(h) * w.detach()
    if case["mode"] == "serve":
        return y, h
    kept = st["h"].double().requires_grad_()
    dh, dw = torch.autograd.grad(_rms(kept) * w, (kept, w), st["dy"].double())
    dh = dh + st["dh"].double()
    grads = torch.autograd.grad(branch, (x,) if u is None else (x, u), dh)
    return y, h, grads[0], case["keep"] * dh, dw, grads[1] if u is not None else None


def _exact_kv4(st):
    """Values are found again from the definition: the factor by its logarithm, the number by the distances to all that there are."""
    case, dev = st["case"], st["q"].device
    qs, kvs = _lens(case)
    page, Hkv, d, G = case["page"], case["Hkv"], case["d"], case["Hq"] // case["Hkv"]
    level = torch.tensor(LEVELS, dtype=torch.float64, device=dev)

    def rounded(x):
        g = x.double().unflatten(-1, (-1, GROUP))
        top = g.abs().amax(-1, keepdim=True)
        s = torch.exp2(torch.ceil(torch.log2(torch.where(top > 0, top, 6.0) / 6.0)))
        away = ((g / s).abs()[..., None] - level).abs()
        near = away.amin(-1, keepdim=True)
        tied = away == near
        even = tied & (torch.arange(8, device=dev) % 2 == 0)
        code = torch.where(tied.sum(-1) > 1, even.int().argmax(-1), tied.int().argmax(-1))
        return (torch.sign(g) * level[code] * s).flatten(-2)

    def past(name, n):      # [kv, Hkv, d] of sequence n, the new tokens last
        ids = st["page_table"][n, :-(-kvs[n] // page)].long()
        codes, exponents = (t[ids].transpose(1, 2).flatten(0, 1)[:kvs[n]] for t in _held(st, name))
        sign = torch.where(torch.arange(16, device=dev) < 8, 1.0, -1.0).double()
        value = level.repeat(2) * sign
        x = torch.stack([value[(codes % 16).long()], value[(codes // 16).long()]], -1).flatten(-2)
        x = (x.unflatten(-1, (-1, GROUP)) * torch.exp2(exponents.double() - 127)[..., None]).flatten(-2)
        lo = sum(qs[:n])
        new = torch.cat([rounded(r) for r in st[name][lo:lo + qs[n]].split(256)])
        return torch.cat([x[:kvs[n] - qs[n]], new])

    rows, read = [], ([], [])
    for n, (lo, m) in enumerate(zip(_prefix(qs), qs)):
        k, v = past("k", n), past("v", n)
        if case["back"] != "none":
            b = kvs[n] if case["back"] == "all" else m
            read[0].append(k[kvs[n] - b:])
            read[1].append(v[kvs[n] - b:])
        if case["attend"]:
            q = st["q"][lo:lo + m].double().unflatten(1, (-1, G)).permute(1, 2, 0, 3).flatten(1, 2)     # [Hkv, G m, d]
            dist = torch.arange(kvs[n] - m, kvs[n], device=dev)[:, None] - torch.arange(kvs[n], device=dev)
            hide = (dist < 0) | (dist >= case["window"] if case["window"] else dist < 0)
            s = (q @ k.permute(1, 2, 0).contiguous() * d ** -0.5).unflatten(1, (G, m)).masked_fill(hide, -math.inf)
            p = torch.softmax(s, -1).flatten(1, 2)
            rows.append((p @ v.transpose(0, 1).contiguous()).unflatten(1, (G, m)).permute(2, 0, 1, 3).flatten(1, 2))
    out = (torch.cat(rows),) if case["attend"] else ()
    return out + tuple(torch.cat(r) for r in read) if case["back"] != "none" else out


def exact(case, seed):
    st = prepare(case, seed)
    return {"conv": _exact_conv, "out_norm": _exact_out_norm, "block_norm": _exact_block_norm, "kv4": _exact_kv4}[case["op"]](st)


# --- what a pass cannot do without

def work(case):
    qs, kvs = _lens(case)
    T, N = sum(qs), case["N"]
    es = 4 if case.get("dtype") == "f32" else 2
    train = case.get("mode") == "train"
    if case["op"] == "conv":
        W, C = case["W"], sum(_parts(case)[0])
        states = (2 if case["states"] else 1) * N * (W - 1) * C * es
        small = C * (W + case["bias"]) * es
        by = 2 * T * C * es + states + small
        if train:       # x, the gradients in and out, states and weights again, and their gradients
            by += 3 * T * C * es + 2 * states + small + 4 * C * (W + case["bias"])
        return {"bytes": by, "flops": T * C * (2 * W + 4) * (4 if train else 1)}
    if case["op"] == "out_norm":
        row, gated = T * case["H"] * case["d"] * es, case["act"] != "none"
        by = row * (2 + gated) + case["d"] * es
        if train:
            by += row * (3 + 2 * gated) + case["d"] * (es + 4)
        return {"bytes": by, "flops": T * case["H"] * case["d"] * (30 if train else 10)}
    if case["op"] == "block_norm":
        row, stream = T * case["D"] * es, T * case["D"] * (4 if case["stream"] == "f32" else 2)
        vectors = case["D"] * es * (1 + case["gate"])
        by = 2 * row + 2 * stream + vectors
        if train:       # dy, dh, h (and the branch) in, both gradients out; one of them where they are the same
            same = not (case["gate"] or case["post"] or case["scale"] != 1 or case["keep"] != 1 or case["stream"] != case["dtype"])
            by += row * (1 + (case["gate"] or case["post"]) + (not same)) + 3 * stream + vectors + 4 * case["D"] * (1 + case["gate"])
        return {"bytes": by, "flops": T * case["D"] * (30 if train else 10)}
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    held = d // 2 + d // GROUP      # bytes of a token and head in the cache
    by, flops = 2 * T * Hkv * (2 * d + held), 8 * T * Hkv * d
    if case["attend"]:
        keys = pairs = 0
        for q, kv in zip(qs, kvs):
            w = case["window"] or kv
            keys += min(kv, w + q - 1)
            pairs += sum(min(p + 1, w) for p in range(kv - q, kv))
        by += 4 * T * Hq * d + 2 * keys * Hkv * held
        flops += 4 * pairs * Hq * d
    if case["back"] != "none":
        by += 2 * (sum(kvs) if case["back"] == "all" else T) * Hkv * (held + 2 * d)
    return {"bytes": by, "flops": flops}
