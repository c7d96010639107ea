"""Plain statements in 64 bits of what the operators around a mixer compute, and the bounds that their arithmetic keeps, on the CPU.  Every function takes and
returns float64 tensors; nothing of the library is used.  Each returns values with how far fp32 arithmetic and one rounding to the output's type may be from them."""
import torch

from tests.attention_reference import E32, HALF

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def act(kind, g):
    """(factor, derivative, bound of either's error): the exponential of an fp32 product is off by |g| + 2 roundings, the reciprocal by two more, and the
    derivative of g s(g) multiplies 1 - s, off by some roundings of one, by g.  The reciprocal of 1 + exp(-g) gives zero in the place of a number under the least normal
    one, 2^-126: s is off by as much then (g < -87), and g s by |g| of it"""
    s = torch.sigmoid(g)
    err = (g.abs() + 16) * E32
    if kind == "sigmoid":
        return s, s * (1 - s), err * s + 2 ** -126, 2 * err
    return g * s, s * (1 + g * (1 - s)), err * (g * s).abs() + g.abs() * 2 ** -126, err * (2 + g.abs())


def lines(x, state, lens, W):
    """every sequence's rows behind the W - 1 rows of its state (zeros where there is none)"""
    out, at = [], 0
    for n, m in enumerate(lens):
        past = state[n] if state is not None else torch.zeros(W - 1, x.shape[1], dtype=x.dtype)
        out.append(torch.cat([past, x[at:at + m]]))
        at += m
    return out


def taps(line, w):
    """sums over the W taps at every row of a sequence"""
    W = w.shape[1]
    return sum(w[:, j] * line[j:len(line) - (W - 1) + j] for j in range(W))


def conv(x, w, b, state, lens, on, dtype):
    """x [T, C], on: whether SiLU is applied, per channel; ((y, bound), final state)"""
    W, ys, bounds, last = w.shape[1], [], [], []
    for line in lines(x, state, lens, W):
        z = taps(line, w) + (b if b is not None else 0.0)
        ez = (W + 2) * E32 * (taps(line.abs(), w.abs()) + (b.abs() if b is not None else 0.0))
        f, _, ef, _ = act("silu", z)
        y = torch.where(on, f, z)
        ys.append(y)
        bounds.append(HALF[dtype] * y.abs() + 1.2 * torch.where(on, 1.1 * ez + ef, ez))
        last.append(line[len(line) - (W - 1):])
    return (torch.cat(ys), torch.cat(bounds)), torch.stack(last) if last else torch.zeros(0, W - 1, x.shape[1], dtype=x.dtype)


def conv_grad(x, w, b, state, lens, on, dy, dlast, dtype):
    """((dx, bound), (dw, bound), (db, bound), (dstate, bound))"""
    W, C = w.shape[1], x.shape[1]
    dx, ex, ds, es = [], [], [], []
    sums = [torch.zeros(C, W, dtype=torch.float64) for _ in range(2)] + [torch.zeros(C, dtype=torch.float64) for _ in range(2)]
    at, rows = 0, sum(lens)
    for n, line in enumerate(lines(x, state, lens, W)):
        m = lens[n]
        g = dy[at:at + m]
        at += m
        z = taps(line, w) + (b if b is not None else 0.0)
        ez = (W + 2) * E32 * (taps(line.abs(), w.abs()) + (b.abs() if b is not None else 0.0))
        _, d, _, ed = act("silu", z)
        dz = torch.where(on, g * d, g)
        edz = torch.where(on, g.abs() * (ez + ed) + 2 * E32 * dz.abs(), torch.zeros(()).double())
        back = lambda t, v: sum(v[:, j] * torch.nn.functional.pad(t, (0, 0, j, W - 1 - j)) for j in range(W))  # noqa: E731  (rows of the line, the state's first)
        de, err = back(dz, w), back(edz, w.abs()) + (W + 2) * E32 * back(dz.abs(), w.abs())
        if dlast is not None:
            de[m:] += dlast[n]
            err[m:] += 2 * E32 * (dlast[n].abs() + de[m:].abs())
        err = err + HALF[dtype] * de.abs()
        dx.append(de[W - 1:])
        ex.append(err[W - 1:])
        ds.append(de[:W - 1])
        es.append(err[:W - 1])
        for j in range(W):
            part = line[j:j + m]
            sums[0][:, j] += (dz * part).sum(0)
            sums[1][:, j] += ((edz + (rows + 8) * E32 * dz.abs()) * part.abs()).sum(0)
        sums[2] += dz.sum(0)
        sums[3] += (edz + (rows + 8) * E32 * dz.abs()).sum(0)
    whole = lambda v: torch.cat(v) if v else torch.zeros(0, C, dtype=torch.float64)  # noqa: E731
    states = lambda v: torch.stack(v) if v else torch.zeros(0, W - 1, C, dtype=torch.float64)  # noqa: E731
    return (whole(dx), whole(ex)), (sums[0], sums[1]), (sums[2], sums[3]), (states(ds), states(es))


def rms(x, eps):
    return 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)


def out_norm(o, g, w, eps, kind, dtype):
    d = o.shape[-1]
    n = o * rms(o, eps) * (w if w is not None else 1.0)
    f, _, ef, _ = act(kind, g) if g is not None else (torch.ones(()).double(), 0, torch.zeros(()).double(), 0)
    y = n * f
    return y, HALF[dtype] * y.abs() + 1.2 * ((d + 16) * E32 * y.abs() + n.abs() * ef)


def out_norm_grad(o, g, w, eps, kind, dy, dtype):
    """((do, bound), (dgate, bound) or None, (dw, bound))"""
    d, rows = o.shape[-1], o.shape[0] * o.shape[1]
    r = rms(o, eps)
    n, ww = o * r, w if w is not None else torch.ones(()).double()
    f, df, ef, edf = act(kind, g) if g is not None else (torch.ones(()).double(), None, torch.zeros(()).double(), None)
    a, ea = dy * f, dy.abs() * ef
    dn = a * ww
    do = r * (dn - n * (dn * n).mean(-1, keepdim=True))
    size = lambda t: r * (t + n.abs() * (t * n.abs()).mean(-1, keepdim=True))  # noqa: E731
    edo = HALF[dtype] * do.abs() + 1.2 * ((2 * d + 32) * E32 * size(dn.abs()) + size(ea * ww.abs()))
    dg = None
    if g is not None:
        v = dy * n * ww * df
        dg = (v, HALF[dtype] * v.abs() + 1.2 * ((d + 16) * E32 * v.abs() + (dy * n * ww).abs() * edf))
    dw, edw = (a * n).sum((0, 1)), ((ea + a.abs() * (d + 16 + rows) * E32) * n.abs()).sum((0, 1))
    return (do, edo), dg, (dw, 1.2 * edw)


def block_norm(x, res, w, u, post, scale, keep, eps, dtype, stream):
    """((y, bound), (h, bound))"""
    D = x.shape[-1]
    m = x * rms(x, eps) if post else x
    part = scale * (u if u is not None else 1.0) * m
    h = part + (keep * res if res is not None else 0.0)
    eh = (D + 20 if post else 4) * E32 * part.abs() + (4 * E32 * (keep * res).abs() if res is not None else 0.0)
    r = rms(h, eps)
    y = h * r * (w if w is not None else 1.0)
    ey = r * eh * (w.abs() if w is not None else 1.0) + y.abs() * ((D + 16) * E32 + r * r * (h.abs() * eh).mean(-1, keepdim=True))
    return (y, HALF[dtype] * y.abs() + 1.2 * ey), (h, HALF[stream] * h.abs() + 1.2 * eh)


def block_norm_grad(dy, dh, h, x, w, u, post, scale, keep, eps, dtype, stream):
    """((dx, bound), (dresidual, bound), (dw, bound), (du, bound))"""
    T, D = h.shape
    r = rms(h, eps)
    q, dz = h * r, dy * (w if w is not None else 1.0)
    H = r * (dz - q * (dz * q).mean(-1, keepdim=True)) + (dh if dh is not None else 0.0)
    step = (2 * D + 64) * E32
    size = r * (dz.abs() + q.abs() * (dz * q).abs().mean(-1, keepdim=True)) + (dh.abs() if dh is not None else 0.0)
    eH = step * size
    dres = keep * H
    f = scale * (u if u is not None else torch.ones(()).double())
    b, eb = f * H, f.abs() * (eH + 4 * E32 * size)
    m = x if x is not None else torch.zeros(()).double()
    dx, ex = b, eb
    if post:
        rx = rms(x, eps)
        m = x * rx
        dx = rx * (b - m * (b * m).mean(-1, keepdim=True))
        spread = lambda t: rx * (t + m.abs() * (t * m.abs()).mean(-1, keepdim=True))  # noqa: E731
        ex = spread(eb) + step * spread((f * H).abs() + eb)
    dw, edw = (dy * q).sum(0), (dy.abs() * q.abs()).sum(0) * (D + 32 + T) * E32
    du, edu = scale * (H * m).sum(0), abs(scale) * (((eH + size * (D + 32 + T) * E32) * m.abs()).sum(0))
    return (dx, HALF[dtype] * dx.abs() + 1.2 * ex), (dres, HALF[stream] * dres.abs() + 1.2 * abs(keep) * (eH + 4 * E32 * size)), (dw, 1.2 * edw), (du, 1.2 * edu)
