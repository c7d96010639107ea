// The operators around a mixer (short convolution, output norm, block norm) in the Python module `_attention`: their C ABI called with tensors.  Work and memory belong to the tensors' device, whichever
// is the current one.
#include <ATen/core/DimVector.h>

#include <vector>

#include "dn_binding.hpp"

namespace {

using namespace dn_binding;

struct Lib {
    decltype(&deltanet_short_conv_fwd) conv_fwd;
    decltype(&deltanet_short_conv_workspace_bytes) conv_bytes;
    decltype(&deltanet_short_conv_bwd) conv_bwd;
    decltype(&deltanet_out_norm_fwd) out_fwd;
    decltype(&deltanet_out_norm_workspace_bytes) out_bytes;
    decltype(&deltanet_out_norm_bwd) out_bwd;
    decltype(&deltanet_block_norm_fwd) block_fwd;
    decltype(&deltanet_block_norm_workspace_bytes) block_bytes;
    decltype(&deltanet_block_norm_bwd) block_bwd;
} lib;

void together(const at::Tensor &with, std::initializer_list<const at::Tensor *> ts) {
    for (const at::Tensor *t : ts)
        if (t && t->device() != with.device()) throw Refusal{PyExc_ValueError, "all tensors must be on one device"};
}

// elements between the rows of t [T, C] or [B, L, C], whose elements are contiguous
int64_t row_step(const at::Tensor &t, const char *name, at::ScalarType type, at::IntArrayRef shape) {
    on_device(t, name, type, shape);
    const int64_t n = t.dim(), C = t.size(n - 1);
    if (t.stride(n - 1) != 1 && C > 1) throw Refusal{PyExc_ValueError, std::string(name) + " must be contiguous within its rows"};
    const int64_t L = t.size(n - 2), B = n == 3 ? t.size(0) : 1;
    if (B > 1 && L > 1 && t.stride(0) != L * t.stride(1)) throw Refusal{PyExc_ValueError, std::string(name) + " must have evenly spaced rows"};
    return L > 1 ? t.stride(n - 2) : B > 1 ? t.stride(0) : C;
}

bool truth(PyObject *o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) throw Refusal{nullptr, ""}; // (the object's own error)
    return v != 0;
}

// the items of a sequence
struct Items {
    PyObject *seq;
    Items(PyObject *o, const char *what) : seq(PySequence_Fast(o, what)) { if (!seq) throw Refusal{nullptr, ""}; }
    ~Items() { Py_DECREF(seq); }
    Items(const Items &) = delete;
    Py_ssize_t size() const { return PySequence_Fast_GET_SIZE(seq); }
    PyObject *operator[](Py_ssize_t i) const { return PySequence_Fast_GET_ITEM(seq, i); }
};

// --- short convolution

struct Conv {
    dn_conv_shape s = {};
    at::Tensor copy;
    std::vector<int32_t> host;
    at::ScalarType type;
    at::DimVector lead; // leading sizes of x
    int64_t sequences = 0;
    bool split;
    Conv(const at::Tensor &x, const at::Tensor &w, PyObject *splits, PyObject *silu, PyObject *cu_, PyObject *cu_host) : split(splits != Py_None) {
        const at::Tensor *cu = maybe(cu_, "cu_seqlens");
        s.dtype = type_of(x, "x");
        type = x.scalar_type();
        if (x.dim() != (cu ? 2 : 3)) throw Refusal{PyExc_ValueError, "x must be [B, L, C], or [T, C] with cu_seqlens"};
        const int64_t n = x.dim(), C = x.size(n - 1);
        lead.append(x.sizes().begin(), x.sizes().end() - 1);
        s.x_stride = row_step(x, "x", type, x.sizes());
        s.B = cu ? 1 : int32(x.size(0), "B"); s.L = int32(x.size(n - 2), "L"); s.C = int32(C, "C");
        if (w.dim() != 2) throw Refusal{PyExc_ValueError, "weight must be [C, W]"};
        whole(w, "weight", type, {C, w.size(1)});
        s.W = int32(w.size(1), "W");
        sequences = s.B;
        if (cu) {
            whole(*cu, "cu_seqlens", at::kInt, cu->sizes());
            if (cu->dim() != 1 || cu->size(0) < 1) throw Refusal{PyExc_ValueError, "cu_seqlens must be [sequences + 1]"};
            together(x, {cu});
            sequences = cu->size(0) - 1;
            s.num_seqs = int32(sequences, "sequences");
            s.cu_seqlens = ints(*cu, copy);
            if (cu_host != Py_None) {
                const Items at(cu_host, "cu_seqlens_host must be a sequence of integers");
                if (at.size() != sequences + 1) throw Refusal{PyExc_ValueError, "cu_seqlens_host must have the shape of cu_seqlens"};
                host.resize(at.size());
                for (Py_ssize_t i = 0; i < at.size(); ++i) {
                    const long long v = PyLong_AsLongLong(at[i]);
                    if (v == -1 && PyErr_Occurred()) throw Refusal{nullptr, ""};
                    host[i] = int32(v, "cu_seqlens_host");
                }
                s.cu_seqlens_host = host.data();
            }
        }
        if (split) {
            const Items at(splits, "splits must be a sequence of widths");
            if (at.size() < 1 || at.size() > 3) throw Refusal{PyExc_ValueError, "splits must hold one to three widths"};
            s.parts = (int32_t)at.size();
            for (int i = 0; i < s.parts; ++i) s.width[i] = int32(integer(at[i], "splits"), "splits");
        } else {
            s.parts = 1;
            s.width[0] = s.C;
        }
        if (PyBool_Check(silu)) {
            for (int i = 0; i < s.parts; ++i) s.silu[i] = silu == Py_True;
        } else {
            const Items at(silu, "silu must be a truth value, or one for each part");
            if (at.size() != s.parts) throw Refusal{PyExc_ValueError, "silu must be a truth value, or one for each part"};
            for (int i = 0; i < s.parts; ++i) s.silu[i] = truth(at[i]);
        }
    }
    at::DimVector shape(int64_t C) const {
        at::DimVector v(lead);
        v.push_back(C);
        return v;
    }
    at::DimVector states() const { return {sequences, s.W - 1, s.C}; }
    // the tensors of the parts (given as one tensor where there is one part without splits)
    void parts(PyObject *given, const char *name, const at::Tensor &x, bool make, at::Tensor (&t)[3], void *(&p)[3]) const {
        for (int i = 0; i < s.parts; ++i) if (s.width[i] < 0) throw Refusal{PyExc_ValueError, "splits must be widths"};
        if (given == Py_None) {
            if (!make) throw Refusal{PyExc_TypeError, std::string(name) + " must be a tensor"};
            for (int i = 0; i < s.parts; ++i) t[i] = fresh(shape(s.width[i]), x, type);
        } else if (!split) {
            t[0] = tensor(given, name);
            whole(t[0], name, type, shape(s.C));
        } else {
            const Items at(given, "a sequence of the parts' tensors is wanted");
            if (at.size() != s.parts) throw Refusal{PyExc_ValueError, std::string(name) + " must hold a tensor for each part"};
            for (int i = 0; i < s.parts; ++i) {
                t[i] = tensor(at[i], name);
                whole(t[i], name, type, shape(s.width[i]));
            }
        }
        for (int i = 0; i < s.parts; ++i) {
            together(x, {&t[i]});
            p[i] = t[i].data_ptr();
        }
    }
};

PyObject *conv_fwd(Args a) {
    const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "weight"), *b = maybe(a[2], "bias"), *s0 = maybe(a[3], "initial_state"), *given = maybe(a[10], "final_state");
    Conv c(x, w, a[4], a[5], a[6], a[7]);
    const c10::DeviceGuard on(x.device());
    together(x, {&w, b, s0, given});
    if (b) whole(*b, "bias", c.type, {c.s.C});
    if (s0) whole(*s0, "initial_state", c.type, c.states());
    at::Tensor y[3], last;
    void *p[3] = {};
    c.parts(a[9], "y", x, true, y, p);
    const bool want = given || truth(a[8]);
    if (want) last = out(given, "final_state", c.states(), x, c.type);
    const int rc = lib.conv_fwd(&c.s, x.data_ptr(), w.data_ptr(), ptr(b), ptr(s0), p, want ? last.data_ptr() : nullptr, stream_of(x));
    if (rc) return PyLong_FromLong(rc);
    PyObject *ys = !c.split ? THPVariable_Wrap(y[0]) : c.s.parts == 1 ? tuple_of({&y[0]}) : c.s.parts == 2 ? tuple_of({&y[0], &y[1]}) : tuple_of({&y[0], &y[1], &y[2]});
    PyObject *ls = want ? THPVariable_Wrap(last) : Py_NewRef(Py_None), *r = ys && ls ? PyTuple_Pack(2, ys, ls) : nullptr;
    Py_XDECREF(ys);
    Py_XDECREF(ls);
    return r;
}

PyObject *conv_bwd(Args a) {
    const at::Tensor &x = tensor(a[0], "x"), &w = tensor(a[1], "weight"), *b = maybe(a[3], "bias"), *s0 = maybe(a[4], "initial_state"), *dsT = maybe(a[5], "dfinal_state");
    const at::Tensor *gx = maybe(a[10], "dx"), *gw = maybe(a[11], "dweight"), *gb = maybe(a[12], "dbias"), *gs = maybe(a[13], "dinitial_state"), *ws = maybe(a[14], "workspace");
    Conv c(x, w, a[6], a[7], a[8], a[9]);
    const c10::DeviceGuard on(x.device());
    together(x, {&w, b, s0, dsT, gx, gw, gb, gs, ws});
    if (b) whole(*b, "bias", c.type, {c.s.C});
    if (s0) whole(*s0, "initial_state", c.type, c.states());
    if (dsT) whole(*dsT, "dfinal_state", c.type, c.states());
    if (gb && !b) throw Refusal{PyExc_ValueError, "no gradient of a bias that is not there"};
    at::Tensor dy[3], dx, dw, db, ds0;
    void *p[3] = {};
    c.parts(a[2], "dy", x, false, dy, p);
    dx = gx ? *gx : fresh(x.sizes(), x, c.type);
    c.s.dx_stride = row_step(dx, "dx", c.type, x.sizes());
    dw = out(gw, "dweight", w.sizes(), x, at::kFloat);
    if (b) db = out(gb, "dbias", {c.s.C}, x, at::kFloat);
    const bool states = s0 || gs;
    if (states) ds0 = out(gs, "dinitial_state", c.states(), x, c.type);
    size_t need = 0;
    int rc = lib.conv_bytes(&c.s, &need);
    if (rc) return PyLong_FromLong(rc);
    const Scratch scratch(ws, need, x);
    rc = lib.conv_bwd(&c.s, x.data_ptr(), w.data_ptr(), p, ptr(b), ptr(s0), ptr(dsT), dx.data_ptr(), fptr(&dw), b ? fptr(&db) : nullptr,
                      states ? ds0.data_ptr() : nullptr, scratch.p(), scratch.bytes, stream_of(x));
    return rc ? PyLong_FromLong(rc) : tuple_of({&dx, &dw, b ? &db : nullptr, states ? &ds0 : nullptr});
}

// --- output norm

// [T, H, d] or [B, L, H, d] as [rows, H, d]
at::Tensor heads(const at::Tensor &t, const char *name) {
    if (t.dim() == 4) return flat(t, name);
    if (t.dim() != 3) throw Refusal{PyExc_ValueError, std::string(name) + " must be [T, heads, d] or [B, L, heads, d]"};
    return t;
}

struct Out {
    dn_out_norm_shape s = {};
    at::ScalarType type;
    Out(const at::Tensor &o, const at::Tensor *gate, const at::Tensor *w, PyObject *eps, PyObject *act) {
        s.dtype = type_of(o, "o");
        type = o.scalar_type();
        const at::Tensor x = heads(o, "o");
        s.T = int32(x.size(0), "T"); s.H = int32(x.size(1), "heads"); s.d = int32(x.size(2), "d");
        s.o_stride = rows(x, "o", type, s.T, s.H, s.d);
        if (gate) {
            on_device(*gate, "gate", type, o.sizes());
            s.gate_stride = rows(heads(*gate, "gate"), "gate", type, s.T, s.H, s.d);
        }
        if (w) whole(*w, "weight", type, {s.d});
        s.eps = (float)number(eps, "eps");
        s.act = int32(integer(act, "act"), "act");
    }
};

PyObject *out_fwd(Args a) {
    const at::Tensor &o = tensor(a[0], "o"), *gate = maybe(a[1], "gate"), *w = maybe(a[2], "weight"), *gy = maybe(a[5], "y");
    const Out x(o, gate, w, a[3], a[4]);
    const c10::DeviceGuard on(o.device());
    together(o, {gate, w, gy});
    const at::Tensor y = out(gy, "y", o.sizes(), o, x.type);
    const int rc = lib.out_fwd(&x.s, o.data_ptr(), ptr(gate), ptr(w), y.data_ptr(), stream_of(o));
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(y);
}

PyObject *out_bwd(Args a) {
    const at::Tensor &o = tensor(a[0], "o"), &dy = tensor(a[1], "dy"), *gate = maybe(a[2], "gate"), *w = maybe(a[3], "weight");
    const at::Tensor *go = maybe(a[6], "d_o"), *gg = maybe(a[7], "dgate"), *gw = maybe(a[8], "dweight"), *ws = maybe(a[9], "workspace");
    Out x(o, gate, w, a[4], a[5]);
    const c10::DeviceGuard on(o.device());
    together(o, {&dy, gate, w, go, gg, gw, ws});
    whole(dy, "dy", x.type, o.sizes());
    if (gg && !gate) throw Refusal{PyExc_ValueError, "no gradient of a gate that is not there"};
    if (gw && !w) throw Refusal{PyExc_ValueError, "no gradient of a weight that is not there"};
    const at::Tensor d_o = out(go, "d_o", o.sizes(), o, x.type);
    at::Tensor dg, dw;
    if (gate) {
        dg = gg ? *gg : fresh(o.sizes(), o, x.type);
        on_device(dg, "dgate", x.type, o.sizes());
        x.s.dgate_stride = rows(heads(dg, "dgate"), "dgate", x.type, x.s.T, x.s.H, x.s.d);
    }
    if (w) dw = out(gw, "dweight", {x.s.d}, o, at::kFloat);
    size_t need = 0;
    int rc = lib.out_bytes(&x.s, &need);
    if (rc) return PyLong_FromLong(rc);
    const Scratch scratch(ws, w ? need : 0, o);
    rc = lib.out_bwd(&x.s, o.data_ptr(), dy.data_ptr(), ptr(gate), ptr(w), d_o.data_ptr(), gate ? dg.data_ptr() : nullptr, w ? fptr(&dw) : nullptr, scratch.p(), scratch.bytes, stream_of(o));
    return rc ? PyLong_FromLong(rc) : tuple_of({&d_o, gate ? &dg : nullptr, w ? &dw : nullptr});
}

// --- block norm

struct Block {
    dn_block_norm_shape s = {};
    at::ScalarType type, stream;
    // `like`: a tensor of the rows' sizes and of the elements' type; `held`: one of the stream's, if there is any
    Block(const at::Tensor &like, const char *name, const at::Tensor *held, const char *held_name, const at::Tensor *w, const at::Tensor *gate, PyObject *post, PyObject *scale, PyObject *keep, PyObject *eps) {
        s.dtype = type_of(like, name);
        type = like.scalar_type();
        if (like.dim() != 2 && like.dim() != 3) throw Refusal{PyExc_ValueError, std::string(name) + " must be [T, D] or [B, L, D]"};
        s.stream_dtype = held ? type_of(*held, held_name) : s.dtype;
        stream = held ? held->scalar_type() : type;
        if (stream != type && stream != at::kFloat) throw Refusal{PyExc_TypeError, std::string(held_name) + " must have the tensors' type or be float32"};
        const int64_t n = like.dim();
        s.T = int32(n == 3 ? like.size(0) * like.size(1) : like.size(0), "rows");
        s.D = int32(like.size(n - 1), "D");
        if (w) whole(*w, "weight", type, {s.D});
        if (gate) whole(*gate, "gate", type, {s.D});
        s.post_norm = truth(post);
        s.scale = (float)number(scale, "scale");
        s.residual_scale = (float)number(keep, "residual_scale");
        s.eps = (float)number(eps, "eps");
    }
};

PyObject *block_fwd(Args a) {
    const at::Tensor &x = tensor(a[0], "x"), *res = maybe(a[1], "residual"), *w = maybe(a[2], "weight"), *gate = maybe(a[3], "gate"), *gy = maybe(a[8], "y"), *gh = maybe(a[9], "h");
    Block k(x, "x", res ? res : gh, res ? "residual" : "h", w, gate, a[4], a[5], a[6], a[7]);
    const c10::DeviceGuard on(x.device());
    together(x, {res, w, gate, gy, gh});
    k.s.x_stride = row_step(x, "x", k.type, x.sizes());
    if (res) k.s.residual_stride = row_step(*res, "residual", k.stream, x.sizes());
    const at::Tensor y = out(gy, "y", x.sizes(), x, k.type);
    // without a residual, norm, gate or scale the stream is the branch itself, unless y takes its place or its rows are apart (the backward pass takes a contiguous one)
    const bool same = !res && !gh && !gate && !k.s.post_norm && k.s.scale == 1.f && x.is_contiguous() && !(gy && gy->data_ptr() == x.data_ptr());
    const at::Tensor h = same ? x : out(gh, "h", x.sizes(), x, k.stream);
    const int rc = lib.block_fwd(&k.s, x.data_ptr(), ptr(res), ptr(w), ptr(gate), y.data_ptr(), same ? nullptr : h.data_ptr(), stream_of(x));
    return rc ? PyLong_FromLong(rc) : tuple_of({&y, &h});
}

PyObject *block_bwd(Args a) {
    const at::Tensor &dy = tensor(a[0], "dy"), &h = tensor(a[1], "h"), *x = maybe(a[2], "x"), *w = maybe(a[3], "weight"), *dh = maybe(a[4], "dh"), *gate = maybe(a[5], "gate");
    const at::Tensor *gx = maybe(a[11], "dx"), *gr = maybe(a[12], "dresidual"), *gw = maybe(a[13], "dweight"), *gg = maybe(a[14], "dgate"), *ws = maybe(a[15], "workspace");
    Block k(dy, "dy", &h, "h", w, gate, a[6], a[7], a[8], a[9]);
    const c10::DeviceGuard on(dy.device());
    together(dy, {&h, x, w, dh, gate, gx, gr, gw, gg, ws});
    whole(dy, "dy", k.type, dy.sizes());
    whole(h, "h", k.stream, dy.sizes());
    if (dh) whole(*dh, "dh", k.stream, dy.sizes());
    const bool branch = k.s.post_norm || gate;
    if (branch) {
        if (!x) throw Refusal{PyExc_ValueError, "x is needed with post_norm or a gate"};
        k.s.x_stride = row_step(*x, "x", k.type, dy.sizes());
    }
    if (gw && !w) throw Refusal{PyExc_ValueError, "no gradient of a weight that is not there"};
    if (gg && !gate) throw Refusal{PyExc_ValueError, "no gradient of a gate that is not there"};
    const bool want = gr || truth(a[10]);
    // one tensor where both gradients are the same numbers
    const bool same = want && !gx && !gr && !branch && k.s.scale == k.s.residual_scale && k.type == k.stream;
    const at::Tensor dx = out(gx, "dx", dy.sizes(), dy, k.type);
    at::Tensor dr, dw, dg;
    if (want) dr = same ? dx : out(gr, "dresidual", dy.sizes(), dy, k.stream);
    if (w) dw = out(gw, "dweight", {k.s.D}, dy, at::kFloat);
    if (gate) dg = out(gg, "dgate", {k.s.D}, dy, at::kFloat);
    size_t need = 0;
    int rc = lib.block_bytes(&k.s, &need);
    if (rc) return PyLong_FromLong(rc);
    const Scratch scratch(ws, w || gate ? need : 0, dy);
    rc = lib.block_bwd(&k.s, dy.data_ptr(), ptr(dh), h.data_ptr(), branch ? ptr(x) : nullptr, ptr(w), ptr(gate), dx.data_ptr(), want && !same ? dr.data_ptr() : nullptr,
                       w ? fptr(&dw) : nullptr, gate ? fptr(&dg) : nullptr, scratch.p(), scratch.bytes, stream_of(dy));
    return rc ? PyLong_FromLong(rc) : tuple_of({&dx, want ? &dr : nullptr, w ? &dw : nullptr, gate ? &dg : nullptr});
}

} // namespace

namespace dn_binding {
extern const Symbol layer_symbols[];
extern PyMethodDef layer_methods[];

const Symbol layer_symbols[] = {
    {"deltanet_short_conv_fwd", (void **)&lib.conv_fwd}, {"deltanet_short_conv_workspace_bytes", (void **)&lib.conv_bytes}, {"deltanet_short_conv_bwd", (void **)&lib.conv_bwd},
    {"deltanet_out_norm_fwd", (void **)&lib.out_fwd}, {"deltanet_out_norm_workspace_bytes", (void **)&lib.out_bytes}, {"deltanet_out_norm_bwd", (void **)&lib.out_bwd},
    {"deltanet_block_norm_fwd", (void **)&lib.block_fwd}, {"deltanet_block_norm_workspace_bytes", (void **)&lib.block_bytes}, {"deltanet_block_norm_bwd", (void **)&lib.block_bwd},
    {nullptr, nullptr}};
PyMethodDef layer_methods[] = {ENTRY("short_conv_fwd", conv_fwd, 11), ENTRY("short_conv_bwd", conv_bwd, 15), ENTRY("out_norm_fwd", out_fwd, 6),
                               ENTRY("out_norm_bwd", out_bwd, 10), ENTRY("block_norm_fwd", block_fwd, 10), ENTRY("block_norm_bwd", block_bwd, 16),
                               {nullptr, nullptr, 0, nullptr}};
} // namespace dn_binding
