// Python module `_attention`: the attention operators' C ABI (include/deltanet.h) called with tensors.  Checks of arguments, outputs and workspaces
// that the caller did not bring, the current stream: what attention.py would do, at a fraction of the interpreter's time (a call of
// deltanet_paged_attn_fwd costs the host 10 us through ctypes; a decode step makes some tens of such calls, each of a few
// microseconds on the device).  Every function returns its result, or the negative dn_status of the call as an integer.
#include <Python.h>

#include <ATen/ATen.h>
#include <dlfcn.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <initializer_list>
#include <sstream>
#include <string>

#include "../../include/deltanet.h"

namespace {

// The library's entry points, found once in the file that the package names.
struct Lib {
    decltype(&deltanet_qk_norm_rope_fwd) norm_rope_fwd;
    decltype(&deltanet_qk_norm_rope_workspace_bytes) norm_rope_bytes;
    decltype(&deltanet_qk_norm_rope_bwd) norm_rope_bwd;
    decltype(&deltanet_paged_append) append;
    decltype(&deltanet_paged_norm_rope_append) norm_rope_append;
    decltype(&deltanet_paged_read) read;
    decltype(&deltanet_paged_attn_workspace_bytes) attn_bytes;
    decltype(&deltanet_paged_attn_fwd) attn;
} lib;
PyObject *g_raw_stream = nullptr; // device index -> handle of its current stream

struct Refusal { PyObject *type; std::string text; };

std::string text_of(at::IntArrayRef s) {
    std::ostringstream o;
    o << '(';
    for (size_t i = 0; i < s.size(); ++i) o << (i ? ", " : "") << s[i];
    o << ')';
    return o.str();
}

const at::Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) throw Refusal{PyExc_TypeError, std::string(name) + " must be a tensor"};
    return THPVariable_Unpack(o);
}
const at::Tensor *maybe(PyObject *o, const char *name) { return o == Py_None ? nullptr : &tensor(o, name); }

void on_device(const at::Tensor &t, const char *name, at::ScalarType type, at::IntArrayRef shape) {
    if (!t.is_cuda()) throw Refusal{PyExc_ValueError, std::string(name) + " must be a device tensor"};
    if (t.scalar_type() != type) throw Refusal{PyExc_TypeError, std::string(name) + " must be " + at::toString(type) + ", got " + at::toString(t.scalar_type())};
    if (t.sizes() != shape) throw Refusal{PyExc_ValueError, std::string(name) + " must have shape " + text_of(shape) + ", got " + text_of(t.sizes())};
}
void whole(const at::Tensor &t, const char *name, at::ScalarType type, at::IntArrayRef shape) {
    on_device(t, name, type, shape);
    if (!t.is_contiguous()) throw Refusal{PyExc_ValueError, std::string(name) + " must be contiguous"};
}
// elements between the rows of t [T, heads, d], whose rows are contiguous
int64_t rows(const at::Tensor &t, const char *name, at::ScalarType type, int64_t T, int64_t H, int64_t d) {
    on_device(t, name, type, {T, H, d});
    if ((t.stride(2) != 1 && d > 1) || (t.stride(1) != d && H > 1)) throw Refusal{PyExc_ValueError, std::string(name) + " must be contiguous within its rows of heads x d"};
    return T > 1 ? t.stride(0) : H * d;
}

// The array of integers in t; one that begins inside a 16-byte word (a part of a larger batch's) as a copy that does not, made on the call's stream.
const int32_t *ints(const at::Tensor &t, at::Tensor &copy) {
    if (reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0) return t.data_ptr<int32_t>();
    copy = t.clone();
    return copy.data_ptr<int32_t>();
}

int32_t int32(int64_t v, const char *name) {
    if (v < INT32_MIN || v > INT32_MAX) throw Refusal{PyExc_ValueError, std::string(name) + " does not fit 32 bits"};
    return (int32_t)v;
}
int64_t integer(PyObject *o, const char *name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); throw Refusal{PyExc_TypeError, std::string(name) + " must be an integer"}; }
    return v;
}
double number(PyObject *o, const char *name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); throw Refusal{PyExc_TypeError, std::string(name) + " must be a number"}; }
    return v;
}

int type_of(const at::Tensor &t, const char *name) {
    if (t.scalar_type() == at::kFloat) return DN_F32;
    if (t.scalar_type() == at::kBFloat16) return DN_BF16;
    throw Refusal{PyExc_TypeError, std::string(name) + " must be float32 or bfloat16, got " + at::toString(t.scalar_type())};
}

void *ptr(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }
float *fptr(const at::Tensor *t) { return static_cast<float *>(ptr(t)); }

// handle of the current stream of t's device
void *stream_of(const at::Tensor &t) {
    PyObject *at = PyLong_FromLong(t.get_device());
    PyObject *h = at ? PyObject_CallFunctionObjArgs(g_raw_stream, at, nullptr) : nullptr;
    Py_XDECREF(at);
    if (!h) throw Refusal{nullptr, ""};
    void *s = reinterpret_cast<void *>(PyLong_AsLongLong(h));
    Py_DECREF(h);
    if (PyErr_Occurred()) throw Refusal{nullptr, ""};
    return s;
}

at::Tensor out(const at::Tensor *given, const char *name, at::IntArrayRef shape, const at::Tensor &like, at::ScalarType type) {
    if (!given) return at::empty(shape, like.options().dtype(type));
    whole(*given, name, type, shape);
    return *given;
}

// the caller's workspace, or one for this call (none if none is needed)
struct Scratch {
    at::Tensor held;
    size_t bytes = 0;
    Scratch(const at::Tensor *given, size_t need, const at::Tensor &like) {
        if (given) {
            if (!given->is_cuda() || !given->is_contiguous()) throw Refusal{PyExc_ValueError, "workspace must be a contiguous device tensor"};
            held = *given;
            bytes = given->nbytes();
        } else if (need) {
            held = at::empty({(int64_t)need}, like.options().dtype(at::kByte));
            bytes = need;
        }
    }
    void *p() const { return bytes ? held.data_ptr() : nullptr; }
};

dn_rope rope_of(const at::Tensor *table, PyObject *eps, PyObject *interleaved) {
    const int pairs = PyObject_IsTrue(interleaved);
    if (pairs < 0) throw Refusal{nullptr, ""}; // (the object's own error)
    dn_rope r = {0, pairs, 0, (float)number(eps, "eps")};
    if (table) {
        if (table->dim() != 2) throw Refusal{PyExc_ValueError, "rope must be [max_pos, rot], cosines then sines"};
        whole(*table, "rope", at::kFloat, table->sizes());
        r.max_pos = int32(table->size(0), "rope's rows");
        r.rot = int32(table->size(1), "rope's columns");
    }
    return r;
}
void weights(const at::Tensor *qw, const at::Tensor *kw, at::ScalarType type, int64_t d) {
    if (qw) whole(*qw, "q_weight", type, {d});
    if (kw) whole(*kw, "k_weight", type, {d});
}

// [B, L, H, d] with evenly spaced rows as [B L, H, d]
at::Tensor flat(const at::Tensor &t, const char *name) {
    const int64_t B = t.size(0), L = t.size(1);
    if (B > 1 && L > 1 && t.stride(0) != L * t.stride(1)) throw Refusal{PyExc_ValueError, std::string(name) + " must have evenly spaced rows"};
    return t.as_strided({B * L, t.size(2), t.size(3)}, {L > 1 || B <= 1 ? t.stride(1) : t.stride(0), t.stride(2), t.stride(3)});
}

struct QK {
    at::Tensor q, k, copy;
    const int32_t *positions = nullptr;
    dn_qk_shape s;
    at::ScalarType type;
    QK(const at::Tensor &q_, const at::Tensor &k_, const at::Tensor *pos) : q(q_), k(k_) {
        s.dtype = type_of(q, "q");
        type = q.scalar_type();
        int64_t seq = q.dim() ? q.size(0) : 0;
        if (q.dim() == 4 && k.dim() == 4) {
            if (q.size(0) != k.size(0) || q.size(1) != k.size(1)) throw Refusal{PyExc_ValueError, "q and k must have the same rows"};
            seq = q.size(1);
            q = flat(q, "q");
            k = flat(k, "k");
        }
        if (q.dim() != 3 || k.dim() != 3) throw Refusal{PyExc_ValueError, "q and k must both be [T, heads, d] or [B, L, heads, d]"};
        const int64_t T = q.size(0), d = q.size(2);
        s.q_stride = rows(q, "q", type, T, q.size(1), d);
        s.k_stride = rows(k, "k", type, T, k.size(1), d);
        s.T = int32(T, "T"); s.Hq = int32(q.size(1), "heads"); s.Hkv = int32(k.size(1), "heads"); s.d = int32(d, "d");
        s.seq_len = int32(std::max<int64_t>(seq, 1), "L");
        if (pos) {
            whole(*pos, "positions", at::kInt, {T});
            positions = ints(*pos, copy);
        }
    }
};

struct Paged {
    dn_paged_shape s = {};
    dn_paged_cache c = {};
    at::Tensor copies[3];
    Paged(PyObject *k_pages, PyObject *v_pages, PyObject *page_table, PyObject *kv_len, PyObject *cu, PyObject *k_scale, PyObject *v_scale, int dtype) {
        const at::Tensor &kp = tensor(k_pages, "k_pages"), &vp = tensor(v_pages, "v_pages"), &table = tensor(page_table, "page_table");
        const at::Tensor &lens = tensor(kv_len, "kv_len"), &offsets = tensor(cu, "cu_q"), *ks = maybe(k_scale, "k_scale"), *vs = maybe(v_scale, "v_scale");
        if (kp.dim() != 4 || table.dim() != 2) throw Refusal{PyExc_ValueError, "k_pages must be [num_pages, heads, page_size, d], page_table [sequences, max_pages]"};
        const at::ScalarType held = kp.scalar_type();
        const bool quantised = held == at::kFloat8_e4m3fn;
        if (!quantised && held != (dtype == DN_F32 ? at::kFloat : at::kBFloat16))
            throw Refusal{PyExc_TypeError, std::string("pages must have the tensors' type or be float8_e4m3fn, got ") + at::toString(held)};
        const int64_t pages = kp.size(0), H = kp.size(1), ps = kp.size(2), N = table.size(0);
        whole(kp, "k_pages", held, kp.sizes());
        whole(vp, "v_pages", held, kp.sizes());
        if (quantised) {
            if (!ks || !vs) throw Refusal{PyExc_ValueError, "k_scale and v_scale are needed for an 8-bit cache"};
            whole(*ks, "k_scale", at::kFloat, {pages, H, ps});
            whole(*vs, "v_scale", at::kFloat, {pages, H, ps});
        } else if (ks || vs) throw Refusal{PyExc_ValueError, "scales belong to an 8-bit cache"};
        whole(table, "page_table", at::kInt, table.sizes());
        whole(lens, "kv_len", at::kInt, {N});
        whole(offsets, "cu_q", at::kInt, {N + 1});
        s.num_seqs = int32(N, "sequences"); s.max_pages = int32(table.size(1), "max_pages");
        s.num_pages = int32(pages, "num_pages"); s.Hkv = int32(H, "heads"); s.page_size = int32(ps, "page_size"); s.d = int32(kp.size(3), "d");
        s.dtype = dtype; s.cache_dtype = quantised ? DN_FP8 : dtype;
        s.max_kv = (int32_t)std::min<int64_t>(table.size(1) * ps, 1 << 30); // (the most that a context may have)
        s.cu_q = ints(offsets, copies[0]); s.kv_len = ints(lens, copies[1]); s.page_table = ints(table, copies[2]);
        c.k_pages = kp.data_ptr(); c.v_pages = vp.data_ptr(); c.k_scale = fptr(ks); c.v_scale = fptr(vs);
    }
};
int64_t first_size(const at::Tensor &t, const char *name) {
    if (t.dim() != 3) throw Refusal{PyExc_ValueError, std::string(name) + " must be [T, heads, d], got " + text_of(t.sizes())};
    return t.size(0);
}

PyObject *tuple_of(std::initializer_list<const at::Tensor *> ts) {
    PyObject *r = PyTuple_New((Py_ssize_t)ts.size());
    if (!r) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor *t : ts) {
        PyObject *o = t ? THPVariable_Wrap(*t) : Py_NewRef(Py_None);
        if (!o) { Py_DECREF(r); return nullptr; }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}

// --- the functions (arguments by position; None where the caller left one out)

typedef PyObject *const *Args;

PyObject *norm_rope_fwd(Args a) {
    const at::Tensor *qw = maybe(a[2], "q_weight"), *kw = maybe(a[3], "k_weight"), *table = maybe(a[4], "rope"), *pos = maybe(a[5], "positions");
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k");
    const QK x(q, k, pos);
    const dn_rope r = rope_of(table, a[6], a[7]);
    weights(qw, kw, x.type, x.s.d);
    const at::Tensor qo = out(maybe(a[8], "q_out"), "q_out", q.sizes(), q, x.type), ko = out(maybe(a[9], "k_out"), "k_out", k.sizes(), q, x.type);
    const int rc = lib.norm_rope_fwd(&x.s, &r, x.q.data_ptr(), x.k.data_ptr(), ptr(qw), ptr(kw), fptr(table), x.positions, qo.data_ptr(),
                                     ko.data_ptr(), stream_of(q));
    return rc ? PyLong_FromLong(rc) : tuple_of({&qo, &ko});
}

PyObject *norm_rope_bwd(Args a) {
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &dqo = tensor(a[2], "dq_out"), &dko = tensor(a[3], "dk_out");
    const at::Tensor *qw = maybe(a[4], "q_weight"), *kw = maybe(a[5], "k_weight"), *table = maybe(a[6], "rope"), *pos = maybe(a[7], "positions");
    const QK x(q, k, pos);
    const dn_rope r = rope_of(table, a[8], a[9]);
    weights(qw, kw, x.type, x.s.d);
    whole(dqo, "dq_out", x.type, q.sizes());
    whole(dko, "dk_out", x.type, k.sizes());
    const at::Tensor *given_dqw = maybe(a[12], "dq_weight"), *given_dkw = maybe(a[13], "dk_weight");
    if ((!qw && given_dqw) || (!kw && given_dkw)) throw Refusal{PyExc_ValueError, "no gradient of a weight that is not there"};
    const at::Tensor dq = out(maybe(a[10], "dq"), "dq", q.sizes(), q, x.type), dk = out(maybe(a[11], "dk"), "dk", k.sizes(), q, x.type);
    at::Tensor dqw, dkw;
    if (qw) dqw = out(given_dqw, "dq_weight", {x.s.d}, q, at::kFloat);
    if (kw) dkw = out(given_dkw, "dk_weight", {x.s.d}, q, at::kFloat);
    size_t need = 0;
    int rc = lib.norm_rope_bytes(&x.s, &need);
    if (rc) return PyLong_FromLong(rc);
    const Scratch ws(maybe(a[14], "workspace"), qw || kw ? need : 0, q);
    rc = lib.norm_rope_bwd(&x.s, &r, x.q.data_ptr(), x.k.data_ptr(), dqo.data_ptr(), dko.data_ptr(), ptr(qw), ptr(kw), fptr(table), x.positions,
                           dq.data_ptr(), dk.data_ptr(), qw ? fptr(&dqw) : nullptr, kw ? fptr(&dkw) : nullptr, ws.p(), ws.bytes, stream_of(q));
    return rc ? PyLong_FromLong(rc) : tuple_of({&dq, &dk, qw ? &dqw : nullptr, kw ? &dkw : nullptr});
}

PyObject *append(Args a) {
    const at::Tensor &k = tensor(a[0], "k"), &v = tensor(a[1], "v");
    Paged p(a[2], a[3], a[4], a[5], a[6], a[7], a[8], type_of(k, "k"));
    const int64_t T = first_size(k, "k");
    p.s.T = int32(T, "T"); p.s.Hq = p.s.Hkv;
    p.s.k_stride = rows(k, "k", k.scalar_type(), T, p.s.Hkv, p.s.d);
    p.s.v_stride = rows(v, "v", k.scalar_type(), T, p.s.Hkv, p.s.d);
    const int rc = lib.append(&p.s, k.data_ptr(), v.data_ptr(), &p.c, stream_of(k));
    if (rc) return PyLong_FromLong(rc);
    Py_RETURN_NONE;
}

PyObject *norm_rope_append(Args a) {
    const at::Tensor &q = tensor(a[0], "q"), &k = tensor(a[1], "k"), &v = tensor(a[2], "v");
    const at::Tensor *qw = maybe(a[8], "q_weight"), *kw = maybe(a[9], "k_weight"), *table = maybe(a[10], "rope");
    Paged p(a[3], a[4], a[5], a[6], a[7], a[11], a[12], type_of(q, "q"));
    const at::ScalarType type = q.scalar_type();
    const int64_t T = first_size(q, "q"), Hq = q.size(1);
    p.s.T = int32(T, "T"); p.s.Hq = int32(Hq, "heads");
    p.s.q_stride = rows(q, "q", type, T, Hq, p.s.d);
    p.s.k_stride = rows(k, "k", type, T, p.s.Hkv, p.s.d);
    p.s.v_stride = rows(v, "v", type, T, p.s.Hkv, p.s.d);
    const dn_rope r = rope_of(table, a[13], a[14]);
    weights(qw, kw, type, p.s.d);
    const at::Tensor qo = out(maybe(a[15], "q_out"), "q_out", q.sizes(), q, type);
    const int rc = lib.norm_rope_append(&p.s, &r, q.data_ptr(), k.data_ptr(), v.data_ptr(), ptr(qw), ptr(kw), fptr(table), qo.data_ptr(), &p.c, stream_of(q));
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(qo);
}

PyObject *read(Args a) { // dtype as a dn_dtype
    const at::Tensor &kp = tensor(a[0], "k_pages");
    const int dtype = (int)integer(a[6], "dtype");
    Paged p(a[0], a[1], a[2], a[3], a[4], a[7], a[8], dtype);
    const int32_t T = int32(integer(a[5], "rows"), "rows");
    if (T < 0) return PyLong_FromLong(DN_ERR_SHAPE);
    p.s.Hq = p.s.Hkv;
    const at::ScalarType type = dtype == DN_F32 ? at::kFloat : at::kBFloat16;
    const at::Tensor ko = out(maybe(a[9], "k_out"), "k_out", {T, p.s.Hkv, p.s.d}, kp, type), vo = out(maybe(a[10], "v_out"), "v_out", {T, p.s.Hkv, p.s.d}, kp, type);
    const int rc = lib.read(&p.s, &p.c, p.s.cu_q, T, ko.data_ptr(), vo.data_ptr(), stream_of(kp));
    return rc ? PyLong_FromLong(rc) : tuple_of({&ko, &vo});
}

PyObject *attn(Args a) {
    const at::Tensor &q = tensor(a[0], "q");
    Paged p(a[1], a[2], a[3], a[4], a[5], a[6], a[7], type_of(q, "q"));
    const int64_t T = first_size(q, "q"), Hq = q.size(1);
    p.s.T = int32(T, "T"); p.s.Hq = int32(Hq, "heads");
    p.s.q_stride = rows(q, "q", q.scalar_type(), T, Hq, p.s.d);
    p.s.max_q = a[10] == Py_None ? p.s.T : int32(integer(a[10], "max_q"), "max_q");
    if (a[11] != Py_None) p.s.max_kv = int32(integer(a[11], "max_kv"), "max_kv");
    const int32_t window = int32(integer(a[9], "window"), "window");
    size_t need = 0;
    int rc = lib.attn_bytes(&p.s, window, &need);
    if (rc) return PyLong_FromLong(rc);
    const at::Tensor o = out(maybe(a[12], "o"), "o", q.sizes(), q, q.scalar_type());
    const Scratch ws(maybe(a[13], "workspace"), need, q);
    const float scale = a[8] == Py_None ? 1.f / std::sqrt((float)p.s.d) : (float)number(a[8], "scale");
    rc = lib.attn(&p.s, q.data_ptr(), &p.c, scale, window, o.data_ptr(), ws.p(), ws.bytes, stream_of(q));
    return rc ? PyLong_FromLong(rc) : THPVariable_Wrap(o);
}

// nothing thrown leaves: refusals and torch's own errors (out of memory) become Python exceptions
template <PyObject *(*F)(Args), int N> PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (n != N) return PyErr_Format(PyExc_TypeError, "%d arguments wanted, got %zd", N, n);
    try {
        return F(args);
    } catch (const Refusal &r) {
        if (r.type) PyErr_SetString(r.type, r.text.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// open(path, raw_stream): finds the entry points in the library at `path`
PyObject *open_library(PyObject *, PyObject *args) {
    const char *path;
    PyObject *raw;
    if (!PyArg_ParseTuple(args, "sO", &path, &raw)) return nullptr;
    void *h = dlopen(path, RTLD_NOW | RTLD_LOCAL);
    if (!h) return PyErr_Format(PyExc_OSError, "%s", dlerror());
    struct { const char *name; void **to; } const want[] = {
        {"deltanet_qk_norm_rope_fwd", (void **)&lib.norm_rope_fwd}, {"deltanet_qk_norm_rope_workspace_bytes", (void **)&lib.norm_rope_bytes},
        {"deltanet_qk_norm_rope_bwd", (void **)&lib.norm_rope_bwd}, {"deltanet_paged_append", (void **)&lib.append},
        {"deltanet_paged_norm_rope_append", (void **)&lib.norm_rope_append}, {"deltanet_paged_read", (void **)&lib.read},
        {"deltanet_paged_attn_workspace_bytes", (void **)&lib.attn_bytes}, {"deltanet_paged_attn_fwd", (void **)&lib.attn}};
    for (const auto &w : want)
        if (!(*w.to = dlsym(h, w.name))) return PyErr_Format(PyExc_OSError, "%s has no %s", path, w.name);
    Py_XSETREF(g_raw_stream, Py_NewRef(raw));
    Py_RETURN_NONE;
}

#define ENTRY(NAME, F, N) {NAME, (PyCFunction)(void (*)(void))(PyObject * (*)(PyObject *, PyObject *const *, Py_ssize_t))entry<F, N>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"open", open_library, METH_VARARGS, nullptr},
                         ENTRY("norm_rope_fwd", norm_rope_fwd, 10),
                         ENTRY("norm_rope_bwd", norm_rope_bwd, 15),
                         ENTRY("append", append, 9),
                         ENTRY("norm_rope_append", norm_rope_append, 16),
                         ENTRY("read", read, 11),
                         ENTRY("attn", attn, 14),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_attention", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

} // namespace

extern "C" PyObject *PyInit__attention() { return PyModule_Create(&module); }
