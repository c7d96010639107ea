// What the compiled module's functions share: arguments that are tensors or numbers, their checks, outputs and workspaces that the caller did not bring, the current stream, results and errors.
#pragma once
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/EmptyTensor.h>
#include <c10/core/DeviceGuard.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <initializer_list>
#include <sstream>
#include <string>

#include "../../include/deltanet.h"

namespace dn_binding {

inline PyObject *g_raw_stream = nullptr; // device index -> handle of its current stream

struct Refusal { PyObject *type; std::string text; };

inline std::string text_of(at::IntArrayRef s) {
    std::ostringstream o;
    o << '(';
    for (size_t i = 0; i < s.size(); ++i) o << (i ? ", " : "") << s[i];
    o << ')';
    return o.str();
}

inline const at::Tensor &tensor(PyObject *o, const char *name) {
    if (!THPVariable_Check(o)) throw Refusal{PyExc_TypeError, std::string(name) + " must be a tensor"};
    return THPVariable_Unpack(o);
}
inline const at::Tensor *maybe(PyObject *o, const char *name) { return o == Py_None ? nullptr : &tensor(o, name); }

inline void on_device(const at::Tensor &t, const char *name, at::ScalarType type, at::IntArrayRef shape) {
    if (!t.is_cuda()) throw Refusal{PyExc_ValueError, std::string(name) + " must be a device tensor"};
    if (t.scalar_type() != type) throw Refusal{PyExc_TypeError, std::string(name) + " must be " + at::toString(type) + ", got " + at::toString(t.scalar_type())};
    if (t.sizes() != shape) throw Refusal{PyExc_ValueError, std::string(name) + " must have shape " + text_of(shape) + ", got " + text_of(t.sizes())};
}
inline void whole(const at::Tensor &t, const char *name, at::ScalarType type, at::IntArrayRef shape) {
    on_device(t, name, type, shape);
    if (!t.is_contiguous()) throw Refusal{PyExc_ValueError, std::string(name) + " must be contiguous"};
}
// elements between the rows of t [T, heads, d], whose rows are contiguous
inline int64_t rows(const at::Tensor &t, const char *name, at::ScalarType type, int64_t T, int64_t H, int64_t d) {
    on_device(t, name, type, {T, H, d});
    if ((t.stride(2) != 1 && d > 1) || (t.stride(1) != d && H > 1)) throw Refusal{PyExc_ValueError, std::string(name) + " must be contiguous within its rows of heads x d"};
    return T > 1 ? t.stride(0) : H * d;
}

// The array of integers in t; one that begins inside a 16-byte word (a part of a larger batch's) as a copy that does not, made on the call's stream.
inline const int32_t *ints(const at::Tensor &t, at::Tensor &copy) {
    if (reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0) return t.data_ptr<int32_t>();
    copy = t.clone();
    return copy.data_ptr<int32_t>();
}

inline int32_t int32(int64_t v, const char *name) {
    if (v < INT32_MIN || v > INT32_MAX) throw Refusal{PyExc_ValueError, std::string(name) + " does not fit 32 bits"};
    return (int32_t)v;
}
inline int64_t integer(PyObject *o, const char *name) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) { PyErr_Clear(); throw Refusal{PyExc_TypeError, std::string(name) + " must be an integer"}; }
    return v;
}
inline double number(PyObject *o, const char *name) {
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); throw Refusal{PyExc_TypeError, std::string(name) + " must be a number"}; }
    return v;
}

inline int type_of(const at::Tensor &t, const char *name) {
    if (t.scalar_type() == at::kFloat) return DN_F32;
    if (t.scalar_type() == at::kBFloat16) return DN_BF16;
    throw Refusal{PyExc_TypeError, std::string(name) + " must be float32 or bfloat16, got " + at::toString(t.scalar_type())};
}

inline void *ptr(const at::Tensor *t) { return t ? t->data_ptr() : nullptr; }
inline float *fptr(const at::Tensor *t) { return static_cast<float *>(ptr(t)); }

// handle of the current stream of t's device
inline void *stream_of(const at::Tensor &t) {
    PyObject *at = PyLong_FromLong(t.get_device());
    PyObject *h = at ? PyObject_CallFunctionObjArgs(g_raw_stream, at, nullptr) : nullptr;
    Py_XDECREF(at);
    if (!h) throw Refusal{nullptr, ""};
    void *s = reinterpret_cast<void *>(PyLong_AsLongLong(h));
    Py_DECREF(h);
    if (PyErr_Occurred()) throw Refusal{nullptr, ""};
    return s;
}

// A new tensor on the current device, which is that of `like` (a DeviceGuard of the function's), from like's own allocator: past torch's dispatcher, which takes as long as the allocation (a
// small call makes one to six of them, at half a microsecond each instead of one).
inline at::Tensor fresh(at::IntArrayRef shape, const at::Tensor &like, at::ScalarType type) {
    at::Allocator *from = like.has_storage() ? like.storage().allocator() : nullptr; // (none where the memory came from elsewhere)
    if (!from) return at::empty(shape, like.options().dtype(type));
    return at::detail::empty_generic(shape, from, c10::DispatchKeySet(c10::DispatchKey::CUDA), type, std::nullopt);
}

inline at::Tensor out(const at::Tensor *given, const char *name, at::IntArrayRef shape, const at::Tensor &like, at::ScalarType type) {
    if (!given) return fresh(shape, like, type);
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
            held = fresh({(int64_t)need}, like, at::kByte);
            bytes = need;
        }
    }
    void *p() const { return bytes ? held.data_ptr() : nullptr; }
};
// [B, L, H, d] with evenly spaced rows as [B L, H, d]
inline at::Tensor flat(const at::Tensor &t, const char *name) {
    const int64_t B = t.size(0), L = t.size(1);
    if (B > 1 && L > 1 && t.stride(0) != L * t.stride(1)) throw Refusal{PyExc_ValueError, std::string(name) + " must have evenly spaced rows"};
    return t.as_strided({B * L, t.size(2), t.size(3)}, {L > 1 || B <= 1 ? t.stride(1) : t.stride(0), t.stride(2), t.stride(3)});
}
inline PyObject *tuple_of(std::initializer_list<const at::Tensor *> ts) {
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
typedef PyObject *const *Args;

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

// a symbol of the library, and where the pointer to it goes
struct Symbol { const char *name; void **to; };

} // namespace dn_binding

#define ENTRY(NAME, F, N) {NAME, (PyCFunction)(void (*)(void))(PyObject * (*)(PyObject *, PyObject *const *, Py_ssize_t))dn_binding::entry<F, N>, METH_FASTCALL, nullptr}
