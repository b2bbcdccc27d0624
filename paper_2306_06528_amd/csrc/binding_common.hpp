// What the native calls of layers.py and attention.py share: checks of tensors, their pointers, strides and sizes, streams, errors.
#pragma once
#include "layers_binding.hpp"

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>

#include <cmath>
#include <cstring>
#include <sstream>

#include "../../include/svgd_layers.h"

namespace {

struct Failed {}; // a Python error is set

[[noreturn]] void fail(PyObject *type, const char *format, const char *name)
{
    PyErr_Format(type, format, name);
    throw Failed{};
}

int dtype_of(at::ScalarType t)
{
    return t == at::kFloat ? SVGD_F32 : t == at::kBFloat16 ? SVGD_BF16 : t == at::kHalf ? SVGD_F16 : -1;
}

// An activation as (n, rows, width).
struct Act {
    at::Tensor given, t;
    int64_t n() const { return t.size(0); }
    int particles() const { return n() > INT32_MAX ? INT32_MAX : (int)n(); } // (refused by the library)
    int64_t rows() const { return t.size(1); }
    int64_t width() const { return t.size(2); }
    int dtype() const { return dtype_of(t.scalar_type()); }
    svgd_rows desc() const { return {t.data_ptr(), t.stride(0), t.stride(1)}; }
};

const char *const kNoAct = "%s must be a CUDA tensor (particles, ..., width) of float32, bfloat16 or float16";

Act act(PyObject *obj, const char *name, const Act *like = nullptr)
{
    if (!THPVariable_Check(obj)) fail(PyExc_TypeError, kNoAct, name);
    Act a{THPVariable_Unpack(obj), {}};
    const at::Tensor &g = a.given;
    if (!g.is_cuda() || dtype_of(g.scalar_type()) < 0 || g.dim() < 2) fail(PyExc_TypeError, kNoAct, name);
    if (like && (g.sizes() != like->given.sizes() || g.scalar_type() != like->given.scalar_type() || g.device() != like->given.device()))
        fail(PyExc_ValueError, "%s must have the shape, type and device of the other activations", name);
    if (g.dim() == 3) {
        a.t = g;
    } else {
        const at::NoGradGuard no_grad;
        int64_t rows = 1;
        for (int64_t d = 1; d + 1 < g.dim(); ++d) rows *= g.size(d);
        a.t = g.reshape({g.size(0), rows, g.size(g.dim() - 1)});
    }
    if (a.t.size(2) != 1 && a.t.stride(2) != 1 && a.t.numel()) fail(PyExc_TypeError, "%s must have contiguous rows", name);
    return a;
}

// A parameter or its gradient; None, where that may be, has a null pointer.  Pointers are taken last, behind everything
// that can run other code.
struct Param {
    const at::Tensor *t = nullptr;
    int64_t stride = 0;
    float *p() const { return t ? (float *)t->data_ptr() : nullptr; }
};

Param param(PyObject *obj, const char *name, at::IntArrayRef shape, const Act &x, bool optional = false)
{
    if (optional && obj == Py_None) return {};
    if (!THPVariable_Check(obj)) fail(PyExc_TypeError, "%s must be a float32 CUDA tensor", name);
    const at::Tensor &t = THPVariable_Unpack(obj);
    if (!t.is_cuda() || t.scalar_type() != at::kFloat) fail(PyExc_TypeError, "%s must be a float32 CUDA tensor", name);
    if (t.sizes() != shape) {
        std::ostringstream text;
        text << "%s must have the shape " << shape << ", not " << t.sizes();
        fail(PyExc_ValueError, text.str().c_str(), name);
    }
    if (t.device() != x.given.device()) fail(PyExc_ValueError, "%s must be on the device of the activations", name);
    int64_t size = 1;
    for (int64_t d = t.dim() - 1; d >= 1; --d) {
        if (t.size(d) != 1 && t.stride(d) != size) fail(PyExc_TypeError, "%s must be contiguous within each particle", name);
        size *= t.size(d);
    }
    return {&t, shape[0] != 1 ? t.stride(0) : size};
}

double number(PyObject *obj)
{
    const double v = PyFloat_AsDouble(obj);
    if (v == -1.0 && PyErr_Occurred()) throw Failed{};
    return v;
}

bool truth(PyObject *obj)
{
    const int v = PyObject_IsTrue(obj);
    if (v < 0) throw Failed{};
    return v != 0;
}

int64_t integer(PyObject *obj)
{
    const int64_t v = PyLong_AsLongLong(obj);
    if (v == -1 && PyErr_Occurred()) throw Failed{};
    return v;
}

struct Owned { // a reference, given back at the end
    PyObject *p;
    ~Owned() { Py_XDECREF(p); }
};

// The current device's current stream, if x is on that device: a[0]() says which device it is, a[1](device) its stream.
// Asked for behind the checks: both need a GPU, and what is no tensor on one is to be named first.
bool current_stream(const Act &x, PyObject *const *a, void *&stream)
{
    const Owned device{PyObject_CallNoArgs(a[0])};
    if (!device.p) throw Failed{};
    if (integer(device.p) != x.given.get_device()) return false;
    const Owned s{PyObject_CallFunctionObjArgs(a[1], device.p, nullptr)};
    if (!s.p) throw Failed{};
    stream = PyLong_AsVoidPtr(s.p);
    if (!stream && PyErr_Occurred()) throw Failed{};
    return true;
}

at::Tensor new_like(const Act &a) { return at::empty(a.given.sizes(), a.given.options().memory_format(c10::nullopt)); }
svgd_rows dense(const at::Tensor &t, const Act &a) { return {t.data_ptr(), a.rows() * a.width(), a.width()}; }
at::Tensor bytes(size_t n, const Act &a) { return at::empty({(int64_t)n}, a.given.options().dtype(at::kByte)); }

// Errors of torch as its own Python functions raise them. f: (device is right) the result, a new reference
template <class F> PyObject *guarded(Py_ssize_t got, Py_ssize_t want, F f)
{
    HANDLE_TH_ERRORS
    if (got != want) {
        PyErr_Format(PyExc_TypeError, "%zd arguments, %zd expected", got, want);
        return nullptr;
    }
    try {
        return f();
    } catch (const Failed &) {
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// The library's call without the interpreter's lock; its status becomes an exception in Python.
template <class F> int unlocked(F f)
{
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = f();
    Py_END_ALLOW_THREADS
    return rc;
}

// (status, tensor or None ...)
PyObject *result(int rc, std::initializer_list<const at::Tensor *> tensors)
{
    if (rc != SVGD_OK) return PyLong_FromLong(rc);
    PyObject *const tuple = PyTuple_New((Py_ssize_t)tensors.size());
    if (!tuple) return nullptr;
    Py_ssize_t k = 0;
    for (const at::Tensor *t : tensors) {
        PyObject *item;
        if (t->defined()) {
            item = THPVariable_Wrap(*t);
        } else {
            Py_INCREF(Py_None);
            item = Py_None;
        }
        if (!item) {
            Py_DECREF(tuple);
            return nullptr;
        }
        PyTuple_SET_ITEM(tuple, k++, item);
    }
    return tuple;
}

} // namespace
