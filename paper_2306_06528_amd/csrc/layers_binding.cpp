// What a call of layers.py needs before the library can be called: the checks of its tensors, their pointers, strides and sizes,
// and the tensors that it returns or works in.  In Python these took 10 to 15 us of a call, where the kernels of a small
// one take 4.  Every function returns None, with nothing done, if x is not on the current device: the caller makes that the
// current one and calls again.  Nothing is kept from one call for the next.
#include "layers_binding.hpp"

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>

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

uint64_t low_bits(PyObject *obj) // of any integer, as & (2^64 - 1) gives them
{
    const uint64_t v = PyLong_AsUnsignedLongLongMask(obj);
    if (v == (uint64_t)-1 && PyErr_Occurred()) throw Failed{};
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

at::Tensor stats(PyObject *obj, const char *name, const Act &x)
{
    const char *const what = "%s must be what layer_norm_forward returned for x";
    if (!THPVariable_Check(obj)) fail(PyExc_TypeError, what, name);
    const at::Tensor &t = THPVariable_Unpack(obj);
    if (t.scalar_type() != at::kFloat || t.sizes() != x.given.sizes().slice(0, x.given.dim() - 1) || t.device() != x.given.device() || !t.is_contiguous())
        fail(PyExc_TypeError, what, name);
    return t;
}

struct Block { // a gated feed-forward block's sizes and parameters
    int activation;
    int64_t hidden;
    Param gate, up, down;
};

Block block(const Act &x, PyObject *const *a, PyObject *activation) // a: gate, up, down
{
    Block b;
    const char *const name = PyUnicode_Check(activation) ? PyUnicode_AsUTF8(activation) : "";
    if (!name) throw Failed{};
    b.activation = !strcmp(name, "silu") ? SVGD_SILU : !strcmp(name, "gelu") ? SVGD_GELU : -1;
    if (b.activation < 0) fail(PyExc_ValueError, "activation must be one of %s", "('silu', 'gelu')");
    if (!THPVariable_Check(a[0]) || THPVariable_Unpack(a[0]).dim() != 3) fail(PyExc_TypeError, "%s must be a float32 CUDA tensor (particles, hidden, width)", "gate");
    b.hidden = THPVariable_Unpack(a[0]).size(1);
    b.gate = param(a[0], "gate", {x.n(), b.hidden, x.width()}, x);
    b.up = param(a[1], "up", {x.n(), b.hidden, x.width()}, x);
    b.down = param(a[2], "down", {x.n(), x.width(), b.hidden}, x);
    return b;
}

} // namespace

// layer_norm_forward(current_device, stream_of, x, weight, bias, eps) -> (y, mean, rstd)
PyObject *layer_norm_forward(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 6, [&]() -> PyObject * {
        const Act x = act(a[2], "x");
        const Param w = param(a[3], "weight", {x.n(), x.width()}, x), b = param(a[4], "bias", {x.n(), x.width()}, x, true);
        const double eps = number(a[5]);
        void *stream;
        if (!current_stream(x, a, stream)) Py_RETURN_NONE;
        const at::Tensor y = new_like(x);
        const at::IntArrayRef per_row = x.given.sizes().slice(0, x.given.dim() - 1);
        const at::Tensor mean = at::empty(per_row, x.given.options().dtype(at::kFloat)), rstd = at::empty(per_row, x.given.options().dtype(at::kFloat));
        const int rc = unlocked([&] {
            return svgd_layer_norm_forward(x.dtype(), x.particles(), x.rows(), x.width(), x.desc(), w.p(), w.stride, b.p(), b.stride, eps, dense(y, x),
                                           (float *)mean.data_ptr(), (float *)rstd.data_ptr(), stream);
        });
        return result(rc, {&y, &mean, &rstd});
    });
}

// layer_norm_backward(current_device, stream_of, dy, x, weight, mean, rstd, dweight, dbias, accumulate, want_dx) -> (dx,)
PyObject *layer_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 11, [&]() -> PyObject * {
        const Act x = act(a[3], "x"), dy = act(a[2], "dy", &x);
        const Param w = param(a[4], "weight", {x.n(), x.width()}, x);
        const at::Tensor mean = stats(a[5], "mean", x), rstd = stats(a[6], "rstd", x);
        const Param dw = param(a[7], "dweight", {x.n(), x.width()}, x, true), db = param(a[8], "dbias", {x.n(), x.width()}, x, true);
        const bool accumulate = truth(a[9]), want_dx = truth(a[10]);
        void *stream;
        if (!current_stream(x, a, stream)) Py_RETURN_NONE;
        at::Tensor dx, scratch;
        if (want_dx) dx = new_like(x);
        const size_t need = dw.t || db.t ? svgd_layer_norm_scratch(x.particles(), x.rows(), x.width()) : 0;
        if (need) scratch = bytes(need, x);
        const int rc = unlocked([&] {
            return svgd_layer_norm_backward(x.dtype(), x.particles(), x.rows(), x.width(), dy.desc(), x.desc(), w.p(), w.stride, (float *)mean.data_ptr(),
                                            (float *)rstd.data_ptr(), want_dx ? dense(dx, x) : svgd_rows{nullptr, 0, 0}, dw.p(), dw.stride, db.p(), db.stride,
                                            accumulate, need ? scratch.data_ptr() : nullptr, need, stream);
        });
        return result(rc, {&dx});
    });
}

// gated_ffn_forward(current_device, stream_of, x, gate, up, down, activation, save) -> (y, saved)
PyObject *gated_ffn_forward(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 8, [&]() -> PyObject * {
        const Act x = act(a[2], "x");
        const Block b = block(x, a + 3, a[6]);
        const bool save = truth(a[7]);
        void *stream;
        if (!current_stream(x, a, stream)) Py_RETURN_NONE;
        const at::Tensor y = new_like(x);
        const size_t need = svgd_gated_ffn_buffer(x.particles(), x.rows(), x.width(), b.hidden, save);
        const size_t scratch_need = svgd_gated_ffn_forward_scratch(x.particles(), x.rows(), x.width(), b.hidden);
        at::Tensor buffer = at::empty({(int64_t)(need / 4)}, x.given.options().dtype(at::kFloat)), scratch;
        if (scratch_need) scratch = bytes(scratch_need, x);
        const int rc = unlocked([&] {
            return svgd_gated_ffn_forward(x.dtype(), b.activation, x.particles(), x.rows(), x.width(), b.hidden, x.desc(), b.gate.p(), b.gate.stride, b.up.p(),
                                          b.up.stride, b.down.p(), b.down.stride, dense(y, x), save, buffer.data_ptr(), need,
                                          scratch_need ? scratch.data_ptr() : nullptr, scratch_need, stream);
        });
        if (!save) buffer = at::Tensor();
        return result(rc, {&y, &buffer});
    });
}

// gated_ffn_backward(current_device, stream_of, dy, x, gate, up, down, saved, dgate, dup, ddown, activation, accumulate, want_dx) -> (dx,)
PyObject *gated_ffn_backward(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 14, [&]() -> PyObject * {
        const Act x = act(a[3], "x"), dy = act(a[2], "dy", &x);
        const Block b = block(x, a + 4, a[11]);
        const Param dgate = param(a[8], "dgate", {x.n(), b.hidden, x.width()}, x, true), dup = param(a[9], "dup", {x.n(), b.hidden, x.width()}, x, true),
                    ddown = param(a[10], "ddown", {x.n(), x.width(), b.hidden}, x, true);
        const size_t saved_need = svgd_gated_ffn_buffer(x.particles(), x.rows(), x.width(), b.hidden, 1),
                     need = svgd_gated_ffn_scratch(x.particles(), x.rows(), x.width(), b.hidden);
        const char *const what = "%s must be what gated_ffn_forward returned for x with save=True";
        if (!THPVariable_Check(a[7])) fail(PyExc_TypeError, what, "saved");
        const at::Tensor &saved = THPVariable_Unpack(a[7]);
        if (saved.scalar_type() != at::kFloat || (size_t)saved.numel() * 4 != saved_need || saved.device() != x.given.device() || !saved.is_contiguous())
            fail(PyExc_TypeError, what, "saved");
        const bool accumulate = truth(a[12]), want_dx = truth(a[13]);
        void *stream;
        if (!current_stream(x, a, stream)) Py_RETURN_NONE;
        at::Tensor dx;
        if (want_dx) dx = new_like(x);
        const at::Tensor scratch = bytes(need, x);
        const int rc = unlocked([&] {
            return svgd_gated_ffn_backward(x.dtype(), b.activation, x.particles(), x.rows(), x.width(), b.hidden, dy.desc(), x.desc(), b.gate.p(), b.gate.stride,
                                           b.up.p(), b.up.stride, b.down.p(), b.down.stride, saved.data_ptr(), saved_need,
                                           want_dx ? dense(dx, x) : svgd_rows{nullptr, 0, 0}, dgate.p(), dgate.stride, dup.p(), dup.stride, ddown.p(), ddown.stride,
                                           accumulate, scratch.data_ptr(), need, stream);
        });
        return result(rc, {&dx});
    });
}

// dropout(current_device, stream_of, x, p, seed, call, residual, counter) -> (y,)
PyObject *dropout(PyObject *, PyObject *const *a, Py_ssize_t na)
{
    return guarded(na, 8, [&]() -> PyObject * {
        const Act x = act(a[2], "x");
        const double p = number(a[3]);
        const uint64_t seed = low_bits(a[4]), call = low_bits(a[5]);
        Act residual;
        if (a[6] != Py_None) residual = act(a[6], "residual", &x);
        const int64_t *counter = nullptr;
        if (a[7] != Py_None) {
            const char *const what = "%s must be an int64 tensor of one element on the device of x";
            if (!THPVariable_Check(a[7])) fail(PyExc_TypeError, what, "counter");
            const at::Tensor &t = THPVariable_Unpack(a[7]);
            if (t.scalar_type() != at::kLong || t.numel() != 1 || t.device() != x.given.device()) fail(PyExc_TypeError, what, "counter");
            counter = (const int64_t *)t.data_ptr();
        }
        void *stream;
        if (!current_stream(x, a, stream)) Py_RETURN_NONE;
        const at::Tensor y = new_like(x);
        const int rc = unlocked([&] {
            return svgd_dropout(x.dtype(), x.particles(), x.rows(), x.width(), x.desc(), residual.t.defined() ? residual.desc() : svgd_rows{nullptr, 0, 0},
                                dense(y, x), p, seed, call, counter, stream);
        });
        return result(rc, {&y});
    });
}
