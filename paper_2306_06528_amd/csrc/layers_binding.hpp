// The calls of layers.py and attention.py whose tensors are checked, and whose results are allocated, in native code (layers_binding.cpp, attention_binding.cpp).
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>

PyObject *layer_norm_forward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *layer_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *gated_ffn_forward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *gated_ffn_backward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *dropout(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *linear_forward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *linear_backward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *qk_norm_rotary_forward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *qk_norm_rotary_backward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *attention_forward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *attention_backward(PyObject *, PyObject *const *args, Py_ssize_t count);
