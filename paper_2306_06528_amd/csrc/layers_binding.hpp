// The calls of layers.py whose tensors are checked, and whose results are allocated, in native code (layers_binding.cpp).
#pragma once
#define PY_SSIZE_T_CLEAN
#include <Python.h>

PyObject *layer_norm_forward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *layer_norm_backward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *gated_ffn_forward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *gated_ffn_backward(PyObject *, PyObject *const *args, Py_ssize_t count);
PyObject *dropout(PyObject *, PyObject *const *args, Py_ssize_t count);
