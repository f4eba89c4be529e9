// What the native wrappers of both libraries have in common: how they look at Python's arguments, and make and hand back outputs.  Included by
// each inside the one source of its module.
#pragma once

#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "specsteer.h"

namespace {

PyObject* current_raw_stream = nullptr;  // of a device index

// A plain tensor of its own memory on a GPU, or NULL.
const at::Tensor* gpu_tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.has_storage() && t.layout() == at::kStrided ? &t : nullptr;
}

// The same, contiguous, of this type on this device.
const at::Tensor* ready(PyObject* o, at::ScalarType type, const at::Tensor& like) {
    const at::Tensor* t = gpu_tensor(o);
    return t && t->scalar_type() == type && t->device() == like.device() && t->is_contiguous() ? t : nullptr;
}

bool same_form(const at::Tensor& a, const at::Tensor& b) {
    return a.scalar_type() == b.scalar_type() && a.device() == b.device() && a.sizes() == b.sizes() && a.strides() == b.strides();
}

bool number(PyObject* o, float& v) {
    if (!PyFloat_CheckExact(o) && !PyLong_CheckExact(o)) return false;
    const double x = PyFloat_AsDouble(o);
    if (x == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    v = (float)x;
    return true;
}

bool truth(PyObject* o, bool& v) {
    if (!PyBool_Check(o)) return false;
    v = o == Py_True;
    return true;
}

// torch's current stream on the tensor's device; false with a Python error set.
bool stream_of(const at::Tensor& t, void*& s) {
    PyObject* index = PyLong_FromLong(t.get_device());
    PyObject* handle = index ? PyObject_CallOneArg(current_raw_stream, index) : nullptr;
    Py_XDECREF(index);
    if (!handle) return false;
    s = PyLong_AsVoidPtr(handle);
    Py_DECREF(handle);
    return !PyErr_Occurred();
}

// Without the interpreter's lock, as a call through ctypes is.
template <typename F>
ss_status unlocked(F call) {
    PyThreadState* const saved = PyEval_SaveThread();
    const ss_status rc = call();
    PyEval_RestoreThread(saved);
    return rc;
}

at::Tensor make(const at::Tensor& like, at::IntArrayRef size, at::ScalarType type) { return at::empty(size, like.options().dtype(type).requires_grad(false)); }

// A dict entry; None for an undefined tensor.
bool put(PyObject* dict, const char* key, const at::Tensor& t) {
    PyObject* v = t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None);
    const bool ok = v && PyDict_SetItemString(dict, key, v) == 0;
    Py_XDECREF(v);
    return ok;
}

template <typename T>
T* ptr(const at::Tensor& t) { return t.defined() ? static_cast<T*>(t.data_ptr()) : nullptr; }

}  // namespace
