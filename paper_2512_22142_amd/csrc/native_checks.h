// Checks and conversions that the files of the _native extension share.
#pragma once

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <exception>

#include "cleave.h"

// The functions of native_operators.cpp.
PyMethodDef* operator_methods();

namespace {

// The Python exception is set.
struct Raised {};

[[noreturn]] void raise(PyObject* type, const char* text) {
  PyErr_SetString(type, text);
  throw Raised{};
}

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a torch tensor, not %s", what, Py_TYPE(o)->tp_name);
    throw Raised{};
  }
  return THPVariable_Unpack(o);
}

struct Matrix {
  void* ptr;
  int64_t ld, rows, cols;
  at::ScalarType type;
};

[[maybe_unused]] Matrix matrix(PyObject* o, const char* what) {
  const at::Tensor& t = tensor(o, what);
  if (t.dim() != 2 || t.stride(1) != 1 || !t.is_cuda()) {
    PyErr_Format(PyExc_ValueError, "%s must be a 2-D device tensor with unit column stride", what);
    throw Raised{};
  }
  return Matrix{t.data_ptr(), t.stride(0), t.size(0), t.size(1), t.scalar_type()};
}

// The partial blocks of a plan, `elems` elements.
[[maybe_unused]] float* partial_blocks(PyObject* o, int64_t elems) {
  const at::Tensor& t = tensor(o, "partials");
  if (t.scalar_type() != at::kFloat || !t.is_cuda() || !t.is_contiguous() || t.numel() < elems)
    raise(PyExc_ValueError, "partials must be a contiguous fp32 device tensor of partial_elems elements");
  return static_cast<float*>(t.data_ptr());
}

[[maybe_unused]] int dtype_code(at::ScalarType t) {
  if (t == at::kFloat) return CLEAVE_F32;
  if (t == at::kBFloat16) return CLEAVE_BF16;
  PyErr_Format(PyExc_TypeError, "unsupported dtype torch.%s", c10::toString(t));
  throw Raised{};
}

[[maybe_unused]] int64_t integer(PyObject* o) {   // as int(o)
  if (PyLong_Check(o)) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return v;
  }
  PyObject* n = PyNumber_Long(o);
  if (!n) throw Raised{};
  const long long v = PyLong_AsLongLong(n);
  Py_DECREF(n);
  if (v == -1 && PyErr_Occurred()) throw Raised{};
  return v;
}

[[maybe_unused]] void* address(PyObject* o) {   // an int; None is null
  if (o == Py_None) return nullptr;
  void* p = PyLong_AsVoidPtr(o);
  if (!p && PyErr_Occurred()) throw Raised{};
  return p;
}

// None: torch's current stream; else an object with a `cuda_stream` (None there is
// the null stream), or an address in any form that int() takes.
[[maybe_unused]] void* stream_of(PyObject* o) {
  if (o == Py_None) return c10::hip::getCurrentHIPStream().stream();
  if (PyLong_Check(o)) return address(o);
  if (PyObject* s = PyObject_GetAttrString(o, "cuda_stream")) {
    void* p = s == Py_None ? nullptr : PyLong_AsVoidPtr(s);
    Py_DECREF(s);
    if (!p && PyErr_Occurred()) throw Raised{};
    return p;
  }
  if (!PyErr_ExceptionMatches(PyExc_AttributeError)) throw Raised{};
  PyErr_Clear();
  PyObject* n = PyNumber_Long(o);
  if (!n) throw Raised{};
  void* p = PyLong_AsVoidPtr(n);
  Py_DECREF(n);
  if (!p && PyErr_Occurred()) throw Raised{};
  return p;
}

template <typename F>
PyObject* guarded(F&& body) {
  try {
    return body();
  } catch (const Raised&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

[[maybe_unused]] void expect_args(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) raise(PyExc_TypeError, "wrong number of arguments");
}


template <typename F>
PyCFunction as_function(F* f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(f));
}

}  // namespace
