// What the native parts of the Python binding share: arguments into tensors, addresses and numbers, allocation, the current stream, errors.
#ifndef SBP_BINDING_H_
#define SBP_BINDING_H_

#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/device_lazy_init.h>

#include "sbp.h"

namespace {

PyObject* f_check = nullptr;          // _lib.check: raises for a negative status
PyObject* f_stream = nullptr;         // device index -> handle of torch's current stream there

struct PyFail {};                     // a Python error is set

[[noreturn]] void fail(PyObject* type, const char* fmt, const char* what) {
  PyErr_Format(type, fmt, what);
  throw PyFail{};
}

// the tensor of an argument, or nullptr for None
const at::Tensor* tensor(PyObject* o, const char* name) {
  if (o == Py_None) return nullptr;
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "%s must be a tensor", name);
  return &THPVariable_Unpack(o);
}
const at::Tensor& needed(PyObject* o, const char* name) {
  const at::Tensor* t = tensor(o, name);
  if (!t) fail(PyExc_TypeError, "%s must be a tensor", name);
  return *t;
}

[[maybe_unused]] void* dev(const at::Tensor* t, const char* name) {
  if (!t) return nullptr;
  if (!t->is_cuda()) fail(PyExc_ValueError, "%s must live in GPU memory", name);
  if (!t->is_contiguous()) fail(PyExc_ValueError, "%s must be contiguous", name);
  return t->data_ptr();
}

int32_t dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return SBP_F32;
  if (t.scalar_type() == at::kBFloat16) return SBP_BF16;
  PyErr_Format(PyExc_TypeError, "unsupported dtype %S; use float32 or bfloat16", reinterpret_cast<PyObject*>(torch::getTHPDtype(t.scalar_type())));
  throw PyFail{};
}

// Other Python threads run while memory is allocated or work is enqueued (either may block).
struct WithoutGil {
  PyThreadState* state = PyEval_SaveThread();
  ~WithoutGil() { PyEval_RestoreThread(state); }
};

// as torch.empty: a process that has not used the GPU yet gets torch.cuda's initialization (and with it the fork check), a child
// forked from one that has gets torch's error
at::Tensor empty(at::IntArrayRef sizes, at::ScalarType type, c10::Device device) {
  if (device.is_cuda()) torch::utils::device_lazy_init(at::kCUDA);
  WithoutGil no_gil;
  return at::empty(sizes, at::TensorOptions().dtype(type).device(device));
}

void* stream_of(c10::Device device) {
  PyObject* index = PyLong_FromLong(device.index());
  if (!index) throw PyFail{};
  PyObject* h = PyObject_CallFunctionObjArgs(f_stream, index, nullptr);
  Py_DECREF(index);
  if (!h) throw PyFail{};
  void* s = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  if (!s && PyErr_Occurred()) throw PyFail{};
  return s;
}

void check(int64_t status) {
  if (status >= 0) return;
  PyObject* r = PyObject_CallFunction(f_check, "L", (long long)status);
  Py_XDECREF(r);
  if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, "libsbp call failed");
  throw PyFail{};
}

template <class F>
int32_t enqueue(F&& f) {
  WithoutGil no_gil;
  return f();
}

int64_t integer(PyObject* o, bool whole = false) {                   // whole: numbers that int() would round are refused
  PyObject* n = whole ? PyNumber_Index(o) : PyNumber_Long(o);
  if (!n) throw PyFail{};
  const long long v = PyLong_AsLongLong(n);
  Py_DECREF(n);
  if (v == -1 && PyErr_Occurred()) throw PyFail{};
  return v;
}
[[maybe_unused]] int32_t integer32(PyObject* o) { return (int32_t)integer(o); }       // (as a C int field takes it: the low 32 bits)
[[maybe_unused]] uint64_t bits64(PyObject* o, bool whole = false) {
  PyObject* n = whole ? PyNumber_Index(o) : PyNumber_Long(o);
  if (!n) throw PyFail{};
  const unsigned long long v = PyLong_AsUnsignedLongLongMask(n);
  Py_DECREF(n);
  if (v == (unsigned long long)-1 && PyErr_Occurred()) throw PyFail{};
  return v;
}

PyObject* wrap(const at::Tensor& t) { return THPVariable_Wrap(t); }
PyObject* keep_or_wrap(PyObject* given, const at::Tensor& made) {
  if (given != Py_None) { Py_INCREF(given); return given; }
  if (!made.defined()) Py_RETURN_NONE;
  return wrap(made);
}

[[maybe_unused]] PyObject* pack(std::initializer_list<PyObject*> items) {
  bool ok = true;
  for (PyObject* o : items) ok = ok && o;
  PyObject* r = ok ? PyTuple_New((Py_ssize_t)items.size()) : nullptr;
  Py_ssize_t i = 0;
  for (PyObject* o : items) {
    if (r) PyTuple_SET_ITEM(r, i++, o);
    else Py_XDECREF(o);
  }
  return r;
}

void count(Py_ssize_t n, Py_ssize_t want) {
  if (n != want) fail(PyExc_TypeError, "%s", "wrong number of arguments");
}

}  // namespace
#endif
