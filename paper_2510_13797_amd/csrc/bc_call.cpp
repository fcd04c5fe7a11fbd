// The Python calls of a decode step (over slabs; over pages, append and attention) of the C ABI, as CPython functions: addresses of tensors and structures to the entry point without a Python
// frame or a ctypes conversion for each.  What it gives is host time: the conversions were 2.1 us of a call of 6.7, now 0.9.  (A pass of 16 small steps, called one by
// one, 98 to 109 us, differs from run to run by more than that.)  The entry point's address comes with every call: nothing is kept here.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <cstddef>
#include <cstdint>

namespace {

using DecodeStep = int32_t (*)(const void*, const void*, const void*, const void*, const void*, float*, const void*, const void*,
                               const uint8_t*, void*, size_t, void*);

PyObject* data_ptr_name;

// Address of a tensor (None: null).  False with a Python error set.
bool tensor_address(PyObject* t, void** at) {
  *at = nullptr;
  if (t == Py_None) return true;
  PyObject* n = PyObject_CallMethodNoArgs(t, data_ptr_name);
  if (n == nullptr) return false;
  *at = PyLong_AsVoidPtr(n);
  Py_DECREF(n);
  return *at != nullptr || PyErr_Occurred() == nullptr;
}

// decode_step(entry point, shape, cache, k, v, q, out, beacon_k, beacon_v, active, workspace, workspace_bytes, stream) -> status
// shape, cache: ctypes structures; k ... workspace: tensors or None; the rest: numbers.
PyObject* decode_step(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 13) return PyErr_Format(PyExc_TypeError, "decode_step takes 13 arguments (%zd given)", n);
  const DecodeStep call = reinterpret_cast<DecodeStep>(PyLong_AsVoidPtr(args[0]));
  if (call == nullptr) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "decode_step: no entry point");
    return nullptr;
  }
  const size_t bytes = PyLong_AsSize_t(args[11]);
  if (bytes == static_cast<size_t>(-1) && PyErr_Occurred()) return nullptr;
  void* stream = PyLong_AsVoidPtr(args[12]);
  if (stream == nullptr && PyErr_Occurred()) return nullptr;
  void* at[8];
  for (int i = 0; i < 8; ++i)
    if (!tensor_address(args[3 + i], &at[i])) return nullptr;
  Py_buffer shape, cache;
  if (PyObject_GetBuffer(args[1], &shape, PyBUF_SIMPLE) != 0) return nullptr;
  if (PyObject_GetBuffer(args[2], &cache, PyBUF_SIMPLE) != 0) {
    PyBuffer_Release(&shape);
    return nullptr;
  }
  int32_t status;
  Py_BEGIN_ALLOW_THREADS      // (as ctypes does)
  status = call(shape.buf, cache.buf, at[0], at[1], at[2], static_cast<float*>(at[3]), at[4], at[5], static_cast<const uint8_t*>(at[6]), at[7],
                bytes, stream);
  Py_END_ALLOW_THREADS
  PyBuffer_Release(&cache);
  PyBuffer_Release(&shape);
  return PyLong_FromLong(status);
}

using PagedAppend = int32_t (*)(const void*, const void*, int64_t, const int64_t*, int32_t, const void*, int64_t, const int32_t*, const float*, int32_t,
                                const void*, const void*, float, const int32_t*, const uint8_t*, void*, void*);
using PagedAttend = int32_t (*)(const void*, const void*, int64_t, const int64_t*, int32_t, const void*, float*, const uint8_t*, void*, size_t, void*);

// An argument that is an entry point.
template <typename Call>
Call entry_point(PyObject* x) {
  const Call call = reinterpret_cast<Call>(PyLong_AsVoidPtr(x));
  if (call == nullptr && !PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "no entry point");
  return call;
}
bool number(PyObject* x, int64_t* to) {
  *to = PyLong_AsLongLong(x);
  return *to != -1 || PyErr_Occurred() == nullptr;
}
bool number32(PyObject* x, int32_t* to) {
  int64_t n;
  if (!number(x, &n)) return false;
  if (n != static_cast<int32_t>(n)) {
    PyErr_SetString(PyExc_OverflowError, "a number does not fit 32 bits");
    return false;
  }
  *to = static_cast<int32_t>(n);
  return true;
}
bool stream_of(PyObject* x, void** to) {
  *to = PyLong_AsVoidPtr(x);
  return *to != nullptr || PyErr_Occurred() == nullptr;
}
// Two ctypes structures, held while a call runs.
struct Structures {
  Py_buffer a{}, b{};
  int held = 0;
  bool get(PyObject* x, PyObject* y) {
    if (PyObject_GetBuffer(x, &a, PyBUF_SIMPLE) != 0) return false;
    held = 1;
    if (PyObject_GetBuffer(y, &b, PyBUF_SIMPLE) != 0) return false;
    held = 2;
    return true;
  }
  ~Structures() {
    if (held > 1) PyBuffer_Release(&b);
    if (held > 0) PyBuffer_Release(&a);
  }
};

// paged_append(entry point, shape, pages, rows, row_offsets, max_new, qkv, stride, positions, inv_freq, rot, q_weight, k_weight, eps, keep, active, q, stream) -> status
PyObject* paged_append(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 18) return PyErr_Format(PyExc_TypeError, "paged_append takes 18 arguments (%zd given)", n);
  const auto call = entry_point<PagedAppend>(args[0]);
  int64_t rows, stride;
  int32_t max_new, rot;
  void *off, *qkv, *positions, *inv_freq, *qw, *kw, *keep, *active, *q, *stream;
  const double eps = PyFloat_AsDouble(args[13]);
  if (call == nullptr || (eps == -1.0 && PyErr_Occurred()) || !number(args[3], &rows) || !tensor_address(args[4], &off) || !number32(args[5], &max_new) ||
      !tensor_address(args[6], &qkv) || !number(args[7], &stride) || !tensor_address(args[8], &positions) || !tensor_address(args[9], &inv_freq) ||
      !number32(args[10], &rot) || !tensor_address(args[11], &qw) || !tensor_address(args[12], &kw) || !tensor_address(args[14], &keep) ||
      !tensor_address(args[15], &active) || !tensor_address(args[16], &q) || !stream_of(args[17], &stream))
    return nullptr;
  Structures s;
  if (!s.get(args[1], args[2])) return nullptr;
  int32_t status;
  Py_BEGIN_ALLOW_THREADS
  status = call(s.a.buf, s.b.buf, rows, static_cast<const int64_t*>(off), max_new, qkv, stride, static_cast<const int32_t*>(positions),
                static_cast<const float*>(inv_freq), rot, qw, kw, static_cast<float>(eps), static_cast<const int32_t*>(keep),
                static_cast<const uint8_t*>(active), q, stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

// paged_attend(entry point, shape, pages, rows, row_offsets, max_new, q, out, active, workspace, workspace_bytes, stream) -> status
PyObject* paged_attend(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 12) return PyErr_Format(PyExc_TypeError, "paged_attend takes 12 arguments (%zd given)", n);
  const auto call = entry_point<PagedAttend>(args[0]);
  int64_t rows, bytes;
  int32_t max_new;
  void *off, *q, *out, *active, *workspace, *stream;
  if (call == nullptr || !number(args[3], &rows) || !tensor_address(args[4], &off) || !number32(args[5], &max_new) || !tensor_address(args[6], &q) ||
      !tensor_address(args[7], &out) || !tensor_address(args[8], &active) || !tensor_address(args[9], &workspace) || !number(args[10], &bytes) ||
      !stream_of(args[11], &stream))
    return nullptr;
  if (bytes < 0) return PyErr_Format(PyExc_OverflowError, "workspace_bytes is negative");
  Structures s;
  if (!s.get(args[1], args[2])) return nullptr;
  int32_t status;
  Py_BEGIN_ALLOW_THREADS
  status = call(s.a.buf, s.b.buf, rows, static_cast<const int64_t*>(off), max_new, q, static_cast<float*>(out), static_cast<const uint8_t*>(active), workspace,
                static_cast<size_t>(bytes), stream);
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}

PyMethodDef methods[] = {
    {"paged_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_append)), METH_FASTCALL, nullptr},
    {"paged_attend", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_attend)), METH_FASTCALL, nullptr},
    {"decode_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(decode_step)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_bc_call", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__bc_call() {
  data_ptr_name = PyUnicode_InternFromString("data_ptr");
  return data_ptr_name == nullptr ? nullptr : PyModule_Create(&module);
}
