// What the torch entry points of the operators ask of a tensor, in one call each (a Python extension, no GPU code): a call has a dozen tensors, and asked through Python's
// attributes each costs 0.5 us.  Every function returns None where the tensor is not the common case; the caller's own checks then say what is wrong with it.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <torch/csrc/Device.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>

namespace {

// Whether the storage of `t` reaches to its last element: a program may have freed it, or a part of it, and kept the tensor.
bool held(const at::Tensor& t) {
  if (t.numel() == 0) return true;
  int64_t last = t.storage_offset();
  for (int64_t d = 0; d < t.dim(); ++d) last += (t.size(d) - 1) * t.stride(d);
  return (size_t)(last + 1) * t.element_size() <= t.storage().nbytes();
}

// The tensor behind `o`, if it is one of this type on this device with nothing about it that the library's kernels do not know.
const at::Tensor* plain(PyObject* o, PyObject* device, PyObject* dtype) {
  if (!THPVariable_Check(o) || !THPDevice_Check(device) || !THPDtype_Check(dtype)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != at::kStrided || t.scalar_type() != ((THPDtype*)dtype)->scalar_type || t.device() != ((THPDevice*)device)->device ||
      t.is_neg() || t.is_conj() || t._is_zerotensor() || t.requires_grad() || !held(t))
    return nullptr;
  return &t;
}

PyObject* none() { Py_RETURN_NONE; }

// vector(t, device, dtype, n) -> the address of a contiguous vector of n elements
PyObject* vector(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4) { PyErr_SetString(PyExc_TypeError, "vector(t, device, dtype, n)"); return nullptr; }
  const long long want = PyLong_AsLongLong(a[3]);
  if (want == -1 && PyErr_Occurred()) return nullptr;
  try {
    const at::Tensor* t = plain(a[0], a[1], a[2]);
    if (!t || t->dim() != 1 || t->size(0) != want || !t->is_contiguous()) return none();
    return PyLong_FromUnsignedLongLong((unsigned long long)(uintptr_t)t->data_ptr());
  } catch (const std::exception&) {
    return none();
  }
}

// arrays(t, u, device, dtype, n) -> the addresses of two contiguous arrays of n elements each
PyObject* arrays(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 5) { PyErr_SetString(PyExc_TypeError, "arrays(t, u, device, dtype, n)"); return nullptr; }
  const long long want = PyLong_AsLongLong(a[4]);
  if (want == -1 && PyErr_Occurred()) return nullptr;
  try {
    const at::Tensor *t = plain(a[0], a[2], a[3]), *u = t ? plain(a[1], a[2], a[3]) : nullptr;
    if (!u || t->numel() != want || u->numel() != want || !t->is_contiguous() || !u->is_contiguous()) return none();
    return Py_BuildValue("KK", (unsigned long long)(uintptr_t)t->data_ptr(), (unsigned long long)(uintptr_t)u->data_ptr());
  } catch (const std::exception&) {
    return none();
  }
}

// rows(t, device, dtype, rows, cols) -> (address, distance of rows, rows, columns) of a matrix whose rows may lie apart; rows, cols: -1 for any
PyObject* rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 5) { PyErr_SetString(PyExc_TypeError, "rows(t, device, dtype, rows, cols)"); return nullptr; }
  const long long want_rows = PyLong_AsLongLong(a[3]), want_cols = PyLong_AsLongLong(a[4]);
  if (PyErr_Occurred()) return nullptr;
  try {
    const at::Tensor* t = plain(a[0], a[1], a[2]);
    if (!t || t->dim() != 2) return none();
    const long long r = t->size(0), c = t->size(1);
    if ((want_rows >= 0 && r != want_rows) || (want_cols >= 0 && c != want_cols) || r >= 1ll << 31 || c >= 1ll << 31) return none();
    if (c > 1 && t->stride(1) != 1) return none();
    const void* at = t->data_ptr();
    if (!at && r && c) return none();                  // (no address would stand for no tensor)
    return Py_BuildValue("KLLL", (unsigned long long)(uintptr_t)at, (long long)t->stride(0), r, c);
  } catch (const std::exception&) {
    return none();
  }
}

// empty(rows, cols, dtype, device) -> a new matrix, its contents not set
PyObject* empty(PyObject*, PyObject* const* a, Py_ssize_t n) {
  if (n != 4 || !THPDtype_Check(a[2]) || !THPDevice_Check(a[3])) { PyErr_SetString(PyExc_TypeError, "empty(rows, cols, dtype, device)"); return nullptr; }
  const long long r = PyLong_AsLongLong(a[0]), c = PyLong_AsLongLong(a[1]);
  if (PyErr_Occurred()) return nullptr;
  HANDLE_TH_ERRORS
  return THPVariable_Wrap(at::empty({r, c}, at::TensorOptions().dtype(((THPDtype*)a[2])->scalar_type).device(((THPDevice*)a[3])->device)));
  END_HANDLE_TH_ERRORS
}

// written(t, ...): tensors that were written in place; those of inference mode count no versions
PyObject* written(PyObject*, PyObject* const* a, Py_ssize_t n) {
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (!THPVariable_Check(a[i])) { PyErr_SetString(PyExc_TypeError, "written(tensor, ...)"); return nullptr; }
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  }
  return none();
}

PyMethodDef methods[] = {{"vector", (PyCFunction)(void*)vector, METH_FASTCALL, "vector(t, device, dtype, n) -> address or None"},
                         {"arrays", (PyCFunction)(void*)arrays, METH_FASTCALL, "arrays(t, u, device, dtype, n) -> two addresses or None"},
                         {"rows", (PyCFunction)(void*)rows, METH_FASTCALL, "rows(t, device, dtype, rows, cols) -> (address, distance, rows, columns) or None"},
                         {"empty", (PyCFunction)(void*)empty, METH_FASTCALL, "empty(rows, cols, dtype, device) -> a new matrix"},
                         {"written", (PyCFunction)(void*)written, METH_FASTCALL, "written(t, ...): their versions go up"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", "What the operators ask of their tensors.", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors(void) { return PyModule_Create(&module); }
