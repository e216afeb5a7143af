// Looks at the tensors of a call in one go for the Python front end (binding.py): a call of fifteen small tensors otherwise spends
// more of the host's time on their attributes, one interpreted call each, than the GPU spends on the call.
//
//   look(where, like, spec, *tensors) -> (index of like's GPU, then for each tensor what its kind gives)
//
// spec: one string per tensor, its kind and its name:
//   'i', 'f'  int32 / float32, contiguous                                 -> address, elements
//   'r'       rows of like's type, contiguous but for the first dimension -> address, elements between rows (0: all contiguous), sizes
//   'c'       contiguous of any type                                      -> address, sizes
// None gives zeros and an empty tuple.  Every tensor is on like's GPU.  What does not hold raises the error that set_error() was given,
// as error(hook_status, text).
#include <ATen/core/Tensor.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

namespace {

enum Status { kNull = 1, kShape = 2, kUnsupported = 3 };
PyObject* g_error = nullptr;

PyObject* refuse(Status status, PyObject* where, const char* name, const char* what) {
  PyObject* text = PyUnicode_FromFormat("%U (%s%s%s)", where, name, *name ? ": " : "", what);
  PyObject* error = text && g_error ? PyObject_CallFunction(g_error, "iO", (int)status, text) : nullptr;
  Py_XDECREF(text);
  if (error) {
    PyErr_SetObject((PyObject*)Py_TYPE(error), error);
    Py_DECREF(error);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, what);
  }
  return nullptr;
}

PyObject* sizes_of(const at::Tensor& t) {
  const auto s = t.sizes();
  PyObject* out = PyTuple_New((Py_ssize_t)s.size());
  if (!out) return nullptr;
  for (size_t i = 0; i < s.size(); ++i) {
    PyObject* n = PyLong_FromLongLong(s[i]);
    if (!n) { Py_DECREF(out); return nullptr; }
    PyTuple_SET_ITEM(out, (Py_ssize_t)i, n);
  }
  return out;
}

// Elements between rows that are contiguous themselves; -1: they are not, or lie on top of each other.
int64_t row_stride(const at::Tensor& t) {
  if (t.is_contiguous()) return 0;
  int64_t row = 1;
  for (int64_t i = t.dim() - 1; i > 0; --i) {
    if (t.size(i) != 1 && t.stride(i) != row) return -1;
    row *= t.size(i);
  }
  return t.dim() > 0 && t.stride(0) >= row ? t.stride(0) : -1;
}

PyObject* look_at(PyObject* const* a, Py_ssize_t n) {
  if (n < 3 || !PyUnicode_Check(a[0]) || !PyTuple_Check(a[2]) || PyTuple_GET_SIZE(a[2]) != n - 3) {
    PyErr_SetString(PyExc_TypeError, "look(where, like, spec, *tensors)");
    return nullptr;
  }
  PyObject* const where = a[0];
  if (a[1] == Py_None) return refuse(kNull, where, "", "no tensor");
  if (!THPVariable_Check(a[1])) return refuse(kUnsupported, where, "", "not a tensor");
  const at::Tensor& like = THPVariable_Unpack(a[1]);
  if (!like.is_cuda()) return refuse(kUnsupported, where, "", "device");
  const auto device = like.device();
  Py_ssize_t total = 1;
  for (Py_ssize_t i = 3; i < n; ++i) {
    const char* spec = PyUnicode_AsUTF8(PyTuple_GET_ITEM(a[2], i - 3));
    if (!spec) return nullptr;
    total += *spec == 'r' ? 3 : 2;
  }
  PyObject* out = PyTuple_New(total);
  if (!out) return nullptr;
  Py_ssize_t at = 0;
  bool ok = true;
  auto give = [&](PyObject* x) {
    if (!x) ok = false;
    else PyTuple_SET_ITEM(out, at++, x);
  };
  give(PyLong_FromLong(device.index()));
  for (Py_ssize_t i = 3; ok && i < n; ++i) {
    const char* spec = PyUnicode_AsUTF8(PyTuple_GET_ITEM(a[2], i - 3));
    const char kind = *spec, *name = spec + 1;
    if (a[i] == Py_None) {
      give(PyLong_FromLong(0));
      if (kind != 'c') give(PyLong_FromLong(0));
      if (kind == 'c' || kind == 'r') give(PyTuple_New(0));
      continue;
    }
    if (!THPVariable_Check(a[i])) { refuse(kUnsupported, where, name, "not a tensor"); ok = false; break; }
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    const auto type = t.scalar_type();
    if (t.device() != device) { refuse(kUnsupported, where, name, "device"); ok = false; break; }
    if ((kind == 'i' && type != at::kInt) || (kind == 'f' && type != at::kFloat) || (kind == 'r' && type != like.scalar_type())) {
      refuse(kUnsupported, where, name, "dtype"); ok = false; break;
    }
    const int64_t stride = kind == 'r' ? row_stride(t) : t.is_contiguous() ? 0 : -1;
    if (stride < 0) { refuse(kShape, where, name, "layout"); ok = false; break; }
    give(PyLong_FromUnsignedLongLong((unsigned long long)(uintptr_t)(t.numel() ? t.data_ptr() : nullptr)));
    if (kind == 'r') give(PyLong_FromLongLong(stride));
    give(kind == 'r' || kind == 'c' ? sizes_of(t) : PyLong_FromLongLong(t.numel()));
  }
  if (!ok) { Py_DECREF(out); return nullptr; }
  return out;
}

// (a tensor without storage, say a sparse one, throws)
PyObject* look(PyObject*, PyObject* const* a, Py_ssize_t n) {
  try {
    return look_at(a, n);
  } catch (const std::exception&) {
    return refuse(kUnsupported, a[0], "", "not a plain tensor");
  }
}

PyObject* set_error(PyObject*, PyObject* error) {
  Py_INCREF(error);
  Py_XDECREF(g_error);
  g_error = error;
  Py_RETURN_NONE;
}

PyMethodDef methods[] = {{"look", (PyCFunction)(void*)look, METH_FASTCALL, "look(where, like, spec, *tensors)"},
                         {"set_error", set_error, METH_O, "set_error(type): what look() raises"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
