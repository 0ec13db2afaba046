// Checks of torch tensors for the Python binding's per-step calls (page plans, paged appends,
// prefix attention).  A decoding step makes such calls for every layer, and asking every tensor for
// its type, size, layout and address from Python takes longer than all else the binding does: the
// host's part of a page plan before its launch took 3.4 us so, and takes 1.9 us.  Nothing is kept
// between calls.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <exception>

namespace {

const at::Tensor *tensor(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_ValueError, "%s must be a tensor", name);
    return nullptr;
  }
  return &THPVariable_Unpack(o);
}

PyObject *address(const at::Tensor &t) { return PyLong_FromVoidPtr(t.data_ptr()); }

// No C++ exception leaves an entry point.
template <class F>
PyObject *guarded(F f) {
  try {
    return f();
  } catch (const std::exception &e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, e.what());
  } catch (...) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "unknown error");
  }
  return nullptr;
}

// flat(type, tensor, elements, name, tensor, elements, name, ...): addresses of contiguous GPU
// tensors of that type ("i" int32, "f" float32) and size.
PyObject *flat(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> PyObject * {
    if (n < 1 || n % 3 != 1) return PyErr_Format(PyExc_TypeError, "flat(type, tensor, elements, name, ...)");
    const char *type = PyUnicode_AsUTF8(a[0]);
    if (!type) return nullptr;
    const bool ints = type[0] == 'i';
    PyObject *out = PyTuple_New(n / 3);
    if (!out) return nullptr;
    for (Py_ssize_t i = 0; i < n / 3; ++i) {
      const char *name = PyUnicode_AsUTF8(a[3 * i + 3]);
      const long long count = PyLong_AsLongLong(a[3 * i + 2]);
      const at::Tensor *t = name && !PyErr_Occurred() ? tensor(a[3 * i + 1], name) : nullptr;
      if (t && !(t->scalar_type() == (ints ? at::kInt : at::kFloat) && t->numel() == count && t->is_contiguous() && t->is_cuda())) {
        PyErr_Format(PyExc_ValueError, "%s must be a contiguous %s tensor of %lld elements on the GPU", name,
                     ints ? "int32" : "float32", count);
        t = nullptr;
      }
      PyObject *p = t ? address(*t) : nullptr;
      if (!p) {
        Py_DECREF(out);
        return nullptr;
      }
      PyTuple_SET_ITEM(out, i, p);
    }
    return out;
  });
}

// rows(tensor, bf16, rows or -1, heads or -1, d, name): (address, rows, heads, row stride, head
// stride) of a [rows, heads, d] GPU tensor with contiguous features; the stride of an axis of one
// element, which is never used and may be anything, is given as 0.
PyObject *rows(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> PyObject * {
    if (n != 6) return PyErr_Format(PyExc_TypeError, "rows(tensor, bf16, rows, heads, d, name)");
    const int bf16 = PyObject_IsTrue(a[1]);
    const long long nr = PyLong_AsLongLong(a[2]), nh = PyLong_AsLongLong(a[3]), d = PyLong_AsLongLong(a[4]);
    const char *name = PyUnicode_AsUTF8(a[5]);
    if (bf16 < 0 || !name || PyErr_Occurred()) return nullptr;
    const at::Tensor *t = tensor(a[0], name);
    if (!t) return nullptr;
    if (!(t->scalar_type() == (bf16 ? at::kBFloat16 : at::kFloat) && t->is_cuda() && t->dim() == 3 && t->size(2) == d &&
          t->stride(2) == 1 && (nr < 0 || t->size(0) == nr) && (nh < 0 || t->size(1) == nh)))
      return PyErr_Format(PyExc_ValueError, "%s must be a [rows, heads, %lld] %s tensor on the GPU with contiguous features and "
                          "the call's rows and heads", name, d, bf16 ? "bfloat16" : "float32");
    const long long r = t->size(0), h = t->size(1);
    PyObject *p = address(*t);
    if (!p) return nullptr;
    return Py_BuildValue("(NLLLL)", p, r, h, r > 1 ? (long long)t->stride(0) : 0, h > 1 ? (long long)t->stride(1) : 0);
  });
}

PyMethodDef methods[] = {
    {"flat", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(flat)), METH_FASTCALL, "addresses of contiguous tensors"},
    {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rows)), METH_FASTCALL, "address, shape and strides of rows"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Checks of torch tensors for the binding.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
