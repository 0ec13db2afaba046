// Checks of torch tensors for the Python binding's per-step calls (page plans, paged appends,
// prefix attention).  A decoding step makes such calls for every layer, and asking every tensor for
// its type, size, layout and address from Python takes longer than all else the binding does: the
// host's part of a page plan before its launch took 3.4 us so, and takes 1.9 us.  Nothing is kept
// between calls.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <exception>

#include "../../include/jolt.h"

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

// The address of memory for `need` elements of `type` (nullptr: bytes, of any type): None is 0, a
// whole number an address that the caller answers for, a tensor one of that type, or of plain bytes,
// whose storage reaches that far from its first element.  Returns false with an error set.
bool memory(PyObject *o, const at::ScalarType *type, __int128 need, const char *name, PyObject *&out) {
  if (o == Py_None) return (out = PyLong_FromLong(0)) != nullptr;
  if (PyLong_Check(o)) {
    Py_INCREF(o);
    out = o;
    return true;
  }
  const at::Tensor *t = tensor(o, name);
  if (!t) return false;
  if (type && t->scalar_type() != *type && t->scalar_type() != at::kByte) {
    PyErr_Format(PyExc_ValueError, "%s must be a %s tensor", name, *type == at::kBFloat16 ? "bfloat16" : "float32");
    return false;
  }
  const __int128 held = (__int128)t->storage().nbytes() - (__int128)t->storage_offset() * t->element_size();
  if (held / (type ? (int)at::elementSize(*type) : 1) < need) {
    PyErr_Format(PyExc_ValueError, "%s: the call reaches %lld %s, more than the tensor's memory holds from its first element on", name,
                 (long long)need, type ? "elements" : "bytes");
    return false;
  }
  if (!t->is_cuda()) {
    PyErr_Format(PyExc_ValueError, "%s must be a tensor on the GPU", name);
    return false;
  }
  return (out = address(*t)) != nullptr;
}

// A descriptor of the binding, as the library reads it.
template <class D>
bool descriptor(PyObject *o, const char *name, D &d) {
  Py_buffer b;
  if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE)) return false;
  const bool fits = b.len == (Py_ssize_t)sizeof(D);
  if (fits) std::memcpy(&d, b.buf, sizeof(D));
  else PyErr_Format(PyExc_ValueError, "%s has the wrong size", name);
  PyBuffer_Release(&b);
  return fits;
}

PyObject *two(PyObject *K, const char *k_name, PyObject *V, const char *v_name, int dtype, __int128 need) {
  const at::ScalarType type = dtype == JOLT_BF16 ? at::kBFloat16 : at::kFloat;
  PyObject *k = nullptr, *v = nullptr;
  if (!memory(K, &type, need, k_name, k)) return nullptr;
  if (!memory(V, &type, need, v_name, v)) {
    Py_DECREF(k);
    return nullptr;
  }
  return Py_BuildValue("(NN)", k, v);
}

// pools(descriptor, K_pages, V_pages): their addresses.
PyObject *pools(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> PyObject * {
    if (n != 3) return PyErr_Format(PyExc_TypeError, "pools(descriptor, K_pages, V_pages)");
    jolt_page_desc p;
    if (!descriptor(a[0], "pages", p)) return nullptr;
    return two(a[1], "K_pages", a[2], "V_pages", p.dtype,
               ((__int128)p.n_pages - 1) * p.stride_page + ((__int128)p.n_heads - 1) * p.stride_head +
                   ((__int128)p.page_size - 1) * p.stride_token + p.d);
  });
}

// cell(descriptor, layer, K_prefix, V_prefix): addresses of the cell's keys and values, of which a
// call reads that layer (one that the cell does not have is the library's to refuse).
PyObject *cell(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> PyObject * {
    if (n != 4) return PyErr_Format(PyExc_TypeError, "cell(descriptor, layer, K_prefix, V_prefix)");
    jolt_cell_desc c;
    const long long layer = PyLong_AsLongLong(a[1]);
    if (PyErr_Occurred() || !descriptor(a[0], "prefix", c)) return nullptr;
    return two(a[2], "K_prefix", a[3], "V_prefix", c.dtype,
               (layer < c.n_layers ? (__int128)layer : 0) * c.stride_layer + ((__int128)c.n_heads - 1) * c.stride_head +
                   ((__int128)c.T - 1) * c.stride_token + c.d);
  });
}

// bytes(tensor or address, bytes or None, name): (address, bytes); None takes the tensor's own.
PyObject *bytes(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> PyObject * {
    if (n != 3) return PyErr_Format(PyExc_TypeError, "bytes(tensor, bytes, name)");
    const char *name = PyUnicode_AsUTF8(a[2]);
    if (!name) return nullptr;
    long long need = 0;
    if (a[1] != Py_None) {
      need = PyLong_AsLongLong(a[1]);
      if (PyErr_Occurred()) return nullptr;
      if (need < 0) return PyErr_Format(PyExc_ValueError, "%s: negative size", name);
    } else {
      if (PyLong_Check(a[0])) return PyErr_Format(PyExc_ValueError, "%s: an address needs its size beside it", name);
      const at::Tensor *t = tensor(a[0], name);
      if (!t) return nullptr;
      need = t->numel() * (long long)t->element_size();
    }
    PyObject *p = nullptr;
    return memory(a[0], nullptr, need, name, p) ? Py_BuildValue("(NL)", p, need) : nullptr;
  });
}

// columns(tensor, rows, name): the columns of a [rows, columns] tensor.
PyObject *columns(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded([&]() -> PyObject * {
    if (n != 3) return PyErr_Format(PyExc_TypeError, "columns(tensor, rows, name)");
    const long long rows = PyLong_AsLongLong(a[1]);
    const char *name = PyUnicode_AsUTF8(a[2]);
    if (!name || PyErr_Occurred()) return nullptr;
    const at::Tensor *t = tensor(a[0], name);
    if (!t) return nullptr;
    if (t->dim() != 2 || t->size(0) != rows) return PyErr_Format(PyExc_ValueError, "%s must be [n_req, max_pages]", name);
    return PyLong_FromLongLong(t->size(1));
  });
}

PyMethodDef methods[] = {
    {"flat", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(flat)), METH_FASTCALL, "addresses of contiguous tensors"},
    {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rows)), METH_FASTCALL, "address, shape and strides of rows"},
    {"pools", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(pools)), METH_FASTCALL, "addresses of two pools of pages"},
    {"cell", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(cell)), METH_FASTCALL, "addresses of a cell's keys and values"},
    {"bytes", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(bytes)), METH_FASTCALL, "address and bytes of a workspace"},
    {"columns", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(columns)), METH_FASTCALL, "columns of a table"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "Checks of torch tensors for the binding.", -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
