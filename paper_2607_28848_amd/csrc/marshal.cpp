// marshal.cpp -- checks and packing of a call's tensors for the Python bindings (a CPython module, _marshal).
//
// The calls of a decode step take the GPU 3 to 10 us each, and reading a tensor's type, shape, strides and address from
// Python takes the host 0.8 us a tensor: with eleven tensors the rotation's call was bound by that (8 rows: 11.7 us a call;
// 7.3 with this module).
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <string>

namespace {

// The library's view of a tensor: address, row and head stride in elements (0: dense).
struct View {
  void* ptr;
  int64_t row, head;
};
static_assert(sizeof(View) == 24, "dsv_attn_view");

bool tensor(PyObject* o, PyObject* name, const at::Tensor** t) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%S must be a tensor, got %R", name, reinterpret_cast<PyObject*>(Py_TYPE(o)));
    return false;
  }
  *t = &THPVariable_Unpack(o);
  return true;
}

bool same_type(const at::Tensor& t, PyObject* dtype) {
  return THPDtype_Check(dtype) && t.scalar_type() == reinterpret_cast<THPDtype*>(dtype)->scalar_type;
}

bool whole(PyObject* o, int64_t* x) {
  *x = PyLong_AsLongLong(o);
  return !(*x == -1 && PyErr_Occurred());
}

// view(t, rows, heads, d, dtype, name) -> 24 bytes: t as a tensor [rows][heads][d], or [rows][heads * d], of contiguous heads.
PyObject* view(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  int64_t rows, heads, d;
  if (n != 6) return PyErr_Format(PyExc_TypeError, "view takes 6 arguments");
  const at::Tensor* t = nullptr;
  PyObject* const name = a[5];
  if (!tensor(a[0], name, &t) || !whole(a[1], &rows) || !whole(a[2], &heads) || !whole(a[3], &d)) return nullptr;
  if (!same_type(*t, a[4]))
    return PyErr_Format(PyExc_TypeError, "%S is %s, the call's tensors are %S", name, c10::toString(t->scalar_type()), a[4]);
  const auto shape = t->sizes(), stride = t->strides();
  int64_t row, head, one;
  if (shape.size() == 3 && shape[0] == rows && shape[1] == heads && shape[2] == d) {
    row = stride[0], head = stride[1], one = stride[2];
  } else if (shape.size() == 2 && shape[0] == rows && shape[1] == heads * d) {
    row = stride[0], head = d * stride[1], one = stride[1];
  } else {
    std::string got;
    for (const int64_t x : shape) got += (got.empty() ? "" : ", ") + std::to_string(x);
    if (shape.size() == 1) got += ',';
    return PyErr_Format(PyExc_ValueError, "%S must be [%lld][%lld][%lld], got (%s)", name, (long long)rows, (long long)heads,
                        (long long)d, got.c_str());
  }
  if (one != 1 && rows) return PyErr_Format(PyExc_ValueError, "%S: the elements of a head must be contiguous", name);
  // the library takes a stride of 0 for the dense one
  if ((row == 0 && rows > 1) || (head == 0 && heads > 1 && rows > 0))
    return PyErr_Format(PyExc_ValueError, "%S is broadcast (a stride of 0): make it contiguous", name);
  // a stride of a dimension of one is arbitrary: the dense one then
  const View v = {t->data_ptr(), rows > 1 ? row : 0, heads > 1 && rows > 0 ? head : 0};
  return PyBytes_FromStringAndSize(reinterpret_cast<const char*>(&v), sizeof(v));
  END_HANDLE_TH_ERRORS
}

// vec(t, n, dtype, name) -> the address of a contiguous vector of n elements, 0 for None.
PyObject* vec(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  int64_t len;
  if (n != 4) return PyErr_Format(PyExc_TypeError, "vec takes 4 arguments");
  if (a[0] == Py_None) return PyLong_FromLong(0);
  const at::Tensor* t = nullptr;
  if (!tensor(a[0], a[3], &t) || !whole(a[1], &len)) return nullptr;
  const auto shape = t->sizes();
  if (!same_type(*t, a[2]) || shape.size() != 1 || shape[0] != len || !t->is_contiguous())
    return PyErr_Format(PyExc_ValueError, "%S must be a contiguous %S tensor of %lld elements", a[3], a[2], (long long)len);
  return PyLong_FromVoidPtr(t->data_ptr());
  END_HANDLE_TH_ERRORS
}

// where(*tensors) -> the GPU that the tensors (None: not given) are on, -1 where all of them are in host memory; ValueError
// where they differ, or have no memory.  Tensors without elements are anywhere, as is pinned host memory, which every GPU
// reads and writes: -2 where there are no others.
PyObject* where(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const at::Tensor* first = nullptr;
  for (Py_ssize_t i = 0; i < n; ++i) {
    if (a[i] == Py_None) continue;
    if (!THPVariable_Check(a[i])) return PyErr_Format(PyExc_TypeError, "not a tensor: %R", a[i]);
    const at::Tensor& t = THPVariable_Unpack(a[i]);
    if (t.is_meta()) return PyErr_Format(PyExc_ValueError, "a tensor of the call has no memory");
    if (t.numel() == 0 || (t.is_cpu() && t.is_pinned())) continue;
    if (!first) {
      first = &t;
    } else if (t.device() != first->device()) {
      return PyErr_Format(PyExc_ValueError, "the tensors of a call are on several devices: %s, %s", first->device().str().c_str(),
                          t.device().str().c_str());
    }
  }
  return PyLong_FromLong(!first ? -2 : first->is_cpu() ? -1 : first->device().index());
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {{"view", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(view)), METH_FASTCALL, nullptr},
                         {"vec", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(vec)), METH_FASTCALL, nullptr},
                         {"where", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(where)), METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// The module reads torch's tensors as its headers lay them out: ImportError under another torch or Python than it was built for
// (DSV_TORCH: torch.__version__ then).
PyMODINIT_FUNC PyInit__marshal() {
  const std::string python = std::to_string(PY_MAJOR_VERSION) + "." + std::to_string(PY_MINOR_VERSION) + ".";
  PyObject* torch = PyImport_ImportModule("torch");
  PyObject* version = torch ? PyObject_GetAttrString(torch, "__version__") : nullptr;
  PyObject* text = version ? PyObject_Str(version) : nullptr;
  const char* found = text ? PyUnicode_AsUTF8(text) : nullptr;
  PyObject* made = nullptr;
  if (found) {
    if (std::string(found) != DSV_TORCH || std::string(Py_GetVersion()).rfind(python, 0) != 0)
      PyErr_Format(PyExc_ImportError, "_marshal.so was built for torch %s and Python %s*, this is torch %s and Python %s: build it again",
                   DSV_TORCH, python.c_str(), found, Py_GetVersion());
    else
      made = PyModule_Create(&module);
  }
  Py_XDECREF(text);
  Py_XDECREF(version);
  Py_XDECREF(torch);
  return made;
}
