// A Python module of two functions that the binding asks of every tensor of a call, and torch_version, the
// version it was built against (a tensor's layout is that version's):
//   address(tensor, dtype, device): the device address of a contiguous tensor of this dtype on GPU
//     `device`;
//   rows_address(tensor, dtype, device, rows, heads, dim): (address, row stride in elements) of such a
//     tensor [rows][heads][dim] whose heads are contiguous and whose rows may lie apart.
// Either is None when the tensor is anything else (the caller then finds out what and says so). Read from
// Python, these properties take 0.27 us a tensor, most of a small call's host time; here 0.06 us.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

// The tensor if it is one of this dtype, strided, on this GPU.
const at::Tensor* tensor_on(PyObject* const* args) {
  if (!THPVariable_Check(args[0]) || !THPDtype_Check(args[1])) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(args[0]);
  const c10::Device d = t.device();
  if (t.layout() != c10::kStrided || !d.is_cuda() || d.index() != PyLong_AsLong(args[2]) ||
      t.scalar_type() != reinterpret_cast<THPDtype*>(args[1])->scalar_type)
    return nullptr;
  return &t;
}

PyObject* address(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 3 || !PyLong_Check(args[2])) {
    PyErr_SetString(PyExc_TypeError, "address(tensor, dtype, device)");
    return nullptr;
  }
  try {
    const at::Tensor* t = tensor_on(args);
    if (t == nullptr || !t->is_contiguous()) Py_RETURN_NONE;
    return PyLong_FromVoidPtr(t->data_ptr());
  } catch (...) {  // (a tensor without storage, say)
    Py_RETURN_NONE;
  }
}

PyObject* rows_address(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 6 || !PyLong_Check(args[2]) || !PyLong_Check(args[3]) || !PyLong_Check(args[4]) ||
      !PyLong_Check(args[5])) {
    PyErr_SetString(PyExc_TypeError, "rows_address(tensor, dtype, device, rows, heads, dim)");
    return nullptr;
  }
  const int64_t rows = PyLong_AsLongLong(args[3]), heads = PyLong_AsLongLong(args[4]),
                dim = PyLong_AsLongLong(args[5]);
  if (PyErr_Occurred()) return nullptr;
  try {
    const at::Tensor* t = tensor_on(args);
    if (t == nullptr || t->dim() != 3 || t->size(0) != rows || t->size(1) != heads ||
        t->size(2) != dim || t->stride(2) != 1 || (heads > 1 && t->stride(1) != dim))
      Py_RETURN_NONE;
    PyObject* out = PyTuple_New(2);
    if (out == nullptr) return nullptr;
    PyTuple_SET_ITEM(out, 0, PyLong_FromVoidPtr(t->data_ptr()));
    PyTuple_SET_ITEM(out, 1, PyLong_FromLongLong(rows > 1 ? t->stride(0) : heads * dim));
    return out;
  } catch (...) {
    Py_RETURN_NONE;
  }
}

template <typename F>
PyCFunction fastcall(F f) {
  return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f));
}
PyMethodDef methods[] = {{"address", fastcall(address), METH_FASTCALL, "see the file's head"},
                         {"rows_address", fastcall(rows_address), METH_FASTCALL, "see the file's head"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensor_address", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensor_address(void) {
  PyObject* m = PyModule_Create(&module);
  if (m != nullptr && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION_BUILT) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
