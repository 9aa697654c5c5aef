// The checks that binding.py makes of a call's tensors, in C++: what a tensor method
// costs in Python (its argument parsing, 50 to 100 ns, six for a tensor) adds up to as
// much as the kernel's launch.  Nothing is decided here: where a tensor is not as asked
// the answer is None, and binding.py finds out why.
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

// A tensor or parameter (and no other subclass) of this type on this GPU.
const at::Tensor* plain(PyObject* o, at::ScalarType type, long device) {
  if (!THPVariable_CheckExact(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (t.scalar_type() != type || t.layout() != at::kStrided || !t.is_cuda() || t.get_device() != device) return nullptr;
  return &t;
}

PyObject* address(const at::Tensor& t) { return PyLong_FromUnsignedLongLong(reinterpret_cast<uintptr_t>(t.data_ptr())); }

// address(tensor, dtype, ndim or -1, device): the address of a contiguous tensor, or None.
PyObject* get_address(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 4 || !THPDtype_Check(args[1])) {
    PyErr_SetString(PyExc_TypeError, "address(tensor, dtype, ndim, device)");
    return nullptr;
  }
  const long ndim = PyLong_AsLong(args[2]), device = PyLong_AsLong(args[3]);
  if (PyErr_Occurred()) return nullptr;
  try {
    const at::Tensor* t = plain(args[0], reinterpret_cast<THPDtype*>(args[1])->scalar_type, device);
    if (t == nullptr || (ndim >= 0 && t->dim() != ndim) || !t->is_contiguous()) Py_RETURN_NONE;
    return address(*t);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// rows(tensor, device): (address, stride, tokens, heads, head_dim) of a bf16 tensor
// [tokens][heads][head_dim] whose tokens' values are contiguous, or None.
PyObject* get_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "rows(tensor, device)");
    return nullptr;
  }
  const long device = PyLong_AsLong(args[1]);
  if (PyErr_Occurred()) return nullptr;
  try {
    const at::Tensor* t = plain(args[0], at::kBFloat16, device);
    if (t == nullptr || t->dim() != 3) Py_RETURN_NONE;
    const int64_t tokens = t->size(0), heads = t->size(1), d = t->size(2);
    if (t->stride(2) != 1 || (heads > 1 && t->stride(1) != d)) Py_RETURN_NONE;
    return Py_BuildValue("(KLLLL)", (unsigned long long)reinterpret_cast<uintptr_t>(t->data_ptr()),
                         (long long)(tokens > 1 ? t->stride(0) : heads * d), (long long)tokens, (long long)heads,
                         (long long)d);
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyMethodDef methods[] = {
    {"address", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(get_address)), METH_FASTCALL, nullptr},
    {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(get_rows)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
