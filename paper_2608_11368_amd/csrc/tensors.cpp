// A list of tensors as the C ABI's host arrays, for the Python binding: a model
// has hundreds of gradients, and reading five properties of each through the
// interpreter (about 0.2 us a tensor) took longer than clipping them.
#include <Python.h>

#include <exception>

#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/autograd/python_variable.h>

namespace {

// PAIR_F32, PAIR_BF16, PAIR_F16 of pair.h; -1 for other types.
int32_t dtype_code(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return 0;
    case at::kBFloat16: return 1;
    case at::kHalf: return 2;
    default: return -1;
  }
}

PyObject* refuse(PyObject* type, const char* format, const char* name) {
  PyErr_Format(type, format, name);
  return nullptr;
}

// grad_table(list, name) -> (addresses, sizes, type codes), each bytes.
PyObject* grad_table(PyObject*, PyObject* args) {
  PyObject* list;
  const char* name;
  if (!PyArg_ParseTuple(args, "O!s", &PyList_Type, &list, &name)) return nullptr;
  const Py_ssize_t n = PyList_GET_SIZE(list);
  PyObject* ptrs = PyBytes_FromStringAndSize(nullptr, n * 8);
  PyObject* sizes = PyBytes_FromStringAndSize(nullptr, n * 8);
  PyObject* codes = PyBytes_FromStringAndSize(nullptr, n * 4);
  PyObject* result = nullptr;
  if (ptrs != nullptr && sizes != nullptr && codes != nullptr) {
    auto* ptr = reinterpret_cast<uint64_t*>(PyBytes_AS_STRING(ptrs));
    auto* size = reinterpret_cast<int64_t*>(PyBytes_AS_STRING(sizes));
    auto* code = reinterpret_cast<int32_t*>(PyBytes_AS_STRING(codes));
    try {
      bool tensors = true, placed = true;
      for (Py_ssize_t i = 0; tensors && i < n; ++i)
        tensors = THPVariable_Check(PyList_GET_ITEM(list, i));
      at::ScalarType other = at::ScalarType::Undefined;
      int device = -1;
      for (Py_ssize_t i = 0; tensors && i < n; ++i) {
        const at::Tensor& t = THPVariable_Unpack(PyList_GET_ITEM(list, i));
        if (i == 0) device = t.get_device();
        if (!t.is_cuda() || t.get_device() != device || !t.is_contiguous() || t.is_neg()) {
          placed = false;
          break;
        }
        code[i] = dtype_code(t.scalar_type());
        if (code[i] < 0) other = t.scalar_type();
        size[i] = t.numel();
        ptr[i] = reinterpret_cast<uint64_t>(t.data_ptr());
      }
      if (!tensors)
        refuse(PyExc_ValueError, "%s must be tensors", name);
      else if (!placed)
        refuse(PyExc_ValueError, "%s must be contiguous CUDA (HIP) tensors of one device", name);
      else if (other != at::ScalarType::Undefined)
        PyErr_Format(PyExc_TypeError, "%s must be float32, bfloat16 or float16, got %S", name,
                     reinterpret_cast<PyObject*>(torch::getTHPDtype(other)));
      else
        result = PyTuple_Pack(3, ptrs, sizes, codes);
    } catch (const std::exception& e) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
    }
  }
  Py_XDECREF(ptrs);
  Py_XDECREF(sizes);
  Py_XDECREF(codes);
  return result;
}

PyMethodDef kMethods[] = {
    {"grad_table", grad_table, METH_VARARGS,
     "grad_table(list, name): addresses, sizes and type codes of GPU tensors, as bytes."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors(void) { return PyModule_Create(&kModule); }
