// Tensors as the C ABI's arguments, for the Python binding's calls of many
// tensors: read through the interpreter, a property takes 30 to 60 ns, the checks
// of an argument 0.5 us and a gradient's entry 0.2 us, which is longer than small
// calls, and the clipping of hundreds of gradients, take on the GPU.
#include <Python.h>

#include <exception>

#include <ATen/ops/empty.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/Exceptions.h>
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
    } catch (...) {
      torch::translate_exception_to_python(std::current_exception());
    }
  }
  Py_XDECREF(ptrs);
  Py_XDECREF(sizes);
  Py_XDECREF(codes);
  return result;
}

// address(tensor, name, dtype, least elements = 0, optional = False): the data
// pointer, None for an optional None.
PyObject* address(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n < 3 || n > 5 || !THPDtype_Check(args[2])) {
    PyErr_SetString(PyExc_TypeError, "address(tensor, name, dtype, least=0, optional=False)");
    return nullptr;
  }
  PyObject* name = args[1];
  if (args[0] == Py_None) {
    if (n > 4 && args[4] == Py_True) Py_RETURN_NONE;
    return PyErr_Format(PyExc_ValueError, "%S is required", name);
  }
  if (!THPVariable_Check(args[0]))
    return PyErr_Format(PyExc_ValueError, "%S must be a CUDA (HIP) tensor", name);
  try {
    const at::Tensor& t = THPVariable_Unpack(args[0]);
    if (!t.is_cuda())
      return PyErr_Format(PyExc_ValueError, "%S must be a CUDA (HIP) tensor", name);
    if (t.scalar_type() != reinterpret_cast<THPDtype*>(args[2])->scalar_type)
      return PyErr_Format(PyExc_TypeError, "%S must be %S, got %S", name, args[2],
                          reinterpret_cast<PyObject*>(torch::getTHPDtype(t.scalar_type())));
    if (!t.is_contiguous())
      return PyErr_Format(PyExc_ValueError, "%S must be contiguous", name);
    if (n > 3) {
      const long long least = PyLong_AsLongLong(args[3]);
      if (least == -1 && PyErr_Occurred()) return nullptr;
      if (t.numel() < least)
        return PyErr_Format(PyExc_ValueError, "%S holds %lld elements, needs %lld", name,
                            (long long)t.numel(), least);
    }
    return PyLong_FromUnsignedLongLong(reinterpret_cast<uint64_t>(t.data_ptr()));
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
}

bool half(const at::Tensor& t) {
  return t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kHalf;
}

// cache(k_cache, v_cache) -> (addresses, type code, strides of a page, a slot and
// a head, pages, page, heads, width), or None if they are not a paged cache's
// halves.
PyObject* cache(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 2) {
    PyErr_SetString(PyExc_TypeError, "cache(k_cache, v_cache)");
    return nullptr;
  }
  if (!THPVariable_Check(args[0]) || !THPVariable_Check(args[1])) Py_RETURN_NONE;
  try {
    const at::Tensor &k = THPVariable_Unpack(args[0]), &v = THPVariable_Unpack(args[1]);
    if (!k.is_cuda() || !v.is_cuda() || k.dim() != 4 || !half(k) ||
        v.scalar_type() != k.scalar_type() || v.sizes() != k.sizes() ||
        v.strides() != k.strides() || k.stride(3) != 1)
      Py_RETURN_NONE;
    return Py_BuildValue("KKiLLLLLLL", (unsigned long long)k.data_ptr(),
                         (unsigned long long)v.data_ptr(), (int)dtype_code(k.scalar_type()),
                         (long long)k.stride(0), (long long)k.stride(1), (long long)k.stride(2),
                         (long long)k.size(0), (long long)k.size(1), (long long)k.size(2),
                         (long long)k.size(3));
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
}

// rows(tensor, type code, heads or 0, width) -> (address, strides of a row and a
// head, rows, heads), or None if it is not [rows][heads][width] of that type.
PyObject* rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
  if (n != 4) {
    PyErr_SetString(PyExc_TypeError, "rows(tensor, type code, heads, width)");
    return nullptr;
  }
  if (!THPVariable_Check(args[0])) Py_RETURN_NONE;
  const long code = PyLong_AsLong(args[1]), heads = PyLong_AsLong(args[2]),
             width = PyLong_AsLong(args[3]);
  if ((code == -1 || heads == -1 || width == -1) && PyErr_Occurred()) return nullptr;
  try {
    const at::Tensor& t = THPVariable_Unpack(args[0]);
    if (!t.is_cuda() || t.dim() != 3 || dtype_code(t.scalar_type()) != code ||
        t.size(2) != width || t.stride(2) != 1 || (heads != 0 && t.size(1) != heads))
      Py_RETURN_NONE;
    return Py_BuildValue("KLLLL", (unsigned long long)t.data_ptr(), (long long)t.stride(0),
                         (long long)t.stride(1), (long long)t.size(0), (long long)t.size(1));
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
}

// parts(device, dtype, shape, dtype, shape, ...): uninitialised tensors, each
// 256-byte aligned, of one allocation on the current stream (a shape is a tuple,
// or an int for one dimension).  An allocation takes 1.3 us through the
// interpreter and a part of one cut there 0.55; here a part takes 0.15.
PyObject* parts(PyObject*, PyObject* const* args, Py_ssize_t n) {
  constexpr Py_ssize_t kMost = 16, kDims = 4;
  if (n < 3 || n % 2 == 0 || n / 2 > kMost || !PyLong_Check(args[0])) {
    PyErr_SetString(PyExc_TypeError, "parts(device, dtype, shape, ...)");
    return nullptr;
  }
  const Py_ssize_t count = n / 2;
  at::ScalarType type[kMost];
  int64_t shape[kMost][kDims], start[kMost], bytes = 0;
  size_t dims[kMost];
  for (Py_ssize_t i = 0; i < count; ++i) {
    PyObject *dtype = args[1 + 2 * i], *size = args[2 + 2 * i];
    const bool tuple = PyTuple_Check(size);
    if (!THPDtype_Check(dtype) || (tuple && PyTuple_GET_SIZE(size) > kDims)) {
      PyErr_SetString(PyExc_TypeError, "parts(device, dtype, shape, ...)");
      return nullptr;
    }
    type[i] = reinterpret_cast<THPDtype*>(dtype)->scalar_type;
    dims[i] = tuple ? PyTuple_GET_SIZE(size) : 1;
    int64_t room = (int64_t)c10::elementSize(type[i]);
    for (size_t d = 0; d < dims[i]; ++d) {
      const int64_t v = PyLong_AsLongLong(tuple ? PyTuple_GET_ITEM(size, d) : size);
      if (v == -1 && PyErr_Occurred()) return nullptr;
      if (v < 0 || __builtin_mul_overflow(room, v, &room) || room > (int64_t)1 << 48) {
        PyErr_SetString(PyExc_ValueError, "a size is negative or too large");
        return nullptr;
      }
      shape[i][d] = v;
    }
    start[i] = bytes;
    bytes += (room + 255) / 256 * 256;
  }
  const long device = PyLong_AsLong(args[0]);
  if (device < 0) {
    if (!PyErr_Occurred())
      PyErr_SetString(PyExc_ValueError, "the arguments must be CUDA (HIP) tensors");
    return nullptr;
  }
  PyObject* result = PyTuple_New(count);
  if (result == nullptr) return nullptr;
  try {
    const at::Tensor all = at::empty(
        {bytes}, at::TensorOptions().dtype(at::kByte).device(at::kCUDA, (c10::DeviceIndex)device));
    for (Py_ssize_t i = 0; i < count; ++i) {
      at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(
          c10::Storage(all.storage()), all.key_set(), c10::scalarTypeToTypeMeta(type[i]));
      t.unsafeGetTensorImpl()->set_storage_offset(start[i] / (int64_t)c10::elementSize(type[i]));
      t.unsafeGetTensorImpl()->set_sizes_contiguous(c10::IntArrayRef(shape[i], dims[i]));
      PyObject* wrapped = THPVariable_Wrap(std::move(t));
      if (wrapped == nullptr) {
        Py_DECREF(result);
        return nullptr;
      }
      PyTuple_SET_ITEM(result, i, wrapped);
    }
  } catch (...) {
    Py_DECREF(result);
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
  return result;
}

// written(tensor, list of tensors or None, ...): counts a write that torch has not
// seen, so that autograd notices if it had saved the old values.
PyObject* written(PyObject*, PyObject* const* args, Py_ssize_t n) {
  auto count = [](PyObject* x) {
    if (!THPVariable_Check(x)) return;
    const at::Tensor& t = THPVariable_Unpack(x);
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();   // those have no count
  };
  try {
    for (Py_ssize_t i = 0; i < n; ++i) {
      if (PyList_Check(args[i])) {
        for (Py_ssize_t k = 0; k < PyList_GET_SIZE(args[i]); ++k) count(PyList_GET_ITEM(args[i], k));
      } else {
        count(args[i]);
      }
    }
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
  Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"grad_table", grad_table, METH_VARARGS,
     "grad_table(list, name): addresses, sizes and type codes of GPU tensors, as bytes."},
    {"address", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(address)),
     METH_FASTCALL,
     "address(tensor, name, dtype, least=0, optional=False): a checked tensor's data pointer."},
    {"cache", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(cache)),
     METH_FASTCALL, "cache(k_cache, v_cache): addresses and layout, None if it is no cache."},
    {"rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(rows)),
     METH_FASTCALL, "rows(tensor, type code, heads, width): address and layout, or None."},
    {"parts", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(parts)),
     METH_FASTCALL,
     "parts(device, dtype, shape, ...): uninitialised GPU tensors of one allocation."},
    {"written", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(written)),
     METH_FASTCALL, "written(tensor, list or None, ...): counts a write to each tensor."},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, kMethods,
                       nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors(void) { return PyModule_Create(&kModule); }
