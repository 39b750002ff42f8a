// Python extension module _tensors: the host side of calls over many tensors. A model has hundreds of them, and
// reading each one's type, device, layout, shape and address through Python takes a third of a microsecond, which for
// adapters is longer than the GPU works (224 gradients: norm 73 us of host for 15 of kernels). Here it is a loop over
// the list.
//
// Nothing is computed and nothing is kept; tensors that need more than reading (another type or device, strides,
// None, a subclass that is not memory) are left to the caller, who takes them one by one.
#include <torch/csrc/autograd/python_variable.h>

#include <ATen/core/Tensor.h>
#include <c10/hip/HIPStream.h>
#include <torch/version.h>

#include <cstdint>
#include <cstring>

namespace {

// Whether all of a contiguous tensor lies within its storage, which may have been resized (to nothing, for offloading).
bool fits_storage(const at::Tensor& t) {
  return t.numel() == 0 ||
         (t.storage_offset() + t.numel()) * static_cast<int64_t>(t.element_size()) <= static_cast<int64_t>(t.storage().nbytes());
}

// The tensor behind an entry of a list, if it is plain memory of the device (index, or -1 for the host): strided,
// contiguous, bf16 or fp32. dtype: lce_dtype_t.
const at::Tensor* plain(PyObject* o, int64_t device, int32_t* dtype) {
  if (!THPVariable_Check(o)) return nullptr;
  const at::Tensor& t = THPVariable_Unpack(o);
  if (!t.defined() || t.layout() != at::kStrided || t.unsafeGetTensorImpl()->is_python_dispatch()) return nullptr;
  if (t.scalar_type() == at::kBFloat16) *dtype = 0;
  else if (t.scalar_type() == at::kFloat) *dtype = 1;
  else return nullptr;
  if (device < 0 ? !t.is_cpu() : !t.is_cuda() || t.get_device() != device) return nullptr;
  if (!t.has_storage() || !t.is_contiguous() || t.is_neg() || !fits_storage(t)) return nullptr;
  return &t;
}

bool has_shape(const at::Tensor& t, PyObject* shape) {
  if (!PyTuple_Check(shape) || PyTuple_GET_SIZE(shape) != t.dim()) return false;
  for (int64_t k = 0; k < t.dim(); ++k) {
    const long long n = PyLong_AsLongLong(PyTuple_GET_ITEM(shape, k));
    if (n != t.size(k)) {
      PyErr_Clear();       // (an entry that is no number is no size either)
      return false;
    }
  }
  return true;
}

// describe(tensors, shapes, device, table, row_bytes, o_data, o_n, o_dtype) -> bool Writes each tensor's address
// (uint64 at o_data of its row of the table), element count (int64 at o_n, unless o_n < 0) and type (int32 at
// o_dtype). shapes: None, or the shape (a tuple) that each must have. False, with the table half written, where some
// tensor is not plain memory of the device or not of its shape.
PyObject* describe(PyObject*, PyObject* args) {
  PyObject *list, *shapes;
  Py_buffer table;
  long long device;
  Py_ssize_t row, o_data, o_n, o_dtype;
  if (!PyArg_ParseTuple(args, "O!OLw*nnnn", &PyList_Type, &list, &shapes, &device, &table, &row, &o_data, &o_n, &o_dtype))
    return nullptr;
  const Py_ssize_t n = PyList_GET_SIZE(list);
  const auto fits = [row](Py_ssize_t at, Py_ssize_t size) { return at >= 0 && at + size <= row; };
  bool ok = true;
  if (row <= 0 || n > table.len / row || !fits(o_data, 8) || (o_n >= 0 && !fits(o_n, 8)) || !fits(o_dtype, 4) ||
      (shapes != Py_None && (!PyList_Check(shapes) || PyList_GET_SIZE(shapes) != n))) {
    PyBuffer_Release(&table);
    PyErr_SetString(PyExc_ValueError, "table, offsets and lists do not fit together");
    return nullptr;
  }
  try {
    char* to = static_cast<char*>(table.buf);
    for (Py_ssize_t i = 0; ok && i < n; ++i, to += row) {
      int32_t dtype;
      const at::Tensor* t = plain(PyList_GET_ITEM(list, i), device, &dtype);
      ok = t != nullptr;
      if (ok && shapes != Py_None) ok = has_shape(*t, PyList_GET_ITEM(shapes, i));
      if (!ok) break;
      const uint64_t address = reinterpret_cast<uint64_t>(t->const_data_ptr());
      const int64_t count = t->numel();
      std::memcpy(to + o_data, &address, 8);
      if (o_n >= 0) std::memcpy(to + o_n, &count, 8);
      std::memcpy(to + o_dtype, &dtype, 4);
    }
  } catch (const std::exception&) {
    ok = false;      // a tensor without memory of its own: the caller's affair
  }
  PyBuffer_Release(&table);
  return PyBool_FromLong(ok);
}

// Whether t is `count` elements of a type (bf16 0, fp32 1, bytes 2) one after the other, all within its storage.
bool lies_whole(const at::Tensor& t, int64_t count, int32_t dtype) {
  if (!t.defined() || t.layout() != at::kStrided || t.scalar_type() != (dtype == 2 ? at::kByte : dtype == 1 ? at::kFloat : at::kBFloat16))
    return false;
  return t.has_storage() && t.is_contiguous() && !t.is_neg() && t.numel() == count && fits_storage(t);
}

// stand_at(tensors, table, row_bytes, o_data, o_n = -1, o_dtype = -1) -> bool: whether each tensor still has the
// address in its row and, with o_n and o_dtype, is still as many elements of that type without gaps.
PyObject* stand_at(PyObject*, PyObject* args) {
  PyObject* list;
  Py_buffer table;
  Py_ssize_t row, o_data, o_n = -1, o_dtype = -1;
  if (!PyArg_ParseTuple(args, "O!y*nn|nn", &PyList_Type, &list, &table, &row, &o_data, &o_n, &o_dtype)) return nullptr;
  const Py_ssize_t n = PyList_GET_SIZE(list);
  bool ok = row > 0 && n <= table.len / row && o_data >= 0 && o_data + 8 <= row && o_n + 8 <= row && o_dtype + 4 <= row &&
            (o_n < 0) == (o_dtype < 0);
  try {
    const char* at = static_cast<const char*>(table.buf);
    for (Py_ssize_t i = 0; ok && i < n; ++i, at += row) {
      PyObject* o = PyList_GET_ITEM(list, i);
      uint64_t address;
      std::memcpy(&address, at + o_data, 8);
      ok = THPVariable_Check(o);
      if (ok && o_n >= 0) {
        int64_t count;
        int32_t dtype;
        std::memcpy(&count, at + o_n, 8);
        std::memcpy(&dtype, at + o_dtype, 4);
        ok = lies_whole(THPVariable_Unpack(o), count, dtype);
      }
      ok = ok && reinterpret_cast<uint64_t>(THPVariable_Unpack(o).const_data_ptr()) == address;
    }
  } catch (const std::exception&) {
    ok = false;
  }
  PyBuffer_Release(&table);
  return PyBool_FromLong(ok);
}

// changed(tensors): each counts as changed in place for autograd, as after an optimizer's step.
PyObject* changed(PyObject*, PyObject* list) {
  if (!PyList_Check(list)) {
    PyErr_SetString(PyExc_TypeError, "a list of tensors is wanted");
    return nullptr;
  }
  try {
    for (Py_ssize_t i = 0; i < PyList_GET_SIZE(list); ++i) {
      PyObject* o = PyList_GET_ITEM(list, i);
      if (!THPVariable_Check(o)) continue;
      const at::Tensor& t = THPVariable_Unpack(o);
      if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    }
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
  Py_RETURN_NONE;
}

// current_stream(device) -> int: the hipStream_t that torch works on there (0: the default stream). Through torch's
// Stream object this takes 2 us, a sixth of a small call.
PyObject* current_stream(PyObject*, PyObject* device) {
  const long index = PyLong_AsLong(device);
  if (index == -1 && PyErr_Occurred()) return nullptr;
  try {
    return PyLong_FromVoidPtr(c10::hip::getCurrentHIPStream(static_cast<c10::DeviceIndex>(index)).stream());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

// negative(tensor), dual(tensor) -> bool: whether its memory holds its values with the other sign; whether it has a
// forward-mode tangent. (Through Python 0.3 and 0.8 us of a call that takes 11.)
PyObject* negative(PyObject*, PyObject* o) { return PyBool_FromLong(THPVariable_Check(o) && THPVariable_Unpack(o).is_neg()); }

PyObject* dual(PyObject*, PyObject* o) {
  try {
    return PyBool_FromLong(THPVariable_Check(o) && THPVariable_Unpack(o)._fw_grad(0).defined());
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
    return nullptr;
  }
}

PyMethodDef methods[] = {{"describe", describe, METH_VARARGS, nullptr},
                         {"stand_at", stand_at, METH_VARARGS, nullptr},
                         {"changed", changed, METH_O, nullptr},
                         {"current_stream", current_stream, METH_O, nullptr},
                         {"negative", negative, METH_O, nullptr},
                         {"dual", dual, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// torch_version: whose tensors' layout the module was compiled for
PyMODINIT_FUNC PyInit__tensors() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "torch_version", TORCH_VERSION) != 0) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
