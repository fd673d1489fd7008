// py_tensors.cpp -- the binding's look at a list of tensors (libtc_py.so).
//
// A step of the optimizer gets a list of some hundred tensors, whose
// addresses, sizes, types, devices and strides have to be looked at each time.
// Asked of Python one property at a time that takes 0.1 us each, 75 us for 218
// parameters; here the whole list takes 3 us.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>
#include <memory>
#include <vector>

// Writes the address of each tensor of `list` (a Python list or tuple) to
// column[k * stride].  All must be dense, contiguous, of one dtype, on GPU
// `device` and of sizes[k] elements, n in number.  Returns their dtype as the
// library numbers it (0 binary32, 1 bfloat16, 2 binary16), or -1 if anything
// is otherwise (which of them, the caller finds out).
extern "C" __attribute__((visibility("default"))) int tc_py_addresses(PyObject* list, int64_t n, const int64_t* sizes,
                                                                       int device, uint64_t* column, int64_t stride) {
  try {
    if (!PyList_Check(list) && !PyTuple_Check(list)) return -1;
    if (PySequence_Fast_GET_SIZE(list) != n || n == 0) return -1;
    PyObject** const items = PySequence_Fast_ITEMS(list);
    c10::ScalarType dtype = c10::ScalarType::Undefined;
    for (int64_t k = 0; k < n; ++k) {
      if (!THPVariable_Check(items[k])) return -1;
      const at::Tensor& t = THPVariable_Unpack(items[k]);
      if (!t.defined() || t.layout() != c10::kStrided || !t.is_cuda() || t.get_device() != device) return -1;
      if (k == 0) dtype = t.scalar_type();
      if (t.scalar_type() != dtype || t.numel() != sizes[k] || !t.is_contiguous()) return -1;
      column[k * stride] = (uint64_t)(uintptr_t)t.data_ptr();
    }
    return dtype == c10::ScalarType::Float ? 0 : dtype == c10::ScalarType::BFloat16 ? 1 : dtype == c10::ScalarType::Half ? 2 : -1;
  } catch (...) {
    return -1;
  }
}

// The table of a list that is looked at for the first time: each tensor's
// address to table[k * stride + at] and its elements to table[k * stride + n_at]
// and, unless NULL, to sizes[k]; its first position in the moments (multiples
// of 256, one tensor after the other) to table[k * stride + pos_at].  All must be dense, contiguous, of one dtype
// and on one device.  Returns an object that keeps their memory, or None if
// anything is otherwise.
extern "C" __attribute__((visibility("default"))) PyObject* tc_py_table(PyObject* list, uint64_t* table, int64_t stride,
                                                                         int64_t at, int64_t n_at, int64_t pos_at, int64_t* sizes) {
  using Held = std::vector<c10::Storage>;
  try {
    if (!PyList_Check(list)) Py_RETURN_NONE;
    const int64_t n = PyList_GET_SIZE(list);
    auto held = std::make_unique<Held>();
    held->reserve(n);
    c10::ScalarType dtype = c10::ScalarType::Undefined;
    c10::Device device = c10::kCPU;
    uint64_t pos = 0;
    for (int64_t k = 0; k < n; ++k) {
      PyObject* const item = PyList_GET_ITEM(list, k);
      if (!THPVariable_Check(item)) Py_RETURN_NONE;
      const at::Tensor& t = THPVariable_Unpack(item);
      if (!t.defined() || t.layout() != c10::kStrided || !t.has_storage() || !t.is_contiguous()) Py_RETURN_NONE;
      if (k == 0) {
        dtype = t.scalar_type();
        device = t.device();
      }
      if (t.scalar_type() != dtype || t.device() != device) Py_RETURN_NONE;
      table[k * stride + at] = (uint64_t)(uintptr_t)t.data_ptr();
      table[k * stride + n_at] = (uint64_t)t.numel();
      if (sizes) sizes[k] = t.numel();
      table[k * stride + pos_at] = pos;
      pos += ((uint64_t)t.numel() + 255u) / 256u * 256u;
      held->push_back(t.storage());
    }
    PyObject* const capsule = PyCapsule_New(held.get(), nullptr, [](PyObject* c) { delete static_cast<Held*>(PyCapsule_GetPointer(c, nullptr)); });
    if (capsule) held.release();
    return capsule;
  } catch (...) {
    Py_RETURN_NONE;
  }
}
