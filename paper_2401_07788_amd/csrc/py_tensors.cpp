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

namespace {

// Writes the address of each tensor of `list` (a Python list or tuple) to
// column[k * stride].  All must be dense, contiguous, of one dtype, on GPU
// `device` and of sizes[k] elements, n in number.  Returns their dtype as the
// library numbers it (0 binary32, 1 bfloat16, 2 binary16), or -1 if anything
// is otherwise.
int addresses(PyObject* list, int64_t n, const int64_t* sizes, int device, uint64_t* column, int64_t stride) {
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
}

}  // namespace

// Whether the tensors of `list` (n of them) may be handed to a kernel as the
// optimizer's state: each a vector, dense, contiguous, on GPU `device`, of sizes[k]
// elements and of dtype types[k] (0 binary32, 3 unsigned and 4 signed 8-bit
// integers).  Their addresses go to out[0 .. n).
extern "C" __attribute__((visibility("default"))) int tc_py_state(PyObject* list, int64_t n, const int64_t* sizes,
                                                                   const int8_t* types, int device, uint64_t* out) {
  try {
    if (!PyList_Check(list) || PyList_GET_SIZE(list) != n) return 0;
    for (int64_t k = 0; k < n; ++k) {
      PyObject* const item = PyList_GET_ITEM(list, k);
      if (!THPVariable_Check(item)) return 0;
      const at::Tensor& t = THPVariable_Unpack(item);
      if (!t.defined() || t.layout() != c10::kStrided || !t.is_cuda() || t.get_device() != device) return 0;
      const c10::ScalarType want = types[k] == 0 ? c10::ScalarType::Float : types[k] == 3 ? c10::ScalarType::Byte : c10::ScalarType::Char;
      if (t.scalar_type() != want || t.dim() != 1 || t.numel() != sizes[k] || !t.is_contiguous()) return 0;
      out[k] = (uint64_t)(uintptr_t)t.data_ptr();
    }
    return 1;
  } catch (...) {
    return 0;
  }
}

// The same for all tensors of an optimizer's step in one call: its parameters
// and gradients (n of each, of sizes[k] elements; rows of `stride` words, p in
// the first and g in the second) and its state (n_state tensors, as above).
// Returns the dtypes, the parameters' plus 4 times the gradients', or -1 if
// anything is not as it must be (what, the caller finds out).
extern "C" __attribute__((visibility("default"))) int tc_py_step(PyObject* params, PyObject* grads, int64_t n, const int64_t* sizes,
                                                                  uint64_t* table, int64_t stride, PyObject* state, int64_t n_state,
                                                                  const int64_t* lengths, const int8_t* types, uint64_t* out, int device) {
  try {
    const int p = addresses(params, n, sizes, device, table, stride), g = addresses(grads, n, sizes, device, table + 1, stride);
    if (p < 0 || g < 0 || !tc_py_state(state, n_state, lengths, types, device, out)) return -1;
    return p + 4 * g;
  } catch (...) {
    return -1;
  }
}

// After a step: every tensor of `list` was written in place, and autograd is
// told (as an operation of torch's own would), so that a backward pass that
// saved one of them before is refused.
extern "C" __attribute__((visibility("default"))) void tc_py_written(PyObject* list) {
  try {
    if (!PyList_Check(list) && !PyTuple_Check(list)) return;
    for (Py_ssize_t k = 0; k < PySequence_Fast_GET_SIZE(list); ++k) {
      PyObject* const item = PySequence_Fast_GET_ITEM(list, k);
      if (!THPVariable_Check(item)) continue;
      const at::Tensor& t = THPVariable_Unpack(item);
      // (inference tensors have no counter)
      if (t.defined() && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
    }
  } catch (...) {
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
