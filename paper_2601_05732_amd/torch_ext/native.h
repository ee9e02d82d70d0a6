// What the host code of the Python extension shares: statuses as exceptions, the current stream, allocation.
#pragma once
#include <torch/extension.h>

#include <c10/hip/HIPStream.h>

#include "../../include/mhcl.h"

namespace native {

using at::Tensor;

// Raises what binding.py raises for the same status. As a Python exception from here on: a backward runs in autograd's
// threads, which carry those over to the caller as they are and make a RuntimeError of all others.
[[noreturn]] inline void raise(int status, const char *where) {
  py::gil_scoped_acquire gil;
  const py::object type = py::module_::import("paper_2601_05732_amd.binding").attr("MhclError"), error = type(status, where);
  PyErr_SetObject(type.ptr(), error.ptr());
  python_error e;
  e.persist();
  throw e;
}
inline void check(int status, const char *where) {
  if (status != MHCL_OK) raise(status, where);
}

inline void *stream() { return c10::hip::getCurrentHIPStream().stream(); }

// an empty tensor has no storage: NULL
template <typename T = void>
T *ptr(const Tensor &t) {
  return t.numel() == 0 ? nullptr : static_cast<T *>(t.data_ptr());
}
inline Tensor floats(const Tensor &like, at::IntArrayRef shape) { return at::empty(shape, like.options().dtype(at::kFloat)); }

// as layer.empty_stream: contiguous, first byte `phase` bytes past a 1 KiB boundary
inline Tensor empty_stream(const Tensor &like, at::IntArrayRef shape, int64_t phase) {
  int64_t numel = 1;
  std::vector<int64_t> strides(shape.size());
  for (size_t i = shape.size(); i-- > 0;) {
    strides[i] = numel;
    numel *= shape[i];
  }
  const int64_t size = like.element_size();
  const Tensor buf = at::empty({numel + 1024 / size}, like.options());
  const uintptr_t lead = (static_cast<uintptr_t>(phase) - reinterpret_cast<uintptr_t>(buf.data_ptr())) & 1023u;
  return buf.as_strided(shape, strides, static_cast<int64_t>(lead) / size);
}

void bind_ends(py::module &m);   // ends.cpp

}  // namespace native
