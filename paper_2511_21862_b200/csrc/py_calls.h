// What the functions of the CPython module `_spec_calls` share: checks of tensors, addresses, numbers and streams.
#pragma once
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <stdexcept>
#include <string>

#include "../../include/ooco_batch.h"

namespace {

struct Refused {  // a Python exception is set
};

[[noreturn]] void refuse(const std::string& text) {
  PyErr_SetString(PyExc_ValueError, text.c_str());
  throw Refused{};
}

std::string list(at::IntArrayRef v) {
  std::string s = "[";
  for (size_t i = 0; i < v.size(); ++i) s += (i ? ", " : "") + std::to_string(v[i]);
  return s + "]";
}
std::string describe(const at::Tensor& t) {
  return std::string(c10::toString(t.scalar_type())) + " " + list(t.sizes()) + " with strides " + list(t.strides()) + " on " +
         t.device().str();
}

const at::Tensor& tensor(PyObject* o, const char* what) {
  if (!THPVariable_Check(o)) refuse(std::string(what) + ": expected a tensor");
  return THPVariable_Unpack(o);
}

// Device of the call: that of its first tensor.
int device_of(const at::Tensor& t, const char* what) {
  if (!t.is_cuda()) refuse(std::string(what) + ": expected a CUDA tensor, got " + describe(t));
  return t.get_device();
}

// Address of a contiguous tensor on device `dev`; `sizes` (where given) is its shape, `least` its fewest elements.
void* address(PyObject* o, int dev, at::ScalarType type, const char* what, std::initializer_list<int64_t> sizes = {},
              int64_t least = 0) {
  const at::Tensor& t = tensor(o, what);
  bool ok = t.is_cuda() && t.get_device() == dev && t.scalar_type() == type && t.is_contiguous() && t.numel() >= least;
  if (sizes.size()) ok = ok && t.sizes() == at::IntArrayRef(sizes.begin(), sizes.size());
  if (!ok) {
    std::string s = std::string(what) + ": expected a contiguous " + c10::toString(type) + " tensor";
    if (sizes.size()) s += " of shape " + list(at::IntArrayRef(sizes.begin(), sizes.size()));
    if (least) s += " of at least " + std::to_string(least) + " elements";
    refuse(s + " on cuda:" + std::to_string(dev) + ", got " + describe(t));
  }
  return t.data_ptr();
}
void* optional(PyObject* o, int dev, at::ScalarType type, const char* what, std::initializer_list<int64_t> sizes = {},
               int64_t least = 0) {
  return o == Py_None ? nullptr : address(o, dev, type, what, sizes, least);
}

int64_t integer(PyObject* o) {
  const int64_t v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw Refused{};
  return v;
}
int32_t integer32(PyObject* o, const char* what) {
  const int64_t v = integer(o);
  if (v < INT32_MIN || v > INT32_MAX) refuse(std::string(what) + ": out of range");
  return (int32_t)v;
}
int32_t count32(int64_t n, const char* what) {
  if (n > INT32_MAX) refuse(std::string(what) + ": too many elements");
  return (int32_t)n;
}
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw Refused{};
  return (float)v;
}

template <typename F>
F entry(PyObject* o) {
  return reinterpret_cast<F>((uintptr_t)integer(o));
}
const ooco_shape_t& shape_at(PyObject* o) { return *reinterpret_cast<const ooco_shape_t*>((uintptr_t)integer(o)); }

// The stream's handle: the given torch stream's, or the current one of `dev`.
void* stream_of(PyObject* o, int dev) {
  if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)dev).stream();
  PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
  if (!h) throw Refused{};
  void* p = PyLong_AsVoidPtr(h);
  Py_DECREF(h);
  if (!p && PyErr_Occurred()) throw Refused{};
  return p;
}

// The caches must hold the pool that the shape describes.
int64_t pool_elements(const ooco_shape_t& s) {
  return (s.num_blocks - 1) * s.kv_block_stride + (s.num_kv_heads - 1) * s.kv_head_stride +
         (s.block_size - 1) * s.kv_token_stride + s.head_dim;
}

struct Rows {
  void* p;
  int64_t stride;
};
// bf16 rows [tokens, heads, dim], dense inside a row.
Rows rows(PyObject* o, int dev, int64_t tokens, int64_t heads, int64_t dim, const char* what) {
  const at::Tensor& t = tensor(o, what);
  if (!(t.is_cuda() && t.get_device() == dev && t.scalar_type() == at::kBFloat16 && t.dim() == 3 && t.size(0) == tokens &&
        t.size(1) == heads && t.size(2) == dim && t.stride(2) == 1 && (heads == 1 || t.stride(1) == dim))) {
    refuse(std::string(what) + ": expected BFloat16 " + list({tokens, heads, dim}) + " with dense rows on cuda:" +
           std::to_string(dev) + ", got " + describe(t));
  }
  const int64_t row = heads * dim;
  return {t.data_ptr(), tokens > 1 ? t.stride(0) : (t.stride(0) > row ? t.stride(0) / 8 * 8 : row)};  // (one row has none)
}

template <typename Body>
PyObject* guarded(const char* name, Py_ssize_t given, Py_ssize_t wanted, Body body) {
  if (given != wanted) {
    PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, got %zd", name, wanted, given);
    return nullptr;
  }
  try {
    return PyLong_FromLong(body());
  } catch (const Refused&) {
  } catch (const std::exception& e) {
    if (!PyErr_Occurred()) PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

constexpr at::ScalarType kI32 = at::kInt, kU8 = at::kByte, kBf = at::kBFloat16, kF32 = at::kFloat;

}  // namespace

// Defined in py_batch.cpp, listed in the module of py_spec.cpp.
#define OOCO_CALL(name) PyObject* name(PyObject*, PyObject* const* a, Py_ssize_t n)
OOCO_CALL(fork_pages);
OOCO_CALL(release_pages);
OOCO_CALL(norm_rope_kv_append);
OOCO_CALL(chunk_attention);
OOCO_CALL(shape_logits);
