// CPython module `_spec_calls`: checks the tensors of a call of ooco_spec.h and passes their addresses on.  A call has
// up to twenty tensors, and checking them from Python takes 8 to 14 us, several times what the GPU works on a small
// step; here it takes about one.  The library's entry points come in as addresses, so that the caller chooses the build.
#include <Python.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <stdexcept>
#include <string>

#include "../../include/ooco_spec.h"

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

PyObject* plan_slots(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded("plan_slots", n, 20, [&] {
    const auto fn = entry<decltype(&ooco_plan_slots)>(a[0]);
    const ooco_shape_t& s = shape_at(a[1]);
    const int dev = device_of(tensor(a[2], "context_lens"), "context_lens");
    const int64_t B = s.batch, num_rows = tensor(a[12], "slot_map").numel(), num_free = tensor(a[6], "free_ids").numel();
    const auto* ctx = (const int32_t*)address(a[2], dev, kI32, "context_lens", {B});
    const auto* add = (const int32_t*)address(a[3], dev, kI32, "new_lens", {B});
    auto* table = (int32_t*)address(a[4], dev, kI32, "block_table", {B, s.max_blocks_per_seq});
    auto* held = (int32_t*)address(a[5], dev, kI32, "blocks_held", {B});
    const auto* ids = (const int32_t*)address(a[6], dev, kI32, "free_ids");
    auto* head = (int32_t*)address(a[7], dev, kI32, "free_head", {1});
    auto* held_out = (int32_t*)optional(a[8], dev, kI32, "blocks_held_out", {B});
    auto* head_out = (int32_t*)optional(a[9], dev, kI32, "free_head_out", {1});
    const int32_t row_len = integer32(a[10], "row_len");
    const auto* parents = (const int32_t*)optional(a[11], dev, kI32, "parents", {}, num_rows);
    auto* slots = (int32_t*)address(a[12], dev, kI32, "slot_map");
    auto* pos = (int32_t*)address(a[13], dev, kI32, "positions", {}, num_rows);
    auto* first = (int32_t*)address(a[14], dev, kI32, "first_token", {B + 1});
    auto* granted = (int32_t*)address(a[15], dev, kI32, "granted_lens", {B});
    auto* total = (int32_t*)address(a[16], dev, kI32, "total_lens", {B});
    void* ws = address(a[17], dev, kU8, "workspace");
    auto* status = (int32_t*)optional(a[18], dev, kI32, "status", {1});
    void* st = stream_of(a[19], dev);
    const c10::cuda::OptionalCUDAGuard guard(at::Device(at::kCUDA, (c10::DeviceIndex)dev));
    return fn(&s, ctx, add, table, held, ids, count32(num_free, "free_ids"), head, held_out, head_out, row_len,
              count32(num_rows, "slot_map"), parents, slots, pos, first, granted, total, ws,
              (size_t)THPVariable_Unpack(a[17]).numel(), status, st);
  });
}

// entry, 8-bit cache, shape, ooco_rope_t, inv_freq, q, k, v, positions, slot_map, q_out, k_cache, v_cache, scales, stream
PyObject* rope_kv_append(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded("rope_kv_append", n, 16, [&] {
    const bool kv8 = a[1] == Py_True;
    const ooco_shape_t& s = shape_at(a[2]);
    ooco_rope_t r = *reinterpret_cast<const ooco_rope_t*>((uintptr_t)integer(a[3])), *const rope = &r;
    const at::Tensor& q_t = tensor(a[5], "q");
    const int dev = device_of(q_t, "q");
    r.inv_freq = (const float*)address(a[4], dev, kF32, "inv_freq", {r.rot_dim / 2});
    const int64_t T = q_t.dim() ? q_t.size(0) : -1;
    const Rows q = rows(a[5], dev, T, s.num_q_heads, s.head_dim, "q"), k = rows(a[6], dev, T, s.num_kv_heads, s.head_dim, "k"),
               v = rows(a[7], dev, T, s.num_kv_heads, s.head_dim, "v");
    const auto* pos = (const int32_t*)address(a[8], dev, kI32, "positions", {T});
    const auto* slots = (const int32_t*)address(a[9], dev, kI32, "slot_map", {T});
    const Rows out = rows(a[10], dev, T, s.num_q_heads, s.head_dim, "q_out");
    const at::ScalarType cell = kv8 ? kU8 : kBf;
    void* kc = address(a[11], dev, cell, "k_cache", {}, pool_elements(s));
    void* vc = address(a[12], dev, cell, "v_cache", {}, pool_elements(s));
    void* st = stream_of(a[15], dev);
    const c10::cuda::OptionalCUDAGuard guard(at::Device(at::kCUDA, (c10::DeviceIndex)dev));
    const int32_t tokens = count32(T, "q");
    if (kv8)
      return entry<decltype(&ooco_rope_kv_append_fp8)>(a[0])(&s, rope, tokens, q.p, q.stride, k.p, k.stride, v.p, v.stride, pos,
                                                             slots, out.p, out.stride, kc, vc, real(a[13]), real(a[14]), st);
    return entry<decltype(&ooco_rope_kv_append)>(a[0])(&s, rope, tokens, q.p, q.stride, k.p, k.stride, v.p, v.stride, pos,
                                                       slots, out.p, out.stride, kc, vc, st);
  });
}

// entry, 8-bit cache, fp32 output, shape, q, k_cache, v_cache, block_table, context_lens, parents, tree_sizes, scale, k_scale,
// v_scale, out, workspace, stream
PyObject* tree_attention(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded("tree_attention", n, 17, [&] {
    const bool kv8 = a[1] == Py_True, f32 = a[2] == Py_True;
    const ooco_shape_t& s = shape_at(a[3]);
    const at::Tensor& q_t = tensor(a[4], "q");
    const int dev = device_of(q_t, "q");
    const int64_t B = s.batch, N = q_t.dim() == 4 ? q_t.size(1) : -1;
    const void* q = address(a[4], dev, kBf, "q", {B, N, s.num_q_heads, s.head_dim});
    const at::ScalarType cell = kv8 ? kU8 : kBf;
    const void* kc = address(a[5], dev, cell, "k_cache", {}, pool_elements(s));
    const void* vc = address(a[6], dev, cell, "v_cache", {}, pool_elements(s));
    const auto* table = (const int32_t*)address(a[7], dev, kI32, "block_table", {B, s.max_blocks_per_seq});
    const auto* ctx = (const int32_t*)address(a[8], dev, kI32, "context_lens", {B});
    const auto* parents = (const int32_t*)address(a[9], dev, kI32, "parents", {B, N});
    const auto* sizes = (const int32_t*)optional(a[10], dev, kI32, "tree_sizes", {B});
    void* out = address(a[14], dev, f32 ? kF32 : kBf, "out", {B, N, s.num_q_heads, s.head_dim});
    void* ws = address(a[15], dev, kU8, "workspace");
    const size_t bytes = (size_t)THPVariable_Unpack(a[15]).numel();
    void* st = stream_of(a[16], dev);
    const c10::cuda::OptionalCUDAGuard guard(at::Device(at::kCUDA, (c10::DeviceIndex)dev));
    const int32_t nodes = count32(N, "q");
    if (kv8)
      return entry<decltype(&ooco_tree_attention_fp8)>(a[0])(&s, nodes, q, kc, vc, table, ctx, parents, sizes, real(a[11]),
                                                             real(a[12]), real(a[13]), out, ws, bytes, st);
    return entry<decltype(&ooco_tree_attention)>(a[0])(&s, nodes, q, kc, vc, table, ctx, parents, sizes, real(a[11]), out, ws,
                                                       bytes, st);
  });
}

struct Probs {
  const float* p;
  int64_t seq, node;
};
Probs probs(PyObject* o, int dev, int64_t B, int64_t N, int64_t V, const char* what) {
  const at::Tensor& t = tensor(o, what);
  if (!(t.is_cuda() && t.get_device() == dev && t.scalar_type() == kF32 && t.dim() == 3 && t.size(0) == B && t.size(1) == N &&
        t.size(2) == V && (V == 1 || t.stride(2) == 1))) {
    refuse(std::string(what) + ": expected Float " + list({B, N, V}) + " with dense rows on cuda:" + std::to_string(dev) +
           ", got " + describe(t));
  }
  return {(const float*)t.data_ptr(), t.stride(0), t.stride(1)};
}

// entry, target_probs, draft_probs, tokens, parents, uniforms, path, out_tokens, num_accepted, tree_sizes, stream
PyObject* verify_drafts(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded("verify_drafts", n, 11, [&] {
    const auto fn = entry<decltype(&ooco_verify_drafts)>(a[0]);
    const at::Tensor& t = tensor(a[1], "target_probs");
    const int dev = device_of(t, "target_probs");
    if (t.dim() != 3) refuse("target_probs: expected [batch, nodes, vocabulary], got " + describe(t));
    const int64_t B = t.size(0), N = t.size(1), V = t.size(2);
    const Probs p = probs(a[1], dev, B, N, V, "target_probs");
    const Probs q = a[2] == Py_None ? Probs{nullptr, 0, 0} : probs(a[2], dev, B, N, V, "draft_probs");
    const auto* tokens = (const int32_t*)address(a[3], dev, kI32, "tokens", {B, N});
    const auto* parents = (const int32_t*)optional(a[4], dev, kI32, "parents", {B, N});
    const auto* u = (const float*)address(a[5], dev, kF32, "uniforms", {B, N});
    auto* path = (int32_t*)address(a[6], dev, kI32, "path", {B, N});
    auto* out = (int32_t*)address(a[7], dev, kI32, "out_tokens", {B, N});
    auto* count = (int32_t*)address(a[8], dev, kI32, "num_accepted", {B});
    const auto* sizes = (const int32_t*)optional(a[9], dev, kI32, "tree_sizes", {B});
    void* st = stream_of(a[10], dev);
    const c10::cuda::OptionalCUDAGuard guard(at::Device(at::kCUDA, (c10::DeviceIndex)dev));
    const ooco_verify_t s = {count32(B, "target_probs"), count32(N, "target_probs"), count32(V, "target_probs"), 0, p.seq, p.node,
                             q.seq, q.node};
    return fn(&s, p.p, q.p, tokens, parents, sizes, u, path, out, count, st);
  });
}

// entry, 8-bit cache, shape, k_cache, v_cache, block_table, base_lens, path, num_accepted, context_lens_out, stream
PyObject* kv_keep_path(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded("kv_keep_path", n, 11, [&] {
    const auto fn = entry<decltype(&ooco_kv_keep_path)>(a[0]);
    const ooco_shape_t& s = shape_at(a[2]);
    const at::Tensor& path_t = tensor(a[7], "path");
    const int dev = device_of(path_t, "path");
    const int64_t B = s.batch, N = path_t.dim() == 2 ? path_t.size(1) : -1;
    const at::ScalarType cell = a[1] == Py_True ? kU8 : kBf;
    void* kc = address(a[3], dev, cell, "k_cache", {}, pool_elements(s));
    void* vc = address(a[4], dev, cell, "v_cache", {}, pool_elements(s));
    const auto* table = (const int32_t*)address(a[5], dev, kI32, "block_table", {B, s.max_blocks_per_seq});
    const auto* base = (const int32_t*)address(a[6], dev, kI32, "base_lens", {B});
    const auto* path = (const int32_t*)address(a[7], dev, kI32, "path", {B, N});
    const auto* count = (const int32_t*)address(a[8], dev, kI32, "num_accepted", {B});
    auto* out = (int32_t*)optional(a[9], dev, kI32, "context_lens_out", {B});
    void* st = stream_of(a[10], dev);
    const c10::cuda::OptionalCUDAGuard guard(at::Device(at::kCUDA, (c10::DeviceIndex)dev));
    return fn(&s, count32(N, "path"), kc, vc, table, base, path, count, out, st);
  });
}

#define METHOD(name) {#name, (PyCFunction)(void (*)(void))name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {METHOD(plan_slots),    METHOD(rope_kv_append), METHOD(tree_attention),
                         METHOD(verify_drafts), METHOD(kv_keep_path),   {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_spec_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

#ifndef OOCO_BUILT_FOR
#define OOCO_BUILT_FOR ""
#endif
PyMODINIT_FUNC PyInit__spec_calls() {
  PyObject* m = PyModule_Create(&module);
  if (m && PyModule_AddStringConstant(m, "built_for", OOCO_BUILT_FOR)) {
    Py_DECREF(m);
    return nullptr;
  }
  return m;
}
