// The calls of ooco_batch.h in the module `_spec_calls` (py_spec.cpp).
#include "py_calls.h"

// entry, shape, parents, children, shared_lens, context_lens, block_table, blocks_held, free_ids, free_head, shares, the four
// outputs, copy_src, copy_dst, granted, workspace, status, stream
OOCO_CALL(fork_pages) {
  return guarded("fork_pages", n, 21, [&] {
    const ooco_shape_t& s = shape_at(a[1]);
    const at::Tensor& list = tensor(a[2], "parents");
    const int dev = device_of(list, "parents");
    const int64_t F = list.numel(), B = s.batch, num_free = tensor(a[8], "free_ids").numel();
    const auto* parents = (const int32_t*)address(a[2], dev, kI32, "parents", {F});
    const auto* children = (const int32_t*)address(a[3], dev, kI32, "children", {F});
    const auto* lens = (const int32_t*)optional(a[4], dev, kI32, "shared_lens", {F});
    auto* ctx = (int32_t*)address(a[5], dev, kI32, "context_lens", {B});
    auto* table = (int32_t*)address(a[6], dev, kI32, "block_table", {B, s.max_blocks_per_seq});
    auto* held = (int32_t*)address(a[7], dev, kI32, "blocks_held", {B});
    const auto* ids = (const int32_t*)address(a[8], dev, kI32, "free_ids");
    auto* head = (int32_t*)address(a[9], dev, kI32, "free_head", {1});
    auto* shares = (int32_t*)address(a[10], dev, kI32, "shares", {s.num_blocks});
    auto* ctx_out = (int32_t*)optional(a[11], dev, kI32, "context_lens_out", {B});
    auto* held_out = (int32_t*)optional(a[12], dev, kI32, "blocks_held_out", {B});
    auto* head_out = (int32_t*)optional(a[13], dev, kI32, "free_head_out", {1});
    auto* shares_out = (int32_t*)optional(a[14], dev, kI32, "shares_out", {s.num_blocks});
    auto* src = (int32_t*)address(a[15], dev, kI32, "copy_src", {F});
    auto* dst = (int32_t*)address(a[16], dev, kI32, "copy_dst", {F});
    auto* granted = (int32_t*)address(a[17], dev, kI32, "granted", {F});
    void* ws = address(a[18], dev, kU8, "workspace");
    auto* status = (int32_t*)optional(a[19], dev, kI32, "status", {1});
    void* st = stream_of(a[20], dev);
    const c10::cuda::OptionalCUDAGuard guard(at::Device(at::kCUDA, (c10::DeviceIndex)dev));
    return entry<decltype(&ooco_fork_pages)>(a[0])(&s, count32(F, "parents"), parents, children, lens, ctx, table, held, ids,
                                                   count32(num_free, "free_ids"), head, shares, ctx_out, held_out, head_out,
                                                   shares_out, src, dst, granted, ws,
                                                   (size_t)THPVariable_Unpack(a[18]).numel(), status, st);
  });
}

// entry, shape, rows, keep_lens, context_lens, block_table, blocks_held, free_ids, free_head, shares, the four outputs,
// workspace, status, stream
OOCO_CALL(release_pages) {
  return guarded("release_pages", n, 17, [&] {
    const ooco_shape_t& s = shape_at(a[1]);
    const at::Tensor& list = tensor(a[2], "rows");
    const int dev = device_of(list, "rows");
    const int64_t R = list.numel(), B = s.batch, num_free = tensor(a[7], "free_ids").numel();
    const auto* rows = (const int32_t*)address(a[2], dev, kI32, "rows", {R});
    const auto* lens = (const int32_t*)optional(a[3], dev, kI32, "keep_lens", {R});
    auto* ctx = (int32_t*)address(a[4], dev, kI32, "context_lens", {B});
    const auto* table = (const int32_t*)address(a[5], dev, kI32, "block_table", {B, s.max_blocks_per_seq});
    auto* held = (int32_t*)address(a[6], dev, kI32, "blocks_held", {B});
    auto* ids = (int32_t*)address(a[7], dev, kI32, "free_ids");
    auto* head = (int32_t*)address(a[8], dev, kI32, "free_head", {1});
    auto* shares = (int32_t*)address(a[9], dev, kI32, "shares", {s.num_blocks});
    auto* ctx_out = (int32_t*)optional(a[10], dev, kI32, "context_lens_out", {B});
    auto* held_out = (int32_t*)optional(a[11], dev, kI32, "blocks_held_out", {B});
    auto* head_out = (int32_t*)optional(a[12], dev, kI32, "free_head_out", {1});
    auto* shares_out = (int32_t*)optional(a[13], dev, kI32, "shares_out", {s.num_blocks});
    void* ws = address(a[14], dev, kU8, "workspace");
    auto* status = (int32_t*)optional(a[15], dev, kI32, "status", {1});
    void* st = stream_of(a[16], dev);
    const c10::cuda::OptionalCUDAGuard guard(at::Device(at::kCUDA, (c10::DeviceIndex)dev));
    return entry<decltype(&ooco_release_pages)>(a[0])(&s, count32(R, "rows"), rows, lens, ctx, table, held, ids,
                                                      count32(num_free, "free_ids"), head, shares, ctx_out, held_out, head_out,
                                                      shares_out, ws, (size_t)THPVariable_Unpack(a[14]).numel(), status, st);
  });
}

// entry, 8-bit cache, shape, ooco_rope_t, inv_freq, ooco_head_norm_t, q_weight, k_weight, q, k, v, positions, slot_map, q_out,
// k_cache, v_cache, scales, stream
OOCO_CALL(norm_rope_kv_append) {
  return guarded("norm_rope_kv_append", n, 19, [&] {
    const bool kv8 = a[1] == Py_True;
    const ooco_shape_t& s = shape_at(a[2]);
    ooco_rope_t r = *reinterpret_cast<const ooco_rope_t*>((uintptr_t)integer(a[3]));
    ooco_head_norm_t norm = *reinterpret_cast<const ooco_head_norm_t*>((uintptr_t)integer(a[5]));
    const at::Tensor& q_t = tensor(a[8], "q");
    const int dev = device_of(q_t, "q");
    r.inv_freq = (const float*)address(a[4], dev, kF32, "inv_freq", {r.rot_dim / 2});
    norm.q_weight = optional(a[6], dev, kBf, "q_weight", {s.head_dim});
    norm.k_weight = optional(a[7], dev, kBf, "k_weight", {s.head_dim});
    const int64_t T = q_t.dim() ? q_t.size(0) : -1;
    const Rows q = rows(a[8], dev, T, s.num_q_heads, s.head_dim, "q"), k = rows(a[9], dev, T, s.num_kv_heads, s.head_dim, "k"),
               v = rows(a[10], dev, T, s.num_kv_heads, s.head_dim, "v");
    const auto* pos = (const int32_t*)address(a[11], dev, kI32, "positions", {T});
    const auto* slots = (const int32_t*)address(a[12], dev, kI32, "slot_map", {T});
    const Rows out = rows(a[13], dev, T, s.num_q_heads, s.head_dim, "q_out");
    const at::ScalarType cell = kv8 ? kU8 : kBf;
    void* kc = address(a[14], dev, cell, "k_cache", {}, pool_elements(s));
    void* vc = address(a[15], dev, cell, "v_cache", {}, pool_elements(s));
    void* st = stream_of(a[18], dev);
    const c10::cuda::OptionalCUDAGuard guard(at::Device(at::kCUDA, (c10::DeviceIndex)dev));
    const int32_t tokens = count32(T, "q");
    if (kv8)
      return entry<decltype(&ooco_norm_rope_kv_append_fp8)>(a[0])(&s, &r, &norm, tokens, q.p, q.stride, k.p, k.stride, v.p,
                                                                  v.stride, pos, slots, out.p, out.stride, kc, vc, real(a[16]),
                                                                  real(a[17]), st);
    return entry<decltype(&ooco_norm_rope_kv_append)>(a[0])(&s, &r, &norm, tokens, q.p, q.stride, k.p, k.stride, v.p, v.stride,
                                                            pos, slots, out.p, out.stride, kc, vc, st);
  });
}

// entry, 8-bit cache, shape, q, k_cache, v_cache, block_table, context_lens, first_row, max_chunk, scale, k_scale, v_scale,
// out, workspace, chunk_lens, stream
OOCO_CALL(chunk_attention) {
  return guarded("chunk_attention", n, 17, [&] {
    const bool kv8 = a[1] == Py_True;
    const ooco_shape_t& s = shape_at(a[2]);
    const at::Tensor& q_t = tensor(a[3], "q");
    const int dev = device_of(q_t, "q");
    const int64_t R = q_t.dim() ? q_t.size(0) : -1, B = s.batch;
    const Rows q = rows(a[3], dev, R, s.num_q_heads, s.head_dim, "q");
    const at::ScalarType cell = kv8 ? kU8 : kBf;
    const void* kc = address(a[4], dev, cell, "k_cache", {}, pool_elements(s));
    const void* vc = address(a[5], dev, cell, "v_cache", {}, pool_elements(s));
    const auto* table = (const int32_t*)address(a[6], dev, kI32, "block_table", {B, s.max_blocks_per_seq});
    const auto* ctx = (const int32_t*)address(a[7], dev, kI32, "context_lens", {B});
    const auto* first = (const int32_t*)address(a[8], dev, kI32, "first_row", {B + 1});
    const int32_t max_chunk = integer32(a[9], "max_chunk");
    const Rows out = rows(a[13], dev, R, s.num_q_heads, s.head_dim, "out");
    void* ws = address(a[14], dev, kU8, "workspace");
    const size_t bytes = (size_t)THPVariable_Unpack(a[14]).numel();
    const auto* lens = (const int32_t*)optional(a[15], dev, kI32, "chunk_lens", {B});
    void* st = stream_of(a[16], dev);
    const c10::cuda::OptionalCUDAGuard guard(at::Device(at::kCUDA, (c10::DeviceIndex)dev));
    const int32_t num = count32(R, "q");
    if (kv8)
      return entry<decltype(&ooco_chunk_attention_fp8)>(a[0])(&s, num, max_chunk, q.p, q.stride, kc, vc, table, ctx, first, lens,
                                                              real(a[10]), real(a[11]), real(a[12]), out.p, out.stride, ws,
                                                              bytes, st);
    return entry<decltype(&ooco_chunk_attention)>(a[0])(&s, num, max_chunk, q.p, q.stride, kc, vc, table, ctx, first, lens,
                                                        real(a[10]), out.p, out.stride, ws, bytes, st);
  });
}

namespace {

struct Table {  // [B, N, V] or [B, V] (then N = 1)
  void* p = nullptr;
  int64_t B = 0, N = 0, V = 0, seq = 0, node = 0;
};
Table table_of(PyObject* o, const char* what) {
  const at::Tensor& t = tensor(o, what);
  if (t.dim() != 2 && t.dim() != 3) refuse(std::string(what) + ": expected [batch, vocabulary] or [batch, nodes, vocabulary], got " + describe(t));
  const bool three = t.dim() == 3;
  Table x;
  x.p = t.data_ptr();
  x.B = t.size(0);
  x.N = three ? t.size(1) : 1;
  x.V = t.size(-1);
  x.seq = t.stride(0);
  x.node = three ? t.stride(1) : x.V;
  return x;
}
// A table like `l` of another type, on the same device, with dense rows of `width`.
Table like(PyObject* o, int dev, at::ScalarType type, const Table& l, int64_t width, const char* what) {
  if (o == Py_None) return {};
  const at::Tensor& t = tensor(o, what);
  Table x;
  if (t.dim() == 2 || t.dim() == 3) x = table_of(o, what);
  if (!(t.is_cuda() && t.get_device() == dev && t.scalar_type() == type && x.B == l.B && x.N == l.N && x.V == width &&
        (width == 1 || t.stride(-1) == 1)))
    refuse(std::string(what) + ": expected " + c10::toString(type) + " " + list({l.B, l.N, width}) + " with dense rows on cuda:" +
           std::to_string(dev) + ", got " + describe(t));
  return x;
}

}  // namespace

// entry, logits, out, probs, temperature, repetition, frequency, presence, history, history_lens, prompt_lens, tokens, parents,
// tree_sizes, bias_tokens, bias_values, mask, stream
OOCO_CALL(shape_logits) {
  return guarded("shape_logits", n, 18, [&] {
    const at::Tensor& t = tensor(a[1], "logits");
    const int dev = device_of(t, "logits");
    const Table l = table_of(a[1], "logits");
    if ((t.scalar_type() != kBf && t.scalar_type() != kF32) || (l.V > 1 && t.stride(-1) != 1))
      refuse("logits: expected BFloat16 or Float with dense rows, got " + describe(t));
    const Table out = like(a[2], dev, kF32, l, l.V, "out"), probs = like(a[3], dev, kF32, l, l.V, "probs");
    const auto* temperature = (const float*)optional(a[4], dev, kF32, "temperature", {l.B});
    const auto* repetition = (const float*)optional(a[5], dev, kF32, "repetition", {l.B});
    const auto* frequency = (const float*)optional(a[6], dev, kF32, "frequency", {l.B});
    const auto* presence = (const float*)optional(a[7], dev, kF32, "presence", {l.B});
    int64_t width = 0, entries = 0;
    if (a[8] != Py_None) {
      const at::Tensor& h = tensor(a[8], "history");
      width = h.dim() == 2 ? h.size(1) : -1;
    }
    const auto* history = (const int32_t*)optional(a[8], dev, kI32, "history", {l.B, width});
    const auto* lens = (const int32_t*)optional(a[9], dev, kI32, "history_lens", {l.B});
    const auto* prompts = (const int32_t*)optional(a[10], dev, kI32, "prompt_lens", {l.B});
    const auto* tokens = (const int32_t*)optional(a[11], dev, kI32, "tokens", {l.B, l.N});
    const auto* parents = (const int32_t*)optional(a[12], dev, kI32, "parents", {l.B, l.N});
    const auto* sizes = (const int32_t*)optional(a[13], dev, kI32, "tree_sizes", {l.B});
    if (a[14] != Py_None) {
      const at::Tensor& x = tensor(a[14], "bias_tokens");
      entries = x.dim() == 2 ? x.size(1) : -1;
    }
    const auto* bias_tokens = (const int32_t*)optional(a[14], dev, kI32, "bias_tokens", {l.B, entries});
    const auto* bias_values = (const float*)optional(a[15], dev, kF32, "bias_values", {l.B, entries});
    Table m;
    if (a[16] != Py_None) {
      const at::Tensor& x = tensor(a[16], "mask");
      // (expanded dimensions have a stride of 0: one mask for several rows)
      m = like(a[16], dev, kI32, l, (l.V + 31) / 32, "mask");
      if (x.dim() == 2) m.node = 0;
    }
    void* st = stream_of(a[17], dev);
    const c10::cuda::OptionalCUDAGuard guard(at::Device(at::kCUDA, (c10::DeviceIndex)dev));
    const ooco_logits_t s = {count32(l.B, "logits"), count32(l.N, "logits"), count32(l.V, "logits"), t.scalar_type() == kF32,
                             count32(width, "history"), count32(entries, "bias_tokens"), l.seq, l.node, out.seq, out.node,
                             probs.seq, probs.node, m.seq, m.node};
    return entry<decltype(&ooco_shape_logits)>(a[0])(&s, l.p, temperature, repetition, frequency, presence, history, lens,
                                                     prompts, tokens, parents, sizes, bias_tokens, bias_values,
                                                     (const int32_t*)m.p, (float*)out.p, (float*)probs.p, st);
  });
}
