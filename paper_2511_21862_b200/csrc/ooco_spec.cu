// Host side of ooco_spec.h, except ooco_tree_attention (ooco_api.cu): argument validation and launches.
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "../../include/ooco_spec.h"
#include "api_internal.h"
#include "spec_kernels.cuh"

namespace ooco {

static_assert(kTreeMaxNodes == OOCO_TREE_MAX_NODES, "node limit");
static_assert(kSlotsStatusBadBlock == OOCO_STATUS_BAD_BLOCK && kSlotsStatusRefused == OOCO_STATUS_REFUSED, "status bits");

static int log2_of(int x) {  // x: a power of two
  int k = 0;
  while ((1 << k) < x) ++k;
  return k;
}

static size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

static int finish(cudaError_t e, const char* where) {
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? OOCO_OK : fail_cuda(where, (long)e);
}

static int sm_count_of_current(int* sms) {
  int dev = 0;
  if (current_device(&dev)) return fail_cuda("cudaGetDevice", -1);
  *sms = device_info(dev).sm_count;
  return *sms > 0 ? OOCO_OK : fail_cuda("cudaDeviceGetAttribute", -1);
}

struct Range {
  const void* p;
  size_t bytes;
};
static bool overlap(const Range& a, const Range& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

// Whether any of T rows of `la` bytes, `sa` apart from `a` on, shares memory with any of T rows of `lb` bytes, `sb` apart from
// `b` on (rows of one spacing may lie in one another's gaps, as the parts of a projection do).
static bool rows_overlap(const void* a, int64_t sa, int64_t la, const void* b, int64_t sb, int64_t lb, int64_t T) {
  if (!overlap({a, (size_t)((T - 1) * sa + la)}, {b, (size_t)((T - 1) * sb + lb)})) return false;
  if (T == 1 || sa != sb) return true;
  const int64_t d = (int64_t)((uintptr_t)b - (uintptr_t)a) % sa, gap = d < 0 ? d + sa : d;  // b's row begins this far into a's period
  return gap < la || gap + lb > sa;
}

// Up to this many rows the scanning CTA also writes the rows (one launch).
constexpr int kSlotsOneLaunchRows = 4096;

static int rope_append(const ooco_shape_t* s, const ooco_rope_t* r, int32_t T, const void* q, int64_t q_stride,
                       const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* positions,
                       const int32_t* slot_map, void* q_out, int64_t q_out_stride, void* k_cache, void* v_cache,
                       bool kv8, float k_scale, float v_scale, void* cuda_stream) {
  int rc = validate_shape(s);
  if (rc) return rc;
  if (!r) return OOCO_E_NULLPTR;
  if (r->reserved != 0 || r->rot_dim <= 0 || r->rot_dim > s->head_dim || (r->interleaved != 0 && r->interleaved != 1) ||
      !std::isfinite(r->magnitude) || T < 0)
    return OOCO_E_SHAPE;
  if (r->rot_dim % 16) return OOCO_E_UNSUPPORTED;
  if (kv8) {
    if (!(k_scale > 0.f) || !(v_scale > 0.f)) return OOCO_E_SHAPE;
    if (s->head_dim != 128 || ((s->kv_block_stride | s->kv_head_stride | s->kv_token_stride) & 15)) return OOCO_E_UNSUPPORTED;
  }
  if ((int64_t)s->num_blocks * s->block_size > INT32_MAX) return OOCO_E_UNSUPPORTED;
  if (!r->inv_freq || !k_cache || !v_cache) return OOCO_E_NULLPTR;
  if (T > 0 && (!q || !k || !v || !positions || !slot_map || !q_out)) return OOCO_E_NULLPTR;
  const int64_t q_row = (int64_t)s->num_q_heads * s->head_dim, kv_row = (int64_t)s->num_kv_heads * s->head_dim;
  if (q_stride < q_row || q_out_stride < q_row || k_stride < kv_row || v_stride < kv_row) return OOCO_E_SHAPE;
  if (q == q_out && q_stride != q_out_stride) return OOCO_E_SHAPE;
  if (((q_stride | q_out_stride | k_stride | v_stride) & 7) ||
      (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_out | (uintptr_t)k_cache | (uintptr_t)v_cache) & 15) ||
      ((uintptr_t)r->inv_freq & 3))
    return OOCO_E_UNSUPPORTED;
  if (T == 0) return OOCO_OK;
  if (rows_overlap(q_out, 2 * q_out_stride, 2 * q_row, k, 2 * k_stride, 2 * kv_row, T) ||
      rows_overlap(q_out, 2 * q_out_stride, 2 * q_row, v, 2 * v_stride, 2 * kv_row, T) ||
      (q_out != q && rows_overlap(q_out, 2 * q_out_stride, 2 * q_row, q, 2 * q_stride, 2 * q_row, T)))
    return OOCO_E_SHAPE;
  int sms = 0;
  if ((rc = sm_count_of_current(&sms))) return rc;
  RopeParams p;
  memset(&p, 0, sizeof p);
  p.q = (const uint16_t*)q;
  p.k = (const uint16_t*)k;
  p.v = (const uint16_t*)v;
  p.q_out = (uint16_t*)q_out;
  p.k_cache = (uint8_t*)k_cache;
  p.v_cache = (uint8_t*)v_cache;
  p.positions = positions;
  p.slots = slot_map;
  p.inv_freq = r->inv_freq;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.q_out_stride = q_out_stride;
  p.bstr = s->kv_block_stride;
  p.hstr = s->kv_head_stride;
  p.tstr = s->kv_token_stride;
  p.T = T;
  p.Hq = s->num_q_heads;
  p.Hkv = s->num_kv_heads;
  p.half = r->rot_dim / 2;
  p.bs_log2 = log2_of(s->block_size);
  p.num_slots = (int64_t)s->num_blocks * s->block_size;
  p.magnitude = r->magnitude;
  p.k_scale = k_scale;
  p.v_scale = v_scale;
  // one token per CTA while the tokens alone do not fill the SMs, else tiles that amortise the barriers
  p.tile = T <= 4 * sms ? 1 : kRopeMaxTile;
  const int tiles = (T + p.tile - 1) / p.tile, cap = 8 * sms;
  const dim3 grid(tiles < cap ? tiles : cap), block(kRopeThreads);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const bool pdl = pdl_enabled();
  cudaError_t e;
  if (kv8)
    e = launch_ex(rope_append_kernel<128, true>, grid, block, 0, st, pdl, p, (int)r->interleaved);
  else if (s->head_dim == 128)
    e = launch_ex(rope_append_kernel<128, false>, grid, block, 0, st, pdl, p, (int)r->interleaved);
  else
    e = launch_ex(rope_append_kernel<64, false>, grid, block, 0, st, pdl, p, (int)r->interleaved);
  return finish(e, "launch of the rotary append kernel");
}

static int keep_path(const ooco_shape_t* s, int32_t max_nodes, void* k_cache, void* v_cache, const int32_t* block_table,
                     const int32_t* base_lens, const int32_t* path, const int32_t* num_accepted,
                     int32_t* context_lens_out, bool kv8, void* cuda_stream) {
  int rc = validate_shape(s);
  if (rc) return rc;
  if (max_nodes < 1) return OOCO_E_SHAPE;
  if (max_nodes > OOCO_TREE_MAX_NODES) return OOCO_E_UNSUPPORTED;
  if (kv8 && (s->head_dim != 128 || ((s->kv_block_stride | s->kv_head_stride | s->kv_token_stride) & 15)))
    return OOCO_E_UNSUPPORTED;
  if (!k_cache || !v_cache || !block_table || !base_lens || !path || !num_accepted) return OOCO_E_NULLPTR;
  // (one CTA of a sequence writes its length while others may still read these)
  const size_t w = 4, n = (size_t)s->batch * w;
  for (const Range& r : {Range{base_lens, n}, Range{num_accepted, n}, Range{path, n * max_nodes}, Range{block_table, n * s->max_blocks_per_seq}})
    if (overlap({context_lens_out, n}, r)) return OOCO_E_SHAPE;
  if (((uintptr_t)k_cache | (uintptr_t)v_cache) & 15) return OOCO_E_UNSUPPORTED;
  const int cell = kv8 ? 1 : 2;
  KeepParams p;
  memset(&p, 0, sizeof p);
  p.k_cache = (uint8_t*)k_cache;
  p.v_cache = (uint8_t*)v_cache;
  p.block_table = block_table;
  p.base_lens = base_lens;
  p.path = path;
  p.num_accepted = num_accepted;
  p.context_lens_out = context_lens_out;
  p.bstr = s->kv_block_stride * cell;
  p.hstr = s->kv_head_stride * cell;
  p.tstr = s->kv_token_stride * cell;
  p.B = s->batch;
  p.N = max_nodes;
  p.Hkv = s->num_kv_heads;
  p.row_vecs = s->head_dim * cell / 16;
  p.bs_log2 = log2_of(s->block_size);
  p.NB = s->num_blocks;
  p.MB = s->max_blocks_per_seq;
  const int64_t cols = 2ll * p.Hkv * p.row_vecs, want = (cols + kKeepThreads - 1) / kKeepThreads;
  const dim3 grid(s->batch, (unsigned)(want < 1024 ? want : 1024));
  return finish(launch_ex(keep_path_kernel, grid, dim3(kKeepThreads), 0, (cudaStream_t)cuda_stream, pdl_enabled(), p),
                "launch of the branch-keeping kernel");
}

}  // namespace ooco

using namespace ooco;

extern "C" {

size_t ooco_plan_slots_workspace_bytes(const ooco_shape_t* s) {
  if (validate_shape(s)) return 0;
  return 2 * up256((size_t)s->batch * 4);
}

int ooco_plan_slots(const ooco_shape_t* s, const int32_t* context_lens, const int32_t* new_lens, int32_t* block_table,
                    int32_t* blocks_held, const int32_t* free_ids, int32_t num_free, int32_t* free_head,
                    int32_t* blocks_held_out, int32_t* free_head_out, int32_t row_len, int32_t num_rows,
                    const int32_t* parents, int32_t* slot_map, int32_t* positions, int32_t* first_token,
                    int32_t* granted_lens, int32_t* total_lens, void* workspace, size_t workspace_bytes,
                    int32_t* status, void* cuda_stream) {
  int rc = validate_shape(s);
  if (rc) return rc;
  if (num_free < 0 || row_len < 0 || num_rows < 0) return OOCO_E_SHAPE;
  if (row_len > 0 && (int64_t)s->batch * row_len != num_rows) return OOCO_E_SHAPE;
  if ((int64_t)s->num_blocks * s->block_size > INT32_MAX) return OOCO_E_UNSUPPORTED;
  if (!context_lens || !new_lens || !block_table || !blocks_held || !free_head || !first_token || !granted_lens ||
      !total_lens || !workspace || (num_free > 0 && !free_ids) || (num_rows > 0 && (!slot_map || !positions)))
    return OOCO_E_NULLPTR;
  if (workspace_bytes < ooco_plan_slots_workspace_bytes(s) || ((uintptr_t)workspace & 255)) return OOCO_E_WORKSPACE;
  {  // rows are filled from the inputs after the per-sequence outputs are written: nothing written may share their memory
    const size_t w = 4, n = (size_t)s->batch * w, rows = (size_t)num_rows * w;
    const Range in[] = {{context_lens, n}, {new_lens, n}, {blocks_held, n}, {free_head, w}, {free_ids, num_free * w}, {parents, rows}};
    const Range out[] = {{blocks_held_out == blocks_held ? nullptr : blocks_held_out, n},
                         {free_head_out == free_head ? nullptr : free_head_out, w},
                         {block_table, n * s->max_blocks_per_seq}, {slot_map, rows}, {positions, rows}, {first_token, n + w},
                         {granted_lens, n}, {total_lens, n}, {workspace, ooco_plan_slots_workspace_bytes(s)}, {status, w}};
    constexpr int kOut = sizeof out / sizeof *out;
    for (int i = 0; i < kOut; ++i) {
      for (const Range& r : in)
        if (overlap(out[i], r)) return OOCO_E_SHAPE;
      for (int j = 0; j < i; ++j)
        if (overlap(out[i], out[j])) return OOCO_E_SHAPE;
    }
  }
  int sms = 0;
  if ((rc = sm_count_of_current(&sms))) return rc;
  SlotsParams p;
  memset(&p, 0, sizeof p);
  p.context_lens = context_lens;
  p.new_lens = new_lens;
  p.blocks_held = blocks_held;
  p.free_ids = free_ids;
  p.free_head = free_head;
  p.parents = parents;
  p.block_table = block_table;
  p.blocks_held_out = blocks_held_out ? blocks_held_out : blocks_held;
  p.free_head_out = free_head_out ? free_head_out : free_head;
  p.slot_map = slot_map;
  p.positions = positions;
  p.first_token = first_token;
  p.granted = granted_lens;
  p.total = total_lens;
  p.status = status;
  p.ws_from = (int32_t*)workspace;
  p.ws_held = (int32_t*)((uint8_t*)workspace + up256((size_t)s->batch * 4));
  p.B = s->batch;
  p.bs_log2 = log2_of(s->block_size);
  p.NB = s->num_blocks;
  p.MB = s->max_blocks_per_seq;
  p.num_free = num_free;
  p.row_len = row_len;
  p.num_rows = num_rows;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const bool one = num_rows <= kSlotsOneLaunchRows, pdl = pdl_enabled();
  if ((rc = finish(launch_ex(slots_scan_kernel, dim3(1), dim3(kSlotsThreads), 0, st, pdl, p, one ? 1 : 0),
                   "launch of the slot planning kernel")))
    return rc;
  if (one) return OOCO_OK;
  const int64_t want = ((int64_t)num_rows + 1023) / 1024, cap = 8ll * sms;
  return finish(launch_ex(slots_fill_kernel, dim3((unsigned)(want < cap ? want : cap)), dim3(256), 0, st, pdl, p),
                "launch of the slot map kernel");
}

int ooco_rope_frequencies(int32_t rot_dim, double base, const ooco_rope_scaling_t* sc, float* inv_freq, float* magnitude) {
  if (!inv_freq || !magnitude) return OOCO_E_NULLPTR;
  if (rot_dim < 2 || rot_dim % 2 || !(base > 1.0) || !std::isfinite(base)) return OOCO_E_SHAPE;
  const int kind = sc ? sc->kind : OOCO_ROPE_PLAIN;
  if (kind < OOCO_ROPE_PLAIN || kind > OOCO_ROPE_RAMP) return OOCO_E_SHAPE;
  if (kind != OOCO_ROPE_PLAIN && (!(sc->factor >= 1.0) || !std::isfinite(sc->factor))) return OOCO_E_SHAPE;
  if (kind >= OOCO_ROPE_BANDS && (sc->original_len <= 0 || !(sc->low > 0.0) || !(sc->high > sc->low) || !std::isfinite(sc->high)))
    return OOCO_E_SHAPE;
  if (kind == OOCO_ROPE_STRETCH && rot_dim == 2) return OOCO_E_SHAPE;
  const double pi = 3.14159265358979323846, f = kind ? sc->factor : 1.0;
  const int half = rot_dim / 2;
  if (kind == OOCO_ROPE_STRETCH) base *= std::pow(f, (double)rot_dim / (rot_dim - 2));
  // RAMP: the index whose frequency turns `turns` times over original_len
  auto index_of = [&](double turns) { return rot_dim * std::log(sc->original_len / (turns * 2 * pi)) / (2 * std::log(base)); };
  double lo = 0, hi = 0;
  if (kind == OOCO_ROPE_RAMP) {
    // (the ramp may end beyond the last frequency: the slowest one turns more than `low` times then, and is divided by less)
    lo = std::fmax(std::floor(index_of(sc->high)), 0.0);
    hi = std::fmin(std::ceil(index_of(sc->low)), (double)(rot_dim - 1));
    if (index_of(sc->low) < 0) {  // even the fastest turns less than `low` times
      lo = -1;
      hi = 0;
    } else if (hi <= lo) {
      hi = lo + 1e-3;
    }
  }
  for (int j = 0; j < half; ++j) {
    double w = std::pow(base, -2.0 * j / rot_dim);
    if (kind == OOCO_ROPE_LINEAR) w /= f;
    if (kind == OOCO_ROPE_BANDS) {
      const double turns = sc->original_len * w / (2 * pi);  // original_len / wavelength
      double keep = (turns - sc->low) / (sc->high - sc->low);
      keep = keep < 0 ? 0 : (keep > 1 ? 1 : keep);
      w = (1 - keep) * w / f + keep * w;
    }
    if (kind == OOCO_ROPE_RAMP) {
      double gone = (j - lo) / (hi - lo);
      gone = gone < 0 ? 0 : (gone > 1 ? 1 : gone);
      w = w / f * gone + w * (1 - gone);
    }
    inv_freq[j] = (float)w;
  }
  *magnitude = kind == OOCO_ROPE_RAMP ? (float)(0.1 * std::log(f) + 1.0) : 1.f;
  return OOCO_OK;
}

int ooco_rope_kv_append(const ooco_shape_t* shape, const ooco_rope_t* rope, int32_t num_tokens, const void* q,
                        int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                        const int32_t* positions, const int32_t* slot_map, void* q_out, int64_t q_out_stride,
                        void* k_cache, void* v_cache, void* cuda_stream) {
  return rope_append(shape, rope, num_tokens, q, q_stride, k, k_stride, v, v_stride, positions, slot_map, q_out,
                     q_out_stride, k_cache, v_cache, false, 1.f, 1.f, cuda_stream);
}

int ooco_rope_kv_append_fp8(const ooco_shape_t* shape, const ooco_rope_t* rope, int32_t num_tokens, const void* q,
                            int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                            const int32_t* positions, const int32_t* slot_map, void* q_out, int64_t q_out_stride,
                            void* k_cache, void* v_cache, float k_scale, float v_scale, void* cuda_stream) {
  return rope_append(shape, rope, num_tokens, q, q_stride, k, k_stride, v, v_stride, positions, slot_map, q_out,
                     q_out_stride, k_cache, v_cache, true, k_scale, v_scale, cuda_stream);
}

int ooco_verify_drafts(const ooco_verify_t* s, const float* target_probs, const float* draft_probs, const int32_t* tokens,
                       const int32_t* parents, const int32_t* tree_sizes, const float* uniforms, int32_t* path,
                       int32_t* out_tokens, int32_t* num_accepted, void* cuda_stream) {
  if (!s) return OOCO_E_NULLPTR;
  if (s->batch <= 0 || s->max_nodes <= 0 || s->vocab <= 0 || s->reserved != 0) return OOCO_E_SHAPE;
  if (s->max_nodes > OOCO_TREE_MAX_NODES || s->vocab > OOCO_MAX_VOCAB || s->batch > (1 << 24)) return OOCO_E_UNSUPPORTED;
  if (s->target_node_stride < 0 || s->target_seq_stride < 0 || (draft_probs && (s->draft_node_stride < 0 || s->draft_seq_stride < 0)))
    return OOCO_E_SHAPE;
  if (!target_probs || !tokens || !uniforms || !path || !out_tokens || !num_accepted) return OOCO_E_NULLPTR;
  if (((uintptr_t)target_probs | (uintptr_t)draft_probs) & 3) return OOCO_E_UNSUPPORTED;
  int sms = 0, rc;
  if ((rc = sm_count_of_current(&sms))) return rc;
  VerifyParams p;
  memset(&p, 0, sizeof p);
  p.target = target_probs;
  p.draft = draft_probs;
  p.uniforms = uniforms;
  p.tokens = tokens;
  p.parents = parents;
  p.tree_sizes = tree_sizes;
  p.path = path;
  p.out_tokens = out_tokens;
  p.num_accepted = num_accepted;
  p.t_seq = s->target_seq_stride;
  p.t_node = s->target_node_stride;
  p.d_seq = s->draft_seq_stride;
  p.d_node = s->draft_node_stride;
  p.B = s->batch;
  p.N = s->max_nodes;
  p.V = s->vocab;
  // CTAs per sequence and their threads.  Few sequences (16 CTAs each do not fill the SMs twice): the largest cluster of
  // large CTAs shortens the pass over the vocabulary (4 sequences of 152064 values: 11.7 us; with an earlier, slower pass
  // 13.3, and 17.8 with 8 x 256).  Else 8 CTAs of 256 threads, so that four CTAs per SM hide each other's serial phases (128
  // sequences of 128256 values: 50.5 us; when that was 49.7, 4 x 512 took 58 and 8 x 512 took 65), and fewer as the sequences
  // alone give the GPU enough CTAs.  At least so many that a share's bit map fits shared memory (2^17 values), at most one per
  // tile of the vocabulary.
  int cluster = kVerifyMaxCluster, threads = kVerifyThreads;
  if ((int64_t)s->batch * cluster > 2ll * sms) {
    threads = 256;
    cluster = 8;
    while (cluster > 1 && (int64_t)s->batch * cluster > 8ll * sms) cluster /= 2;
    while ((int64_t)cluster << 17 < s->vocab) cluster *= 2;
  }
  while (cluster > 1 && (int64_t)(cluster / 2) * kVerifyTile >= s->vocab) cluster /= 2;
  static std::atomic<int> configured[64];
  int dev = 0;
  if (cluster > 8 && (current_device(&dev) || dev >= 64 || !configured[dev].load())) {
    const cudaError_t e = cudaFuncSetAttribute(verify_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return fail_cuda("cudaFuncSetAttribute(cluster size)", (long)e);
    if (dev < 64) configured[dev].store(1);
  }
  return finish(launch_clustered(verify_kernel, dim3((unsigned)(s->batch * cluster)), dim3(threads), 0,
                                 (cudaStream_t)cuda_stream, pdl_enabled(), (unsigned)cluster, p, cluster),
                "launch of the verification kernel");
}

int ooco_kv_keep_path(const ooco_shape_t* shape, int32_t max_nodes, void* k_cache, void* v_cache,
                      const int32_t* block_table, const int32_t* base_lens, const int32_t* path,
                      const int32_t* num_accepted, int32_t* context_lens_out, void* cuda_stream) {
  return keep_path(shape, max_nodes, k_cache, v_cache, block_table, base_lens, path, num_accepted, context_lens_out, false,
                   cuda_stream);
}

int ooco_kv_keep_path_fp8(const ooco_shape_t* shape, int32_t max_nodes, void* k_cache, void* v_cache,
                          const int32_t* block_table, const int32_t* base_lens, const int32_t* path,
                          const int32_t* num_accepted, int32_t* context_lens_out, void* cuda_stream) {
  return keep_path(shape, max_nodes, k_cache, v_cache, block_table, base_lens, path, num_accepted, context_lens_out, true,
                   cuda_stream);
}

}  // extern "C"
