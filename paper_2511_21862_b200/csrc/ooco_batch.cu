// Host side of ooco_batch.h, except ooco_chunk_attention (ooco_chunk.cu): argument validation and launches.
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "../../include/ooco_batch.h"
#include "api_internal.h"
#include "logits_kernels.cuh"
#include "page_kernels.cuh"

namespace ooco {

static_assert(kPagesStatusBadBlock == OOCO_STATUS_BAD_BLOCK && kPagesStatusRefused == OOCO_STATUS_REFUSED, "status bits");
static_assert(kLogitsMaxBias == OOCO_MAX_BIAS && OOCO_MAX_SHAPED_VOCAB % (kLogitsMaxCluster * kLogitsBlock) == 0, "limits");

// Attributes of a kernel on the current device, set once: dynamic shared memory and clusters of 16 CTAs.
static int configure(const void* kern, std::atomic<int>* done, int smem) {
  int dev = 0;
  if (current_device(&dev)) return fail_cuda("cudaGetDevice", -1);
  if (dev < 64 && done[dev].load()) return OOCO_OK;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return fail_cuda("cudaFuncSetAttribute", (long)e);
  if (dev < 64) done[dev].store(1);
  return OOCO_OK;
}

// Clusters of the logits kernel that run at a time on the current device.  The last answer is kept (device, size, memory and answer in
// one word); where sizes alternate, the question adds 0.3 us to the 3 that a call takes the host.
static int64_t resident_clusters(const void* kern, std::atomic<uint64_t>& kept, int cluster_log2, size_t smem, int sms) {
  int dev = 0;
  cudaGetDevice(&dev);
  const uint64_t key = ((uint64_t)dev << 40 | (uint64_t)cluster_log2 << 32 | (uint64_t)smem) << 16;
  const uint64_t had = kept.load();
  if ((had & ~0xffffull) == key && (had & 0xffff)) return (int64_t)(had & 0xffff);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = 1u << cluster_log2;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(1u << cluster_log2);
  cfg.blockDim = dim3(kLogitsThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return sms >> cluster_log2 > 0 ? sms >> cluster_log2 : 1;  // (a share of the work for every CTA is all that hangs on it)
  }
  if (n > 0xffff) n = 0xffff;
  kept.store(key | (uint64_t)n);
  return n;
}

static int check_pages(const ooco_shape_t* s, int32_t n, int32_t num_free, const void* workspace, size_t workspace_bytes) {
  int rc = validate_shape(s);
  if (rc) return rc;
  if (n < 0 || num_free < 0) return OOCO_E_SHAPE;
  if (s->batch > OOCO_MAX_PAGE_ROWS || n > OOCO_MAX_PAGE_ROWS || (int64_t)n * s->max_blocks_per_seq > 1ll << 30)
    return OOCO_E_UNSUPPORTED;
  if (!workspace) return OOCO_E_NULLPTR;
  if (workspace_bytes < ooco_pages_workspace_bytes(s, n) || ((uintptr_t)workspace & 255)) return OOCO_E_WORKSPACE;
  return OOCO_OK;
}

// Nothing written shares memory with an input or another output.
static bool disjoint(const Range* in, int n_in, const Range* out, int n_out) {
  for (int i = 0; i < n_out; ++i) {
    for (int j = 0; j < n_in; ++j)
      if (overlap(out[i], in[j])) return false;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return false;
  }
  return true;
}

static PagesParams page_params(const ooco_shape_t* s, int32_t n, int32_t num_free, void* workspace) {
  PagesParams p;
  memset(&p, 0, sizeof p);
  p.ws_off = (int32_t*)workspace;
  p.ws_from = (int32_t*)((uint8_t*)workspace + up256(((size_t)n + 1) * 4));
  p.ws_total = (int32_t*)((uint8_t*)workspace + 2 * up256(((size_t)n + 1) * 4));
  p.ws_head = p.ws_total + kPagesThreads;
  p.n = n;
  p.B = s->batch;
  p.NB = s->num_blocks;
  p.MB = s->max_blocks_per_seq;
  p.bs_log2 = log2_of(s->block_size);
  p.num_free = num_free;
  return p;
}

// One launch of a cluster for few table entries and a small pool (one CTA up to 4096 entries, four a thread: a barrier of a cluster
// costs about as much as they do), a launch per phase on all SMs for more than 65536 (16 CTAs of 4 a thread: from there on the
// cluster's phases take longer than launches).  The host knows the width of the table, not the entries that are concerned: in a table of
// 32768 tokens (2048 entries a row) 6 short rows are given back in 16 us instead of 14, 33 in 31 instead of 18; 33 forks take 14
// us instead of 12 (events on both sides of a call, which add about 5).
template <typename K>
static int launch_pages(K kern, std::atomic<int>* done, int maps, int phases, PagesParams& p, cudaStream_t st, const char* where) {
  const size_t most = 3 * OOCO_MAX_PAGE_ROWS / 8, list = p.n <= kPagesListInSmem ? ((size_t)3 * p.n + 1) * 4 : 0;
  const size_t map = (size_t)maps * ((p.B + 31) / 32) * 4, smem = map > list ? map : list;
  int rc = configure((const void*)kern, done, (int)most), dev = 0;
  if (rc) return rc;
  const int64_t work = (int64_t)p.n * p.MB + p.NB / 4;
  if (work <= 65536) {
    int cluster = 1;
    while (cluster < kPagesMaxCluster && work > (int64_t)cluster * 4096) cluster *= 2;
    p.phase = -1;
    return finish(launch_clustered(kern, dim3(cluster), dim3(kPagesThreads), smem, st, pdl_enabled(), (unsigned)cluster, p), where);
  }
  if ((rc = current_device(&dev))) return rc;
  int grid = device_info(dev).sm_count;
  if (grid <= 0) return fail_cuda("cudaDeviceGetAttribute", -1);
  if (grid > kPagesThreads) grid = kPagesThreads;
  for (p.phase = 1; p.phase <= phases; ++p.phase)
    if ((rc = finish(launch_ex(kern, dim3(grid), dim3(kPagesThreads), smem, st, pdl_enabled(), p), where))) return rc;
  return OOCO_OK;
}

}  // namespace ooco

using namespace ooco;

extern "C" {

size_t ooco_pages_workspace_bytes(const ooco_shape_t* s, int32_t num_rows) {
  if (validate_shape(s) || num_rows < 0) return 0;
  return 2 * up256(((size_t)num_rows + 1) * 4) + up256((kPagesThreads + 1) * 4);
}

int ooco_fork_pages(const ooco_shape_t* s, int32_t n, const int32_t* parents, const int32_t* children,
                    const int32_t* shared_lens, int32_t* context_lens, int32_t* block_table, int32_t* blocks_held,
                    const int32_t* free_ids, int32_t num_free, int32_t* free_head, int32_t* shares,
                    int32_t* context_lens_out, int32_t* blocks_held_out, int32_t* free_head_out, int32_t* shares_out,
                    int32_t* copy_src, int32_t* copy_dst, int32_t* granted, void* workspace, size_t workspace_bytes,
                    int32_t* status, void* cuda_stream) {
  int rc = check_pages(s, n, num_free, workspace, workspace_bytes);
  if (rc) return rc;
  if (!context_lens || !block_table || !blocks_held || !free_head || !shares || (num_free > 0 && !free_ids) ||
      (n > 0 && (!parents || !children || !copy_src || !copy_dst || !granted)))
    return OOCO_E_NULLPTR;
  const size_t w = 4, rows = (size_t)s->batch * w, list = (size_t)n * w, pool = (size_t)s->num_blocks * w;
  // (an output that is the input itself is in place, and then counts as written only)
  const bool c_in = !context_lens_out || context_lens_out == context_lens, h_in = !blocks_held_out || blocks_held_out == blocks_held,
             f_in = !free_head_out || free_head_out == free_head, s_in = !shares_out || shares_out == shares;
  const Range in[] = {{parents, list}, {children, list}, {shared_lens, list}, {free_ids, num_free * w},
                      {c_in ? nullptr : context_lens, rows}, {h_in ? nullptr : blocks_held, rows},
                      {f_in ? nullptr : free_head, w}, {s_in ? nullptr : shares, pool}};
  const Range out[] = {{c_in ? context_lens : context_lens_out, rows}, {h_in ? blocks_held : blocks_held_out, rows},
                       {f_in ? free_head : free_head_out, w}, {s_in ? shares : shares_out, pool},
                       {block_table, rows * s->max_blocks_per_seq}, {copy_src, list}, {copy_dst, list}, {granted, list},
                       {workspace, ooco_pages_workspace_bytes(s, n)}, {status, w}};
  if (!disjoint(in, sizeof in / sizeof *in, out, sizeof out / sizeof *out)) return OOCO_E_SHAPE;
  PagesParams p = page_params(s, n, num_free, workspace);
  p.parents = parents;
  p.children = children;
  p.lens = shared_lens;
  p.context_lens = context_lens;
  p.blocks_held = blocks_held;
  p.free_head = free_head;
  p.shares = shares;
  p.block_table = block_table;
  p.free_ids = const_cast<int32_t*>(free_ids);
  p.context_lens_out = (int32_t*)out[0].p;
  p.blocks_held_out = (int32_t*)out[1].p;
  p.free_head_out = (int32_t*)out[2].p;
  p.shares_out = (int32_t*)out[3].p;
  p.copy_src = copy_src;
  p.copy_dst = copy_dst;
  p.granted = granted;
  p.status = status;
  static std::atomic<int> done[64];
  return launch_pages(fork_pages_kernel, done, 3, 2, p, (cudaStream_t)cuda_stream, "launch of the forking kernel");
}

int ooco_release_pages(const ooco_shape_t* s, int32_t n, const int32_t* rows_, const int32_t* keep_lens, int32_t* context_lens,
                       const int32_t* block_table, int32_t* blocks_held, int32_t* free_ids, int32_t num_free,
                       int32_t* free_head, int32_t* shares, int32_t* context_lens_out, int32_t* blocks_held_out,
                       int32_t* free_head_out, int32_t* shares_out, void* workspace, size_t workspace_bytes,
                       int32_t* status, void* cuda_stream) {
  int rc = check_pages(s, n, num_free, workspace, workspace_bytes);
  if (rc) return rc;
  if (!context_lens || !block_table || !blocks_held || !free_head || !shares || (num_free > 0 && !free_ids) || (n > 0 && !rows_))
    return OOCO_E_NULLPTR;
  const size_t w = 4, rows = (size_t)s->batch * w, list = (size_t)n * w, pool = (size_t)s->num_blocks * w;
  const bool c_in = !context_lens_out || context_lens_out == context_lens, h_in = !blocks_held_out || blocks_held_out == blocks_held,
             f_in = !free_head_out || free_head_out == free_head, s_in = !shares_out || shares_out == shares;
  const Range in[] = {{rows_, list}, {keep_lens, list}, {block_table, rows * s->max_blocks_per_seq},
                      {c_in ? nullptr : context_lens, rows}, {h_in ? nullptr : blocks_held, rows},
                      {f_in ? nullptr : free_head, w}, {s_in ? nullptr : shares, pool}};
  const Range out[] = {{c_in ? context_lens : context_lens_out, rows}, {h_in ? blocks_held : blocks_held_out, rows},
                       {f_in ? free_head : free_head_out, w}, {s_in ? shares : shares_out, pool}, {free_ids, num_free * w},
                       {workspace, ooco_pages_workspace_bytes(s, n)}, {status, w}};
  if (!disjoint(in, sizeof in / sizeof *in, out, sizeof out / sizeof *out)) return OOCO_E_SHAPE;
  PagesParams p = page_params(s, n, num_free, workspace);
  p.parents = rows_;
  p.lens = keep_lens;
  p.context_lens = context_lens;
  p.blocks_held = blocks_held;
  p.free_head = free_head;
  p.shares = shares;
  p.block_table = const_cast<int32_t*>(block_table);
  p.free_ids = free_ids;
  p.context_lens_out = (int32_t*)out[0].p;
  p.blocks_held_out = (int32_t*)out[1].p;
  p.free_head_out = (int32_t*)out[2].p;
  p.shares_out = (int32_t*)out[3].p;
  p.status = status;
  static std::atomic<int> done[64];
  return launch_pages(release_pages_kernel, done, 2, 5, p, (cudaStream_t)cuda_stream, "launch of the releasing kernel");
}

int ooco_norm_rope_kv_append(const ooco_shape_t* shape, const ooco_rope_t* rope, const ooco_head_norm_t* norm,
                             int32_t num_tokens, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                             const void* v, int64_t v_stride, const int32_t* positions, const int32_t* slot_map, void* q_out,
                             int64_t q_out_stride, void* k_cache, void* v_cache, void* cuda_stream) {
  if (!norm) return OOCO_E_NULLPTR;
  return rope_append(shape, rope, norm, num_tokens, q, q_stride, k, k_stride, v, v_stride, positions, slot_map, q_out,
                     q_out_stride, k_cache, v_cache, false, 1.f, 1.f, cuda_stream);
}

int ooco_norm_rope_kv_append_fp8(const ooco_shape_t* shape, const ooco_rope_t* rope, const ooco_head_norm_t* norm,
                                 int32_t num_tokens, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                                 const void* v, int64_t v_stride, const int32_t* positions, const int32_t* slot_map,
                                 void* q_out, int64_t q_out_stride, void* k_cache, void* v_cache, float k_scale,
                                 float v_scale, void* cuda_stream) {
  if (!norm) return OOCO_E_NULLPTR;
  return rope_append(shape, rope, norm, num_tokens, q, q_stride, k, k_stride, v, v_stride, positions, slot_map, q_out,
                     q_out_stride, k_cache, v_cache, true, k_scale, v_scale, cuda_stream);
}

int ooco_shape_logits(const ooco_logits_t* s, const void* logits, const float* temperature, const float* repetition,
                      const float* frequency, const float* presence, const int32_t* history, const int32_t* history_lens,
                      const int32_t* prompt_lens, const int32_t* tokens, const int32_t* parents, const int32_t* tree_sizes,
                      const int32_t* bias_tokens, const float* bias_values, const int32_t* mask, float* out_logits,
                      float* out_probs, void* cuda_stream) {
  if (!s) return OOCO_E_NULLPTR;
  if (s->batch <= 0 || s->max_nodes <= 0 || s->vocab <= 0 || (s->logits_fp32 != 0 && s->logits_fp32 != 1) ||
      s->history_width < 0 || s->max_bias < 0)
    return OOCO_E_SHAPE;
  if (s->batch > (1 << 24) || s->max_nodes > OOCO_TREE_MAX_NODES || s->vocab > OOCO_MAX_SHAPED_VOCAB || s->max_bias > OOCO_MAX_BIAS ||
      s->history_width > OOCO_MAX_HISTORY ||
      (int64_t)s->batch * s->max_nodes * kLogitsMaxCluster > INT32_MAX)
    return OOCO_E_UNSUPPORTED;
  const bool penalties = repetition || frequency || presence;
  if (!logits || (!out_logits && !out_probs)) return OOCO_E_NULLPTR;
  if (penalties && (!history_lens || (s->history_width > 0 && !history))) return OOCO_E_NULLPTR;
  if (!bias_tokens != !bias_values || (s->max_bias > 0 && !bias_tokens)) return OOCO_E_NULLPTR;
  const int64_t B = s->batch, N = s->max_nodes, V = s->vocab, cell = s->logits_fp32 ? 4 : 2;
  // rows of an output must not meet one another, whichever of the two dimensions is the outer one; masks may be shared
  auto nested = [&](int64_t outer, int64_t n_outer, int64_t inner, int64_t n_inner) {
    return (n_inner == 1 || inner >= V) && (n_outer == 1 || (n_inner == 1 ? outer >= V : (outer - V) / inner >= n_inner - 1));
  };
  auto rows_ok = [&](int64_t seq, int64_t node) {
    return seq >= 0 && node >= 0 && (nested(seq, B, node, N) || nested(node, N, seq, B));
  };
  if (s->logits_seq_stride < 0 || s->logits_node_stride < 0 || (mask && (s->mask_seq_stride < 0 || s->mask_node_stride < 0)) ||
      (out_logits && !rows_ok(s->out_seq_stride, s->out_node_stride)) ||
      (out_probs && !rows_ok(s->probs_seq_stride, s->probs_node_stride)))
    return OOCO_E_SHAPE;
  if (((uintptr_t)logits & (cell - 1)) || (((uintptr_t)out_logits | (uintptr_t)out_probs | (uintptr_t)mask) & 3)) return OOCO_E_UNSUPPORTED;
  {
    auto span = [&](int64_t seq, int64_t node, int64_t last, int64_t bytes) {
      return (size_t)(((B - 1) * seq + (N - 1) * node + last) * bytes);
    };
    const size_t lb = span(s->logits_seq_stride, s->logits_node_stride, V, cell), w = 4, b1 = (size_t)B * w;
    auto same = [&](const float* o, int64_t seq, int64_t node) {
      return (const void*)o == logits && s->logits_fp32 && (B == 1 || seq == s->logits_seq_stride) && (N == 1 || node == s->logits_node_stride);
    };
    const Range out[] = {{out_logits, span(s->out_seq_stride, s->out_node_stride, V, 4)},
                         {out_probs, span(s->probs_seq_stride, s->probs_node_stride, V, 4)}};
    if (overlap(out[0], out[1])) return OOCO_E_SHAPE;
    if (overlap(out[0], {logits, lb}) && !same(out_logits, s->out_seq_stride, s->out_node_stride)) return OOCO_E_SHAPE;
    if (overlap(out[1], {logits, lb}) && !same(out_probs, s->probs_seq_stride, s->probs_node_stride)) return OOCO_E_SHAPE;
    const Range in[] = {{temperature, b1}, {repetition, b1}, {frequency, b1}, {presence, b1}, {history, b1 * s->history_width},
                        {history_lens, b1}, {prompt_lens, b1}, {tokens, b1 * N}, {parents, b1 * N}, {tree_sizes, b1},
                        {bias_tokens, b1 * s->max_bias}, {bias_values, b1 * s->max_bias},
                        {mask, span(s->mask_seq_stride, s->mask_node_stride, (V + 31) / 32, 4)}};
    for (const Range& r : in)
      if (overlap(out[0], r) || overlap(out[1], r)) return OOCO_E_SHAPE;
  }
  int dev = 0, rc;
  if ((rc = current_device(&dev))) return rc;
  const int sms = device_info(dev).sm_count;
  if (sms <= 0) return fail_cuda("cudaDeviceGetAttribute", -1);
  LogitsParams p;
  memset(&p, 0, sizeof p);
  p.logits = logits;
  p.temperature = temperature;
  p.repetition = repetition;
  p.frequency = frequency;
  p.presence = presence;
  p.history = history;
  p.history_lens = history_lens;
  p.prompt_lens = prompt_lens;
  p.tokens = tokens;
  p.parents = parents;
  p.tree_sizes = tree_sizes;
  p.bias_tokens = bias_tokens;
  p.bias_values = bias_values;
  p.mask = (const uint32_t*)mask;
  p.out = out_logits;
  p.probs = out_probs;
  p.l_seq = s->logits_seq_stride;
  p.l_node = s->logits_node_stride;
  p.o_seq = s->out_seq_stride;
  p.o_node = s->out_node_stride;
  p.p_seq = s->probs_seq_stride;
  p.p_node = s->probs_node_stride;
  p.m_seq = s->mask_seq_stride;
  p.m_node = s->mask_node_stride;
  p.B = s->batch;
  p.N = s->max_nodes;
  p.V = s->vocab;
  p.L = s->history_width;
  p.M = s->max_bias;
  p.penalties = penalties;
  // CTAs per row: shares of at most 10240 tokens, so that three CTAs fit an SM (256 rows of 152064 tokens in trees of 16: 116 us; an
  // earlier form took 150, and 350 with shares of 20480), and more while the rows alone do not fill the SMs twice and shares of
  // more than 4096 tokens can be halved.  As many clusters as run at a time have equal parts of the rows: the text of a sequence is
  // counted once per part, and no cluster is left for a second wave (the same rows, a launch of 8 nodes per cluster: 133 us).
  const int64_t blocks = (V + kLogitsBlock - 1) / kLogitsBlock;
  int cluster = 1;
  while (cluster < kLogitsMaxCluster && (V > cluster * 10240ll || (B * N * cluster < 2ll * sms && V > cluster * 4096ll))) {
    cluster *= 2;
    ++p.cluster_log2;
  }
  p.share = (int)((blocks + cluster - 1) / cluster * kLogitsBlock);
  const bool half = s->history_width + N < 32768;
  const size_t smem = (size_t)p.share * 4 + (size_t)((p.M + 3) & ~3) * 8 + (penalties ? (size_t)p.share * (half ? 2 : 4) + N * ((N + 31) / 32) * 4 : 0);
  auto aligned = [&](const void* ptr, int64_t seq, int64_t node, int64_t bytes) {
    const int64_t rest = 4 * bytes - 1;
    return !ptr || (!((uintptr_t)ptr & rest) && (B == 1 || !(seq & 3)) && (N == 1 || !(node & 3)));
  };
  const bool wide = aligned(logits, s->logits_seq_stride, s->logits_node_stride, cell) &&
                    aligned(out_logits, s->out_seq_stride, s->out_node_stride, 4) &&
                    aligned(out_probs, s->probs_seq_stride, s->probs_node_stride, 4);
  static std::atomic<int> done[8][64];
  static std::atomic<uint64_t> resident_at[8];
  const int which = (s->logits_fp32 ? 4 : 0) + (wide ? 2 : 0) + (half ? 1 : 0);
  using K = void (*)(LogitsParams);
  static const K kernels[8] = {shape_logits_kernel<__nv_bfloat16, false, false>, shape_logits_kernel<__nv_bfloat16, false, true>,
                               shape_logits_kernel<__nv_bfloat16, true, false>, shape_logits_kernel<__nv_bfloat16, true, true>,
                               shape_logits_kernel<float, false, false>, shape_logits_kernel<float, false, true>,
                               shape_logits_kernel<float, true, false>, shape_logits_kernel<float, true, true>};
  // the most that any call takes: a share's values and whole-word counters, the biases, the ancestors of a full tree
  if ((rc = configure((const void*)kernels[which], done[which], OOCO_MAX_SHAPED_VOCAB / kLogitsMaxCluster * 8 + kLogitsMaxBias * 8 + 8192))) return rc;
  const int64_t resident = resident_clusters((const void*)kernels[which], resident_at[which], p.cluster_log2, smem, sms);
  const int64_t clusters = B * N < resident ? B * N : resident;
  return finish(launch_clustered(kernels[which], dim3((unsigned)(clusters * cluster)), dim3(kLogitsThreads), smem,
                                 (cudaStream_t)cuda_stream, pdl_enabled(), (unsigned)cluster, p),
                "launch of the logits kernel");
}

}  // extern "C"
