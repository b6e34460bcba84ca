// Host side of ooco_chunk_attention (ooco_batch.h): argument validation, tensor maps, launches.
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstring>

#include "../../include/ooco_batch.h"
#include "api_internal.h"
#include "packed_kernels.cuh"

namespace ooco {

static_assert(kPackedStatusRefused == OOCO_STATUS_REFUSED, "status bit");

struct PackedLayout {
  size_t off_tiles, off_items, off_merge, off_merge_first, off_lse, off_o, total;
  int max_tiles, max_items, max_merge, max_part_rows;
};

// Bounds that hold for any lengths.  A tile of s stages is cut into at most 2 s / L chunks, where L >= S / (CTAs x items per
// CTA), S the list's stages over all kv heads: 2 CTAs x items per CTA chunks (x heads) in all, of at most a tile's columns.
static PackedLayout packed_layout(const ooco_shape_t* s, int64_t num_rows, int64_t max_chunk, bool two_tiles) {
  const int64_t G = s->num_q_heads / s->num_kv_heads, cols = G * max_chunk;
  const int64_t cuts[2] = {2ll * kPackedGridCap * packed_items_per_cta(0), 2ll * kPackedGridCap * packed_items_per_cta(1)};
  const int64_t longest = ((int64_t)s->max_blocks_per_seq * s->block_size + kPackedMinStages * kTc2StageTok - 1) / (kPackedMinStages * kTc2StageTok);
  PackedLayout w;
  const int64_t tiles = s->batch + num_rows * G / kTcRows + 1;
  int64_t rows = cuts[0] * (cols < kTcRows ? cols : kTcRows);
  if (two_tiles && cols > kTcRows) rows += cuts[1] * kTc2Rows;
  const int64_t most = num_rows * s->num_q_heads * (longest + 1);  // every row in as many chunks as its context allows
  if (rows > most) rows = most;
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  w.max_tiles = (int)(tiles > INT32_MAX / 4 ? INT32_MAX / 4 : tiles);
  w.max_items = w.max_tiles + (int)(cuts[0] + cuts[1]);
  w.max_merge = (int)(tiles < cuts[0] + cuts[1] ? tiles : cuts[0] + cuts[1]);
  w.max_part_rows = (int)rows;
  w.off_tiles = sizeof(PackedHeader);
  w.off_items = w.off_tiles + up(((size_t)s->batch + 1) * 4);
  w.off_merge = w.off_items + up((size_t)w.max_items * 32);
  w.off_merge_first = w.off_merge + up((size_t)w.max_merge * 16);
  w.off_lse = w.off_merge_first + up(((size_t)w.max_merge + 1) * 4);
  w.off_o = w.off_lse + up((size_t)w.max_part_rows * 4);
  w.total = w.off_o + up((size_t)w.max_part_rows * s->head_dim * 4);
  return w;
}

template <int D, bool KV8, bool kOne>
static int launch_packed(const CUtensorMap& tk, const CUtensorMap& tv, const PackedParams& p, const DeviceInfo& di, int dev,
                         cudaStream_t st, bool dry) {
  auto kern = packed_tc_kernel<D, KV8, kOne>;
  const size_t smem = PackedSmem<D>::total();
  if (smem > (size_t)di.smem_optin) return OOCO_E_UNSUPPORTED;
  static std::atomic<int> configured[64];
  if (dev < 0 || dev >= 64 || !configured[dev].load()) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return fail_cuda("cudaFuncSetAttribute(max dynamic smem)", (long)e);
    if (dev >= 0 && dev < 64) configured[dev].store(1);
  }
  if (dry) return OOCO_OK;
  cudaError_t e = launch_ex(kern, dim3(p.grid), dim3(kTc2Threads), smem, st, pdl_enabled(), tk, tv, p);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? OOCO_OK : fail_cuda("launch of the packed attention kernel", (long)e);
}

static int check_rows(int64_t num_rows, int64_t max_chunk) {
  if (num_rows < 0 || max_chunk < 0 || max_chunk > num_rows) return OOCO_E_SHAPE;
  return OOCO_OK;
}

static int chunk_core(const ooco_shape_t* s, int32_t num_rows, int32_t max_chunk, const void* q, int64_t q_stride,
                      const void* k_cache, const void* v_cache, const int32_t* block_table, const int32_t* context_lens,
                      const int32_t* first_row, const int32_t* chunk_lens, float scale, bool kv8, float k_scale, float v_scale,
                      void* out, int64_t out_stride, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  int rc = validate_shape(s);
  if (rc) return rc;
  if ((rc = check_rows(num_rows, max_chunk))) return rc;
  if (!(scale > 0.f) || !(scale <= 3.0e38f)) return OOCO_E_SHAPE;
  if (kv8) {
    if (!(k_scale > 0.f) || !(v_scale > 0.f) || !(k_scale <= 3.0e38f) || !(v_scale <= 3.0e38f)) return OOCO_E_SHAPE;
    if (s->head_dim != 128 || ((s->kv_block_stride | s->kv_head_stride | s->kv_token_stride) & 15)) return OOCO_E_UNSUPPORTED;
  }
  const int64_t row = (int64_t)s->num_q_heads * s->head_dim, G = s->num_q_heads / s->num_kv_heads;
  if (G * num_rows > INT32_MAX / 2) return OOCO_E_UNSUPPORTED;
  if (!k_cache || !v_cache || !block_table || !context_lens || !first_row || !workspace) return OOCO_E_NULLPTR;
  if (num_rows > 0 && (!q || !out)) return OOCO_E_NULLPTR;
  if (q_stride < row || out_stride < row) return OOCO_E_SHAPE;
  if (((q_stride | out_stride) & 7) || (((uintptr_t)q | (uintptr_t)out | (uintptr_t)k_cache | (uintptr_t)v_cache) & 15))
    return OOCO_E_UNSUPPORTED;
  if (num_rows > 0 && rows_overlap(q, 2 * q_stride, 2 * row, out, 2 * out_stride, 2 * row, num_rows)) return OOCO_E_SHAPE;
  const bool two = !kv8;
  const PackedLayout w = packed_layout(s, num_rows, max_chunk, two);
  if (workspace_bytes < w.total || ((uintptr_t)workspace & 255)) return OOCO_E_WORKSPACE;
  if (num_rows == 0 || max_chunk == 0) return OOCO_OK;
  int dev = 0;
  if ((rc = current_device(&dev))) return rc;
  const DeviceInfo di = device_info(dev);
  if (di.sm_count <= 0) return OOCO_E_CUDA;
  uint8_t* ws = (uint8_t*)workspace;
  PackedParams p;
  memset(&p, 0, sizeof p);
  p.q = (const __nv_bfloat16*)q;
  p.out = (__nv_bfloat16*)out;
  p.block_table = block_table;
  p.context_lens = context_lens;
  p.first_row = first_row;
  p.chunk_lens = chunk_lens;
  p.hdr = (PackedHeader*)ws;
  p.tile_first = (int32_t*)(ws + w.off_tiles);
  p.items = (int4*)(ws + w.off_items);
  p.merge = (int4*)(ws + w.off_merge);
  p.merge_first = (int32_t*)(ws + w.off_merge_first);
  p.part_lse = (float*)(ws + w.off_lse);
  p.part_o = (float*)(ws + w.off_o);
  p.q_stride = q_stride;
  p.out_stride = out_stride;
  p.B = s->batch;
  p.Hq = s->num_q_heads;
  p.Hkv = s->num_kv_heads;
  p.G = (int)G;
  p.bs = s->block_size;
  p.MB = s->max_blocks_per_seq;
  p.NB = s->num_blocks;
  p.num_rows = num_rows;
  p.max_chunk = max_chunk;
  p.two_tiles = two && G * max_chunk > kTcRows;
  p.grid = di.sm_count < kPackedGridCap ? di.sm_count : kPackedGridCap;
  p.max_tiles = w.max_tiles;
  p.max_items = w.max_items;
  p.max_merge = w.max_merge;
  p.max_part_rows = w.max_part_rows;
  p.tile_rows = s->block_size < kTc2StageTok ? s->block_size : kTc2StageTok;
  p.scale_log2e = scale * 1.4426950408889634f * (kv8 ? k_scale * kE4m3WidenFactor : 1.f);
  p.v_scale = kv8 ? v_scale * kE4m3WidenFactor : 1.f;
  CUtensorMap tk, tv;
  if (kv8) {
    if ((rc = encode_kv8_map(&tk, s, k_cache, p.tile_rows)) || (rc = encode_kv8_map(&tv, s, v_cache, p.tile_rows))) return rc;
  } else {
    if ((rc = encode_kv_map(&tk, s, k_cache, p.tile_rows, false)) || (rc = encode_kv_map(&tv, s, v_cache, p.tile_rows, false)))
      return rc;
  }
  cudaStream_t st = (cudaStream_t)cuda_stream;
  auto attention = [&](bool dry) -> int {
    int r = OOCO_OK;
    if (p.two_tiles)
      r = s->head_dim == 128 ? launch_packed<128, false, false>(tk, tv, p, di, dev, st, dry)
                             : launch_packed<64, false, false>(tk, tv, p, di, dev, st, dry);
    if (r) return r;
    if (kv8) return launch_packed<128, true, true>(tk, tv, p, di, dev, st, dry);
    return s->head_dim == 128 ? launch_packed<128, false, true>(tk, tv, p, di, dev, st, dry)
                              : launch_packed<64, false, true>(tk, tv, p, di, dev, st, dry);
  };
  if ((rc = attention(true))) return rc;  // everything that can refuse the call, before the first launch
  const size_t first_bytes = ((size_t)p.B + 1) * 4;
  const int first_in_smem = first_bytes <= 32 * 1024;
  cudaError_t e = launch_ex(packed_plan_kernel, dim3(1), dim3(1024), first_in_smem ? first_bytes : 0, st, pdl_enabled(), p, first_in_smem);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) return fail_cuda("launch of the packed plan kernel", (long)e);
  if ((rc = attention(false))) return rc;
  int64_t blocks = ((int64_t)num_rows * p.Hq + 7) / 8;
  if (blocks > 8ll * di.sm_count) blocks = 8ll * di.sm_count;
  e = launch_ex(s->head_dim == 128 ? packed_merge_kernel<128> : packed_merge_kernel<64>, dim3((unsigned)blocks), dim3(256), 0, st,
                pdl_enabled(), p);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? OOCO_OK : fail_cuda("launch of the packed merge kernel", (long)e);
}

}  // namespace ooco

using namespace ooco;

extern "C" {

size_t ooco_chunk_workspace_bytes(const ooco_shape_t* s, int32_t num_rows, int32_t max_chunk) {
  if (validate_shape(s) || check_rows(num_rows, max_chunk) ||
      (int64_t)(s->num_q_heads / s->num_kv_heads) * num_rows > INT32_MAX / 2)
    return 0;
  return packed_layout(s, num_rows, max_chunk, true).total;
}

int ooco_chunk_attention(const ooco_shape_t* shape, int32_t num_rows, int32_t max_chunk, const void* q, int64_t q_stride,
                         const void* k_cache, const void* v_cache, const int32_t* block_table, const int32_t* context_lens,
                         const int32_t* first_row, const int32_t* chunk_lens, float scale, void* out, int64_t out_stride,
                         void* workspace, size_t workspace_bytes, void* cuda_stream) {
  return chunk_core(shape, num_rows, max_chunk, q, q_stride, k_cache, v_cache, block_table, context_lens, first_row, chunk_lens,
                    scale, false, 1.f, 1.f, out, out_stride, workspace, workspace_bytes, cuda_stream);
}

int ooco_chunk_attention_fp8(const ooco_shape_t* shape, int32_t num_rows, int32_t max_chunk, const void* q, int64_t q_stride,
                             const void* k_cache, const void* v_cache, const int32_t* block_table, const int32_t* context_lens,
                             const int32_t* first_row, const int32_t* chunk_lens, float scale, float k_scale, float v_scale,
                             void* out, int64_t out_stride, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  return chunk_core(shape, num_rows, max_chunk, q, q_stride, k_cache, v_cache, block_table, context_lens, first_row, chunk_lens,
                    scale, true, k_scale, v_scale, out, out_stride, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
