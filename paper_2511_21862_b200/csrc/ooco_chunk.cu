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

// Up to this many tokens by the table's width, and pairs per SM by max_chunk, a call is the one-tile kernel alone, whose CTAs then
// find their pairs by themselves: no plan, decode list or merge, but no cutting of long contexts either.  Measured, without and with
// a plan (1 to 8 new tokens): 4 sequences of 2 kv heads, up to 1024 or 2048 tokens 20 and 37, 28 and 41 us; 37 of 8 heads 37 and 65,
// 60 and 90 us; one new token: 28 and 30, 58 and 71 us.  Beyond: 4 sequences of up to 4096 tokens, one new 43 and 32 us; 74 of 8
// heads, 2048 tokens of an 8-bit cache 101 and 83 us.  The table's width decides, since the host does not know the contexts: 4 sequences
// of at most 256 tokens take 10 to 12 us in a table of 256 tokens, in one of 32768 29 (1 to 8 new tokens) and 20 us (one).
constexpr int64_t kDirectTokens = 2048, kDirectPairsPerSm = 2;

struct PackedLayout {
  size_t off_first, off_tiles, off_before[2], off_start[2], off_order[2], off_dec_first, off_dec_items, off_merge, off_lse, off_o, total;
  int max_tiles, max_merge, max_dec_chunks, max_part_rows, part_rows[2];
};

// CTAs an SM of the decode kernel, as the decode operators launch it.
static int decode_ctas_per_sm(int head_dim, bool kv8, int64_t G) { return kv8 ? (G > 8 ? 1 : 2) : (head_dim == 64 ? 4 : 2); }
// Which calls have a decode list: bf16 caches up to 8 heads a group (one MMA tile of columns), 8-bit ones all.
static bool has_decode(bool kv8, int64_t G) { return kv8 || G <= 8; }

// Bounds that hold for any lengths.  A decode of s stages is cut into at most s / L + 1 items, where L >= S / (CTAs x items per CTA),
// S the list's stages over all kv heads: (CTAs x items per CTA) / heads items beside one a sequence.  Of a tile list every CTA has at
// most two units whose rows are merged.
static PackedLayout packed_layout(const ooco_shape_t* s, int64_t num_rows, int64_t max_chunk) {
  const int64_t G = s->num_q_heads / s->num_kv_heads, cols = G * max_chunk;
  const int64_t longest = ((int64_t)s->max_blocks_per_seq * s->block_size + kPackedMinStages * kTc2StageTok - 1) / (kPackedMinStages * kTc2StageTok);
  PackedLayout w;
  const int64_t tiles = s->batch + num_rows * G / kTcRows + 1;
  const int64_t decodes = s->batch < num_rows ? s->batch : num_rows;
  int64_t chunks = decodes + 4ll * kPackedGridCap * kPackedDecodeItems / s->num_kv_heads + 1;
  if (chunks > decodes * (longest + 1)) chunks = decodes * (longest + 1);
  w.max_tiles = (int)tiles;
  w.max_merge = (int)decodes;
  w.max_dec_chunks = (int)chunks;
  w.part_rows[0] = (int)(chunks * s->num_q_heads);
  w.part_rows[1] = w.part_rows[0] + 2 * kPackedGridCap * kTcRows;
  w.max_part_rows = w.part_rows[1] + (cols > kTcRows ? 2 * kPackedGridCap * kTc2Rows : 0);
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  size_t at = sizeof(PackedHeader);
  auto put = [&](size_t bytes) {
    const size_t here = at;
    at += up(bytes);
    return here;
  };
  w.off_first = put(((size_t)s->batch + 1) * 4);
  w.off_tiles = put((size_t)w.max_tiles * sizeof(PackedTile));
  for (int k = 0; k < 2; ++k) {
    w.off_before[k] = put(((size_t)w.max_tiles + 1) * 8);
    w.off_start[k] = put((size_t)kPackedGridCap * 16);
    w.off_order[k] = put((size_t)w.max_tiles * 4);
  }
  w.off_dec_first = put(((size_t)s->batch + 1) * 4);
  w.off_dec_items = put((size_t)w.max_dec_chunks * s->num_kv_heads * 16);
  w.off_merge = put((size_t)w.max_merge * 16);
  w.off_lse = put((size_t)w.max_part_rows * 4);
  w.off_o = put((size_t)w.max_part_rows * s->head_dim * 4);
  w.total = at;
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

// The decode list: decode_main_kernel in the launch shape of the decode operators, one query token per sequence.
template <int D, int NCW, int NT, int KVM>
static int launch_decodes(const CUtensorMap& tk, const CUtensorMap& tv, DecodeParams& p, const DeviceInfo& di, int ctas_per_sm,
                          cudaStream_t st, int dev, bool dry) {
  using L = SmemLayout<D, NCW, NT, 1, KVM>;
  auto kern = decode_main_kernel<D, NCW, NT, 1, KVM, false, true>;
  const size_t budget = ((size_t)di.smem_optin + 1024) / ctas_per_sm - 1024;
  int nst = KVM == 2 ? 8 : 32;
  while (nst > 2 && L::total(nst, p.GQ) > budget) --nst;
  const size_t smem = L::total(nst, p.GQ);
  if (smem > (size_t)di.smem_optin) return OOCO_E_UNSUPPORTED;
  p.nstages = nst;
  static std::atomic<int> configured[64];
  if (dev < 0 || dev >= 64 || !configured[dev].load()) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, di.smem_optin);
    if (e != cudaSuccess) return fail_cuda("cudaFuncSetAttribute(max dynamic smem)", (long)e);
    if (dev >= 0 && dev < 64) configured[dev].store(1);
  }
  if (dry) return OOCO_OK;
  cudaError_t e = launch_ex(kern, dim3(p.next_item_init), dim3(L::kWarps * 32), smem, st, pdl_enabled(), tk, tv, p);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? OOCO_OK : fail_cuda("launch of the decode attention kernel", (long)e);
}

static int check_rows(const ooco_shape_t* s, int64_t num_rows, int64_t max_chunk) {
  if (num_rows < 0 || max_chunk < 0 || max_chunk > num_rows || (num_rows > 0 && max_chunk == 0)) return OOCO_E_SHAPE;
  // partial rows, tiles and columns are counted in 32 bits
  if (num_rows * (s->num_q_heads / s->num_kv_heads) > INT32_MAX / 4 || (int64_t)s->batch * s->num_q_heads > INT32_MAX / 4)
    return OOCO_E_UNSUPPORTED;
  return OOCO_OK;
}

static int chunk_core(const ooco_shape_t* s, int32_t num_rows, int32_t max_chunk, const void* q, int64_t q_stride,
                      const void* k_cache, const void* v_cache, const int32_t* block_table, const int32_t* context_lens,
                      const int32_t* first_row, const int32_t* chunk_lens, float scale, bool kv8, float k_scale, float v_scale,
                      void* out, int64_t out_stride, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  int rc = validate_shape(s);
  if (rc) return rc;
  if ((rc = check_rows(s, num_rows, max_chunk))) return rc;
  if (!(scale > 0.f) || !(scale <= 3.0e38f)) return OOCO_E_SHAPE;
  if (kv8) {
    if (!(k_scale > 0.f) || !(v_scale > 0.f) || !(k_scale <= 3.0e38f) || !(v_scale <= 3.0e38f)) return OOCO_E_SHAPE;
    if (s->head_dim != 128 || ((s->kv_block_stride | s->kv_head_stride | s->kv_token_stride) & 15)) return OOCO_E_UNSUPPORTED;
  }
  const int64_t row = (int64_t)s->num_q_heads * s->head_dim, G = s->num_q_heads / s->num_kv_heads;
  if (!k_cache || !v_cache || !block_table || !context_lens || !first_row || !workspace) return OOCO_E_NULLPTR;
  if (num_rows > 0 && (!q || !out)) return OOCO_E_NULLPTR;
  if (q_stride < row || out_stride < row) return OOCO_E_SHAPE;
  if (((q_stride | out_stride) & 7) || (((uintptr_t)q | (uintptr_t)out | (uintptr_t)k_cache | (uintptr_t)v_cache) & 15))
    return OOCO_E_UNSUPPORTED;
  if (num_rows > 0 && rows_overlap(q, 2 * q_stride, 2 * row, out, 2 * out_stride, 2 * row, num_rows)) return OOCO_E_SHAPE;
  const bool two = !kv8;
  const PackedLayout w = packed_layout(s, num_rows, max_chunk);
  if (workspace_bytes < w.total || ((uintptr_t)workspace & 255)) return OOCO_E_WORKSPACE;
  if (num_rows == 0) return OOCO_OK;
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
  p.tile_first = (int32_t*)(ws + w.off_first);
  p.tiles = (PackedTile*)(ws + w.off_tiles);
  for (int k = 0; k < 2; ++k) {
    p.before[k] = (int64_t*)(ws + w.off_before[k]);
    p.start[k] = (int4*)(ws + w.off_start[k]);
    p.order[k] = (int32_t*)(ws + w.off_order[k]);
    p.part_rows[k] = w.part_rows[k];
  }
  p.merge = (int4*)(ws + w.off_merge);
  p.part_lse = (float*)(ws + w.off_lse);
  p.part_o = (float*)(ws + w.off_o);
  p.q_stride = q_stride;
  p.out_stride = out_stride;
  p.B = s->batch;
  p.Hq = s->num_q_heads;
  p.Hkv = s->num_kv_heads;
  p.G = (int)G;
  p.D = s->head_dim;
  p.bs = s->block_size;
  p.MB = s->max_blocks_per_seq;
  p.NB = s->num_blocks;
  p.num_rows = num_rows;
  p.max_chunk = max_chunk;
  p.two_tiles = two && G * max_chunk > kTcRows;
  p.grid = di.sm_count < kPackedGridCap ? di.sm_count : kPackedGridCap;
  p.dec_first = (int32_t*)(ws + w.off_dec_first);
  p.dec_items = (int4*)(ws + w.off_dec_items);
  p.max_dec_chunks = w.max_dec_chunks;
  p.decode = has_decode(kv8, G);
  p.dec_grid = di.sm_count * decode_ctas_per_sm(s->head_dim, kv8, G);
  if (p.dec_grid > 4 * kPackedGridCap) p.dec_grid = 4 * kPackedGridCap;
  p.max_tiles = w.max_tiles;
  p.max_merge = w.max_merge;
  p.max_part_rows = w.max_part_rows;
  p.early = !kv8 && (p.decode || p.two_tiles);
  p.dec_stage_bytes = 2.f * kTc2StageTok * s->head_dim * (kv8 ? 1 : 2);
  p.tile_rows = s->block_size < kTc2StageTok ? s->block_size : kTc2StageTok;
  p.scale_log2e = scale * 1.4426950408889634f * (kv8 ? k_scale * kE4m3WidenFactor : 1.f);
  p.v_scale = kv8 ? v_scale * kE4m3WidenFactor : 1.f;
  const int64_t direct_tiles = (G * max_chunk + kTcRows - 1) / kTcRows;
  if ((int64_t)p.MB * p.bs <= kDirectTokens && direct_tiles * p.B * p.Hkv <= kDirectPairsPerSm * di.sm_count)
    p.direct_tiles = (int)direct_tiles;
  CUtensorMap tk, tv;
  if (kv8) {
    if ((rc = encode_kv8_map(&tk, s, k_cache, p.tile_rows)) || (rc = encode_kv8_map(&tv, s, v_cache, p.tile_rows))) return rc;
  } else {
    if ((rc = encode_kv_map(&tk, s, k_cache, p.tile_rows, false)) || (rc = encode_kv_map(&tv, s, v_cache, p.tile_rows, false)))
      return rc;
  }
  // the decode list's view of the same workspace; 128-byte boxes of at most a stage's tokens
  DecodeParams d;
  memset(&d, 0, sizeof d);
  const bool wide = kv8 && G > 8;
  const int dec_stage = kv8 ? 128 : 64;
  CUtensorMap dk, dv;
  if (p.decode) {
    d.q = p.q;
    d.out = p.out;
    d.block_table = block_table;
    d.context_lens = context_lens;
    d.hdr = &p.hdr->dec;
    d.items = p.dec_items;
    d.seq_first = p.dec_first;
    d.part_o = p.part_o;
    d.part_lse = p.part_lse;
    d.B = p.B;
    d.Hq = p.Hq;
    d.Hkv = p.Hkv;
    d.G = d.GQ = p.G;
    d.Sq = 1;
    d.D = s->head_dim;
    d.bs = p.bs;
    d.MB = p.MB;
    d.NB = p.NB;
    d.max_items = w.max_dec_chunks * p.Hkv;
    d.tile_rows = s->block_size < dec_stage ? s->block_size : dec_stage;
    d.next_item_init = p.dec_grid;
    d.first_row = first_row;
    d.q_stride = q_stride;
    d.out_stride = out_stride;
    d.early = p.two_tiles || (kv8 && max_chunk > 1);
    // (scores come from the codes' own values here: only V carries the widening factor)
    d.scale_log2e = scale * 1.4426950408889634f * k_scale;
    d.v_scale = p.v_scale;
    bool five_d = !kv8 && s->head_dim == 128 && encode_kv_map(&dk, s, k_cache, d.tile_rows, true) == OOCO_OK;
    d.split_halves = five_d ? 0 : 1;
    if (kv8)
      rc = encode_kv8_map(&dk, s, k_cache, d.tile_rows);
    else if (!five_d)
      rc = encode_kv_map(&dk, s, k_cache, d.tile_rows, false);
    if (!rc) rc = kv8 ? encode_kv8_map(&dv, s, v_cache, d.tile_rows) : encode_kv_map(&dv, s, v_cache, d.tile_rows, five_d);
    if (rc) return rc;
  }
  const int cps = decode_ctas_per_sm(s->head_dim, kv8, G);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (p.direct_tiles) {
    const int64_t pairs = direct_tiles * p.B * p.Hkv;
    p.early = 0;
    if (pairs < p.grid) p.grid = (int)pairs;
    if (kChecked) {  // any CTA may report before the first has written the status word
      const cudaError_t e = cudaMemsetAsync(&p.hdr->dec.status, 0, sizeof(p.hdr->dec.status), st);
      if (e != cudaSuccess) return fail_cuda("clearing the status word", (long)e);
    }
    return kv8 ? launch_packed<128, true, true>(tk, tv, p, di, dev, st, false)
               : (s->head_dim == 128 ? launch_packed<128, false, true>(tk, tv, p, di, dev, st, false)
                                     : launch_packed<64, false, true>(tk, tv, p, di, dev, st, false));
  }
  auto decodes = [&](bool dry) -> int {
    if (kv8) return wide ? launch_decodes<128, 8, 2, 2>(dk, dv, d, di, cps, st, dev, dry) : launch_decodes<128, 8, 1, 2>(dk, dv, d, di, cps, st, dev, dry);
    return s->head_dim == 128 ? launch_decodes<128, 4, 1, 0>(dk, dv, d, di, cps, st, dev, dry)
                              : launch_decodes<64, 4, 1, 0>(dk, dv, d, di, cps, st, dev, dry);
  };
  const bool tiles = !p.decode || max_chunk > 1;
  auto attention = [&](bool dry) -> int {
    int r = OOCO_OK;
    if (p.two_tiles)
      r = s->head_dim == 128 ? launch_packed<128, false, false>(tk, tv, p, di, dev, st, dry)
                             : launch_packed<64, false, false>(tk, tv, p, di, dev, st, dry);
    if (kv8) {
      if (tiles) r = launch_packed<128, true, true>(tk, tv, p, di, dev, st, dry);
      return r ? r : decodes(dry);
    }
    if (!r && p.decode) r = decodes(dry);
    if (r || !tiles) return r;
    return s->head_dim == 128 ? launch_packed<128, false, true>(tk, tv, p, di, dev, st, dry)
                              : launch_packed<64, false, true>(tk, tv, p, di, dev, st, dry);
  };
  if ((rc = attention(true))) return rc;  // everything that can refuse the call, before the first launch
  const size_t seq_bytes = (size_t)p.B * 20 + 4;
  const int in_smem = seq_bytes <= 26 * 1024;  // (with the static part under 48 KiB)
  cudaError_t e = launch_ex(packed_plan_kernel, dim3(1), dim3(1024), in_smem ? seq_bytes : 0, st, pdl_enabled(), p, in_smem);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) return fail_cuda("launch of the packed plan kernel", (long)e);
  if ((rc = attention(false))) return rc;
  e = launch_ex(s->head_dim == 128 ? packed_merge_kernel<128> : packed_merge_kernel<64>, dim3((unsigned)(4 * di.sm_count)), dim3(256), 0,
                st, pdl_enabled(), p);
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? OOCO_OK : fail_cuda("launch of the packed merge kernel", (long)e);
}

}  // namespace ooco

using namespace ooco;

extern "C" {

size_t ooco_chunk_workspace_bytes(const ooco_shape_t* s, int32_t num_rows, int32_t max_chunk) {
  if (validate_shape(s) || check_rows(s, num_rows, max_chunk)) return 0;
  return packed_layout(s, num_rows, max_chunk).total;
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
