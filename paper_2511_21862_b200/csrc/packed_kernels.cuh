// Attention of the new tokens of all sequences over the paged cache, rows packed: plan -> tiles on tcgen05 -> merge.
//
// The G n_b score columns (query x head of the group) of a (sequence, kv head) pair go, by their number, to one of three lists,
// each with a kernel of its own, because what bounds them differs:
//   decode_main_kernel               one query token (a decode): as the decode operators, HBM-bound
//   packed_tc_kernel<.., one tile>   else at most 128 columns: the cache is read once for few columns, HBM-bound.  The scores of a
//                                    stage run while the softmax threads still work on the stage before.
//   packed_tc_kernel<.., two tiles>  a piece of a prompt, tiles of 256 columns: two 128-row halves share every K / V slot and take
//                                    turns on the tensor pipe, tensor-bound
// How the CTAs of a tile kernel share the (tile, kv head) pairs of their list is the plan's choice.  Many or short pairs: the CTAs
// pull whole pairs, the longest first; what ends early leaves its SM to the decode kernel.  Few long ones (the longest is more than
// half of a CTA's share, or three quarters of it and the decodes' time together): all their stages (128 tokens) stand in a row,
// which is cut into as many pieces of equal length as there are CTAs; a pair that a cut goes through becomes two or more units,
// whose rows are merged, at most two of them per CTA.  Measured, pulled and cut: 16 or 4 pieces of 480 tokens of prompts beside 48
// or 60 decodes 432 and 481, 240 and 260 us; one piece of 1024 or 128 tokens of a prompt of 8192, 64 q heads 293 and 284, 164 and 86.
// Few pairs with short contexts (both known to the host) need none of this: the one-tile kernel alone finds its pairs by itself.
// The CTA is that of chunk_tc2_kernel (chunk_tc2_kernels.cuh), which has one number of query tokens for all sequences; there
// also stands why its MMAs, slots and warps are as they are.  What differs: a stage's meta words say all about its unit (rows,
// columns, partial rows), so that sequences of any lengths share a launch; head_dim 64 has half the slot, twice the slots and half
// the MMAs; an 8-bit cache runs every column on the one-tile kernel, which widens a stage for every 128 columns again (4 pieces of
// 2048 new tokens of prompts of 8192, 64 q heads: 2614 us, 1714 over a bf16 cache; 3784 with the kernel of two CTAs an SM that the
// operator of one number of query tokens runs there).  Decodes alone, 96 of 1024 to 32768 tokens: 6.6 TB/s with 4 or 8 heads a group,
// 6.4 with 10 or 16 on the one-tile kernel, 6.0 at head_dim 64; over the 8-bit cache 5.6 with 8 heads, 3.9 with 16.
#pragma once
#include <cstddef>

#include "chunk_tc2_kernels.cuh"
#include "cta_util.cuh"

namespace ooco {

constexpr int kPackedEnd = 1 << 18;          // flag of a stage's meta words: the end marker
constexpr int kPackedGridCap = 160;          // most CTAs of an attention kernel (bounds the workspace)
// Lists: 0 = one tile, 1 = two tiles, 2 = decodes.
constexpr int kPackedDecodeItems = 6;        // items of the decode list that the plan aims at per CTA
constexpr int kPackedMinStages = 2;          // shortest item: 256 tokens
// What a unit of a tile list costs beside its stages (its last products, writing its rows, the next one's queries), in stages: 64
// sequences of 480 new tokens, CTAs of 10 and of 150 units for 479 stages took 1050 and 1970 us.
constexpr int kPackedUnitCost = 3;
constexpr int kPackedMinPiece = 6;           // shortest piece of a tile list, in stages
__host__ __device__ constexpr int packed_tile(int list) { return list == 1 ? kTc2Rows : kTcRows; }  // columns of a tile
constexpr int kPackedStatusRefused = 128;

template <int D>
struct PackedSmem {
  static constexpr int NK = D == 128 ? kTc2KSlots : 4, NV = D == 128 ? kTc2VSlots : 6;  // (the meta ring is longer than either)
  static constexpr int kSlotBytes = (D / 64) * kTc2HalfBytes, kQBytes = (D / 64) * kTcRows * 128;
  __host__ __device__ static size_t total() {
    return 1024 + 2 * (size_t)kQBytes + (size_t)(NK + NV) * kSlotBytes + kTc2MetaRing * 48 + NV * sizeof(VStageDesc) + 512;
  }
};

struct PackedHeader {  // first bytes of the workspace
  WsHeader dec;          // status word; work units (item x kv head) of the decode list and the next one that no CTA has taken
  int32_t merge_rows;    // rows of the sequences of the decode list whose tokens are cut into several items
  int64_t stages[2];     // length of the tile lists' rows, over all kv heads
  int32_t pull[2];       // whether their CTAs pull whole pairs
  int32_t pairs[2];      // (tile, kv head) pairs of the lists, and the next one to be pulled
  int32_t next[2];
  int32_t pieces[2];     // else: pieces of the list's row of stages
  int32_t pad[50];
};
static_assert(sizeof(PackedHeader) == 512 && offsetof(PackedHeader, dec) == 0, "the status word leads the workspace");

struct alignas(16) PackedTile {
  int32_t b, c0, stages, first;  // sequence; first column; stages of 128 tokens that its last column sees (at least 1); first tile of
  int32_t r0, n, T, end;         // the sequence; first row of q, query tokens, context; end of the sequence's tiles
};
static_assert(sizeof(PackedTile) == 32, "two vectors");

struct PackedParams {
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  const int32_t *block_table, *context_lens, *first_row, *chunk_lens;
  PackedHeader* hdr;
  int32_t* tile_first;   // [B + 1] first tile of each sequence
  PackedTile* tiles;     // [max_tiles]
  int64_t* before[2];    // [max_tiles + 1] length of the list's row before each tile (one kv head)
  int4* start[2];        // [grid] where each piece of the list begins: {tile, kv head, place in the pair, -}
  int32_t* order[2];     // [max_tiles] the list's tiles, longest first (where pairs are pulled)
  int4* merge;           // [max_merge] decode list: {row of q, -, chunks, first partial row}
  float* part_o;         // [max_part_rows, D] normalised partial rows: the decode list's, then two units of every CTA for each tile list
  float* part_lse;       // [max_part_rows] log2-domain log-sum-exp of each
  int64_t q_stride, out_stride;
  int4* dec_items;       // [max_dec_chunks, Hkv] items of decode_main_kernel
  int32_t* dec_first;    // [B + 1] their chunks, counted over the sequences
  int32_t B, Hq, Hkv, G, D, bs, MB, NB, num_rows, max_chunk;
  int32_t two_tiles;     // 1: more than 128 columns go to the two-tile list
  int32_t decode;        // 1: sequences with one query token go to the decode list
  int32_t direct_tiles;  // > 0: no plan, no merge: the one-tile kernel alone, this many tiles for every sequence (some may be empty)
  int32_t early;         // one-tile kernel: it may start before the kernel in front of it has ended (see packed_plan_kernel)
  int32_t grid, dec_grid, max_tiles, max_merge, max_part_rows, max_dec_chunks, tile_rows;
  int32_t part_rows[2];  // first partial row of each tile list
  float scale_log2e, v_scale;
  float dec_stage_bytes; // K and V of 128 tokens of one kv head
};

// Columns of a tile, and tokens that the last of them sees.
__device__ __forceinline__ int packed_cols(const PackedParams& p, const PackedTile& t, int list) {
  return min(packed_tile(list), p.G * t.n - t.c0);
}
__device__ __forceinline__ int packed_seen(const PackedParams& p, const PackedTile& t, int list) {
  return min(t.T, max(0, t.T - t.n + 1 + (t.c0 + packed_cols(p, t, list) - 1) / p.G));
}
// A list's row: the stages of every pair behind kPackedUnitCost more for the pair itself, sequence by sequence, kv head by kv head,
// tile by tile (neighbours read the same K and V).  A cut in front of or inside the additional ones lies between two pairs.
// How many pieces the row is cut into (none shorter than kPackedMinPiece, unless it is the only one), and where piece k, which is
// CTA k's, begins.
__device__ __forceinline__ int packed_pieces(int64_t stages, int grid) {
  return (int)max((int64_t)1, min(stages / kPackedMinPiece, (int64_t)grid));
}
__device__ __forceinline__ int64_t packed_cut(int64_t stages, int k, int pieces) {
  return stages / pieces * k + stages % pieces * k / pieces;
}
// First partial row of a unit of CTA k: its pair begins in its piece (then it goes on in the next), or it began before.
__device__ __forceinline__ int packed_part(const PackedParams& p, int list, int k, bool begins) {
  return p.part_rows[list] + (2 * k + (begins ? 1 : 0)) * packed_tile(list);
}

// ------------------------------------------------------------------------------------ plan
struct PackedSeq {
  int r0, n, T;  // first row, query tokens, context
};
__device__ __forceinline__ PackedSeq packed_seq(const PackedParams& p, int b, bool* refused = nullptr) {
  PackedSeq s;
  s.r0 = p.first_row[b];
  long long n = (long long)p.first_row[b + 1] - s.r0;
  if (p.chunk_lens) n = min(n, (long long)p.chunk_lens[b]);
  if (s.r0 < 0 || n < 0) n = 0;
  n = min(n, (long long)p.num_rows - s.r0);
  if (n > p.max_chunk) {
    n = 0;
    if (refused) *refused = true;
  }
  s.n = n < 0 ? 0 : (int)n;
  const long long cap = (long long)p.MB * p.bs, t = p.context_lens[b];
  s.T = (int)(t < 0 ? 0 : (t > cap ? cap : t));
  return s;
}
__device__ __forceinline__ int packed_list(const PackedParams& p, const PackedSeq& s) {
  if (p.decode && s.n == 1) return 2;
  return p.two_tiles && p.G * s.n > kTcRows ? 1 : 0;
}

// One CTA.  Tiles of all sequences in their order, the stages before each (one sum for each tile list), the tile with which every
// CTA's piece begins; and the decode list: items of near-equal length, longest first, so that its dynamic schedule ends evenly.
// Latency-bound: a few block-wide scans; up to 1024 tiles are kept by the threads.
// The kernels behind the plan run side by side where SMs are free: each waits for the plan only, in that it can start only when all
// CTAs of the one in front of it have waited (for the plan), and ends by waiting for the end of that one.
__global__ void __launch_bounds__(1024) packed_plan_kernel(const PackedParams p, const int in_smem) {
  extern __shared__ int4 s_seq[];   // when they fit: [B] first row, query tokens, context, then [B + 1] first tile
  __shared__ long long s_warp[32], s_sum;
  __shared__ long long s_before[2][1025];
  __shared__ int s_hist[1024], s_most[4], s_share;
  __shared__ unsigned long long s_best;
  __shared__ float s_beside;  // what the decodes take, in stages of the two-tile kernel
  const int tid = threadIdx.x;
  grid_dep_wait();
  grid_dep_launch();
  int* first = in_smem ? reinterpret_cast<int*>(s_seq + p.B) : p.tile_first;
  auto seq = [&](int b) {
    if (!in_smem) return packed_seq(p, b);
    const int4 v = s_seq[b];
    return PackedSeq{v.x, v.y, v.z};
  };
  s_hist[tid] = 0;
  if (tid == 0) s_sum = 0, s_best = ~0ull;
  bool refused = false, decodes = false;
  long long tiles = 0;
  for (int b0 = 0; b0 < p.B; b0 += 1024) {
    const int b = b0 + tid;
    long long nt = 0, total;
    if (b < p.B) {
      const PackedSeq q = packed_seq(p, b, &refused);
      if (in_smem) s_seq[b] = make_int4(q.r0, q.n, q.T, 0);
      const int list = packed_list(p, q), per = packed_tile(list);
      if (q.T > 0) nt = ((long long)p.G * q.n + per - 1) / per;  // (without a context: zeros, below)
      decodes |= list == 2 && nt > 0;
    }
    const long long upto = tiles + block_scan(nt, s_warp, &total);
    if (b < p.B) first[b] = (int)min(upto - nt, (long long)INT32_MAX);
    tiles += total;
  }
  const bool overflow = tiles > p.max_tiles;  // (rows that overlap)
  const int NT = overflow ? 0 : (int)tiles;
  if (tid == 0) first[p.B] = NT;
  refused = __syncthreads_or(refused);
  decodes = __syncthreads_or(decodes);
  auto tile_of = [&](int i, int& list) {
    int lo = 0, hi = p.B;  // largest b with first[b] <= i
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= i) lo = mid; else hi = mid;
    }
    const PackedSeq q = seq(lo);
    list = packed_list(p, q);
    const int per = packed_tile(list);
    PackedTile t;
    t.b = lo;
    t.c0 = (i - first[lo]) * per;
    t.first = first[lo];
    t.end = first[lo + 1];
    t.r0 = q.r0;
    t.n = q.n;
    t.T = q.T;
    t.stages = max(1, (packed_seen(p, t, list) + kTc2StageTok - 1) / kTc2StageTok);
    return t;
  };
  const bool single = NT <= 1024;
  PackedTile kept = {};
  int kept_list = -1;
  if (single && tid < NT) kept = tile_of(tid, kept_list);
  auto tile_at = [&](int i, int& list) {
    if (!single) return tile_of(i, list);
    list = kept_list;
    return kept;
  };
  // ---- tile lists
  long long sums[2] = {0, 0};
  long long dec_sum = 0;
  int longest_tile[2] = {0, 0}, list_tiles[2] = {0, 0};
  for (int i0 = 0; i0 < NT; i0 += 1024) {
    const int i = i0 + tid;
    int list = -1;
    PackedTile t = {};
    if (i < NT) t = tile_at(i, list);
    if (list == 2) dec_sum += t.stages;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k == 1 && !p.two_tiles) continue;
      const long long v = list == k ? t.stages + kPackedUnitCost : 0;
      long long total;
      const long long at = sums[k] + block_scan(v, s_warp, &total) - v;
      sums[k] += total;
      if (i < NT) {
        p.before[k][i] = at;
        if (single) s_before[k][i] = at;
      }
    }
    if (i < NT && list != 2) p.tiles[i] = t;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (list == k) {
        longest_tile[k] = max(longest_tile[k], t.stages);
        ++list_tiles[k];
      }
  }
  if (tid < 4) s_most[tid] = 0;
  if (tid == 0)
    for (int k = 0; k < 2; ++k) {
      p.hdr->stages[k] = sums[k] * p.Hkv;
      p.before[k][NT] = sums[k];
      if (single) s_before[k][NT] = sums[k];
    }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (list_tiles[k]) {
      atomicMax(&s_most[k], longest_tile[k]);
      atomicAdd(&s_most[2 + k], list_tiles[k]);
    }
  __syncthreads();
  auto bucket = [](int len) { return 1023 - min(len, 1023); };
  // s_hist (numbers of things of a bucket) becomes the first place of each bucket; the user clears it for the next
  auto places = [&] {
    __syncthreads();
    long long all;
    const int mine = s_hist[tid];
    const long long before = block_scan(mine, s_warp, &all) - mine;
    s_hist[tid] = (int)before;
    __syncthreads();
  };
  if (decodes) {
    for (int o = 16; o; o >>= 1) dec_sum += __shfl_xor_sync(0xffffffffu, dec_sum, o);
    if ((tid & 31) == 0 && dec_sum) atomicAdd((unsigned long long*)&s_sum, (unsigned long long)dec_sum);
    __syncthreads();
    // Pieces of prompts beside decodes: the first are bound by the tensor pipe, the others by HBM, which fewer SMs can keep busy.  So
    // the two-tile kernel leaves some SMs to the decode kernel, which starts there at once: the number that lets both end soonest,
    // by the time of a stage on an SM and the rates of HBM and of an SM's decodes (bytes a us).  (Over the 8-bit cache both kernels
    // are bound by the SMs: 445 us one behind the other, 495 side by side.)
    constexpr float kHbm = 6.9e6f, kSm = 75e3f;
    const float stage_us = p.D == 128 ? 2.3f : 1.5f, bytes = (float)s_sum * p.Hkv * p.dec_stage_bytes;
    if (sums[1] > 0 && tid < p.grid) {
      const int c = tid + 1, rest = p.grid - c;
      const float two = (float)sums[1] * p.Hkv * stage_us / c;
      const float t = rest ? fmaxf(two, fmaxf(bytes / kHbm, bytes / (kSm * rest))) : two + bytes / kHbm;
      atomicMin((unsigned long long*)&s_best, (unsigned long long)__float_as_uint(t) << 32 | c);
    }
    __syncthreads();
    if (tid == 0) s_share = sums[1] > 0 ? (int)(s_best & 0xffffffff) : p.grid, s_beside = bytes / kHbm / stage_us;
    __syncthreads();
  }
  for (int k = 0; k < 2; ++k) {
    const float share = (float)sums[k] * p.Hkv / p.grid, longest = (float)(s_most[k] + kPackedUnitCost);
    const bool pull = k == 1 && decodes ? longest <= 0.75f * (share + s_beside) : longest <= 0.5f * share;
    if (tid == 0) {
      p.hdr->pull[k] = pull;
      p.hdr->pairs[k] = s_most[2 + k] * p.Hkv;
      p.hdr->next[k] = p.grid;
    }
    if (sums[k] == 0) continue;
    if (pull) {
      for (int i = tid; i < NT; i += 1024) {
        int list;
        const PackedTile t = tile_at(i, list);
        if (list == k) atomicAdd(&s_hist[bucket(t.stages)], 1);
      }
      places();
      for (int i = tid; i < NT; i += 1024) {
        int list;
        const PackedTile t = tile_at(i, list);
        if (list == k) p.order[k][atomicAdd(&s_hist[bucket(t.stages)], 1)] = i;
      }
      __syncthreads();
      s_hist[tid] = 0;
      __syncthreads();
      continue;
    }
    auto before = [&](int i) { return single ? s_before[k][i] : p.before[k][i]; };
    const int pieces = packed_pieces(sums[k] * p.Hkv, k == 1 && decodes ? s_share : p.grid);
    if (tid == 0) p.hdr->pieces[k] = pieces;
    for (int c = tid; c < pieces; c += 1024) {
      const long long x = packed_cut(sums[k] * p.Hkv, c, pieces);
      int lo = 0, hi = p.B;  // the sequence: largest b whose stages before it, of all heads, are no more than x
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before(first[mid]) * p.Hkv <= x) lo = mid; else hi = mid;
      }
      const int t0 = first[lo], t1 = first[lo + 1];
      const long long base = before(t0), per_head = before(t1) - base, rest = x - base * p.Hkv;
      const int h = (int)(rest / per_head);
      const long long at = base + rest - h * per_head;
      lo = t0;
      hi = t1;  // the tile
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before(mid) <= at) lo = mid; else hi = mid;
      }
      p.start[k][c] = make_int4(lo, h, (int)(at - before(lo)), 0);
    }
  }
  // ---- decode list
  int merge_rows = 0, n_items = 0;
  bool dec_overflow = false;
  if (decodes) {
    const long long ctas = (long long)p.dec_grid * kPackedDecodeItems;
    const int longest = max(kPackedMinStages, (int)((s_sum * p.Hkv + ctas - 1) / ctas));
    auto cut = [&](int stages, int& nch, int& len) {  // chunks of `len` stages each but the last
      nch = (stages + longest - 1) / longest;
      len = (stages + nch - 1) / nch;
      nch = (stages + len - 1) / len;
    };
    long long run = 0, kept_at = 0;  // (chunks << 32 | sequences in several chunks) so far
    auto visit = [&](bool again, auto f) {
      run = 0;
      for (int i0 = 0; i0 < NT; i0 += 1024) {
        const int i = i0 + tid;
        int list = -1, nch = 0, len = 1;
        PackedTile t = {};
        if (i < NT) t = tile_at(i, list);
        if (list == 2) cut(t.stages, nch, len);
        long long at = kept_at;
        if (!(again && single)) {
          const long long v = list == 2 ? ((long long)nch << 32) | (nch > 1 ? 1 : 0) : 0;
          long long total;
          at = run + block_scan(v, s_warp, &total) - v;
          run += total;
          kept_at = at;
        }
        if (list == 2) f(t, nch, len, (int)(at >> 32), (int)(at & 0xffffffff));
      }
    };
    visit(false, [&](const PackedTile& t, int nch, int len, int chunk, int m) {
      p.dec_first[t.b] = chunk;
      p.dec_first[t.b + 1] = chunk + nch;  // (what the next sequence writes there, if it is one of the list)
      atomicAdd(&s_hist[bucket(len)], nch - 1);
      atomicAdd(&s_hist[bucket(t.stages - (nch - 1) * len)], 1);
      if (nch > 1 && m < p.max_merge) p.merge[m] = make_int4(t.r0, 0, nch, chunk * p.Hq);
    });
    // Rows that several sequences claim: more chunks, or more sequences in several, than the workspace was sized for by the rows.
    // Partial rows would lie behind its end, so the list is dropped as a whole, as too many tiles are.
    const int cut_sequences = (int)(run & 0xffffffff);
    dec_overflow = run >> 32 > p.max_dec_chunks || cut_sequences > p.max_merge;
    if (!dec_overflow) {
      n_items = (int)(run >> 32);
      merge_rows = cut_sequences * p.Hq;
      places();
    }
    if (!dec_overflow) visit(true, [&](const PackedTile& t, int nch, int len, int chunk, int) {
      for (int c = 0; c < nch; ++c) {
        const int at = atomicAdd(&s_hist[bucket(min(len, t.stages - c * len))], 1);
        if (!checked(chk_index(at, p.max_dec_chunks), &p.hdr->dec.status, kStatusBadIndex)) continue;
        const int t0 = c * len * kTc2StageTok;
        for (int h = 0; h < p.Hkv; ++h)
          p.dec_items[(size_t)at * p.Hkv + h] = make_int4(t.b, (chunk + c) * p.Hkv + h, t0, min(t.T, t0 + len * kTc2StageTok));
      }
    });
  }
  if (tid == 0) {
    p.hdr->dec.status = (overflow || dec_overflow ? kStatusPlanOverflow : 0) | (refused ? kPackedStatusRefused : 0);
    p.hdr->dec.n_items = n_items * p.Hkv;
    p.hdr->dec.next_item = p.dec_grid;
    p.hdr->merge_rows = merge_rows;
  }
  for (int b = tid >> 5; b < p.B; b += 32) {  // query tokens of a sequence without a context
    const PackedSeq q = seq(b);
    if (q.T > 0) continue;
    const int vecs = p.Hq * p.D / 8;
    for (long long i = tid & 31; i < (long long)q.n * vecs; i += 32)
      *reinterpret_cast<uint4*>(p.out + (q.r0 + i / vecs) * p.out_stride + 8 * (i % vecs)) = make_uint4(0u, 0u, 0u, 0u);
  }
}

// ------------------------------------------------------------------------------------ merge
// One warp per row (a column of a (tile, kv head) pair): the partial rows, normalised, are averaged with the weights of their
// log-sum-exps, in the order of the tokens.  part(c) = partial row of piece c.
template <int D, typename F>
__device__ __forceinline__ void merge_row(const PackedParams& p, int pieces, F part, __nv_bfloat16* dst) {
  constexpr int V = D / 32;  // dims per lane
  const int lane = threadIdx.x & 31;
  float M = -INFINITY, den = 0.f, acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  for (int c0 = 0; c0 < pieces; c0 += 32) {
    const int cnt = min(32, pieces - c0);
    const float lse = lane < cnt ? p.part_lse[part(c0 + lane)] : -INFINITY;
    float gm = lse;
#pragma unroll
    for (int o = 16; o; o >>= 1) gm = fmaxf(gm, __shfl_xor_sync(0xffffffffu, gm, o));
    const float Mn = fmaxf(M, gm), Ms = Mn == -INFINITY ? 0.f : Mn;
    const float resc = exp2f(M - Ms), w_lane = exp2f(lse - Ms);
    M = Mn;
    float ws = w_lane;
#pragma unroll
    for (int o = 16; o; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
    den = den * resc + ws;
#pragma unroll
    for (int i = 0; i < V; ++i) acc[i] *= resc;
#pragma unroll 8
    for (int j = 0; j < cnt; ++j) {
      const float w = __shfl_sync(0xffffffffu, w_lane, j);
      const float* o = p.part_o + (int64_t)part(c0 + j) * D + lane * V;
      if (V == 4) {
        const float4 x = *reinterpret_cast<const float4*>(o);
        acc[0] += w * x.x; acc[1] += w * x.y; acc[V - 2] += w * x.z; acc[V - 1] += w * x.w;
      } else {
        const float2 x = *reinterpret_cast<const float2*>(o);
        acc[0] += w * x.x; acc[V - 1] += w * x.y;
      }
    }
  }
  const float inv = den > 0.f ? 1.f / den : 0.f;
#pragma unroll
  for (int i = 0; i < V; i += 2) *reinterpret_cast<uint32_t*>(dst + lane * V + i) = pack_bf16x2(acc[i] * inv, acc[i + 1] * inv);
}

// The same for `kRows` neighbouring columns in two pieces, the usual case of a pair that was cut: all their loads in flight together.
// first, second = partial rows of the first column; row(c) = where column c goes, for c < n.
template <int D, int kRows, typename F>
__device__ __forceinline__ void merge_pairs(const PackedParams& p, int first, int second, int n, F row) {
  constexpr int V = D / 32;
  const int lane = threadIdx.x & 31;
  float a[kRows], b[kRows], x[kRows][V], y[kRows][V];
#pragma unroll
  for (int c = 0; c < kRows; ++c) {
    a[c] = b[c] = -INFINITY;
    if (c >= n) continue;
    a[c] = p.part_lse[first + c];
    b[c] = p.part_lse[second + c];
    const float* u = p.part_o + (int64_t)(first + c) * D + lane * V;
    const float* w = p.part_o + (int64_t)(second + c) * D + lane * V;
#pragma unroll
    for (int i = 0; i < V; i += 2) {
      *reinterpret_cast<float2*>(&x[c][i]) = *reinterpret_cast<const float2*>(u + i);
      *reinterpret_cast<float2*>(&y[c][i]) = *reinterpret_cast<const float2*>(w + i);
    }
  }
#pragma unroll
  for (int c = 0; c < kRows; ++c) {
    if (c >= n) continue;
    const float M = fmaxf(a[c], b[c]), Ms = M == -INFINITY ? 0.f : M;
    const float wa = exp2f(a[c] - Ms), wb = exp2f(b[c] - Ms), den = wa + wb, inv = den > 0.f ? 1.f / den : 0.f;
    __nv_bfloat16* dst = row(c);
#pragma unroll
    for (int i = 0; i < V; i += 2)
      *reinterpret_cast<uint32_t*>(dst + lane * V + i) =
          pack_bf16x2((wa * x[c][i] + wb * y[c][i]) * inv, (wa * x[c][i + 1] + wb * y[c][i + 1]) * inv);
  }
}

constexpr int kMergeRows = 4;  // neighbouring columns of a pair that a warp merges at a time

// A warp's units of work: for each tile list that was cut into pieces, each cut and each group of kMergeRows columns (those of the
// pair that the cut goes through, if it is the pair's first); then the rows of the decode list.
template <int D>
__global__ void __launch_bounds__(256) packed_merge_kernel(const PackedParams p) {
  grid_dep_launch();
  grid_dep_wait();
  const int warps = gridDim.x * 8, me = blockIdx.x * 8 + (threadIdx.x >> 5);
  for (int list = 0; list < 2; ++list) {
    const int64_t stages = p.hdr->stages[list];
    if (stages == 0 || p.hdr->pull[list]) continue;
    const int pieces = p.hdr->pieces[list], groups = packed_tile(list) / kMergeRows;
    for (int u = me; u < (pieces - 1) * groups; u += warps) {
      const int k = 1 + u / groups, col0 = u % groups * kMergeRows;
      const int4 at = p.start[list][k];
      if (at.z <= kPackedUnitCost) continue;  // between two pairs
      const PackedTile t = p.tiles[at.x];
      const int h = at.y, cols = packed_cols(p, t, list);
      const int64_t begin = packed_cut(stages, k, pieces) - at.z + kPackedUnitCost, end = begin + t.stages;
      if (col0 >= cols || packed_cut(stages, k - 1, pieces) > begin) continue;  // (not the pair's first cut)
      int last = k;  // the piece that holds the pair's last stage
      while (last + 1 < pieces && packed_cut(stages, last + 1, pieces) < end) ++last;
      auto row = [&](int c) {
        const int column = t.c0 + col0 + c;
        return p.out + (int64_t)(t.r0 + column / p.G) * p.out_stride + (int64_t)(h * p.G + column % p.G) * D;
      };
      const int n = min(kMergeRows, cols - col0);
      if (last == k)
        merge_pairs<D, kMergeRows>(p, packed_part(p, list, k - 1, true) + col0, packed_part(p, list, k, false) + col0, n, row);
      else
        for (int c = 0; c < n; ++c)
          merge_row<D>(p, last - k + 2, [&](int i) { return packed_part(p, list, k - 1 + i, i == 0) + col0 + c; }, row(c));
    }
  }
  const int rows = p.hdr->merge_rows;
  for (int r = me; r < rows; r += warps) {
    const int4 m = p.merge[r / p.Hq];
    const int hq = r % p.Hq;
    if (!checked(chk_index((long long)m.w + (long long)m.z * p.Hq - 1, p.max_part_rows), &p.hdr->dec.status, kStatusBadIndex)) continue;
    merge_row<D>(p, m.z, [&](int c) { return m.w + c * p.Hq + hq; }, p.out + (int64_t)m.x * p.out_stride + (int64_t)hq * D);
  }
}

// ------------------------------------------------------------------------------------ tiles
// Barriers: stage number n (counted over the whole kernel, bookkeeping stages and the end marker included) uses K slot n % NK,
// V slot n % NV, meta entry n % 8 and, for each tile, barrier n & 1 of the pairs [2] below with phase parity (n >> 1) & 1;
// every tile takes a turn of its barriers on every stage, with or without work.  The meta ring is longer than the slots that a
// stage must find free, so an entry is rewritten only after all readers of its stage.
template <int D, bool KV8, bool kOne>
__global__ void __launch_bounds__(kTc2Threads, 1)
packed_tc_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                 const PackedParams p) {
  using L = PackedSmem<D>;
  constexpr int NH = D / 64;                               // 64-dim halves of a row
  constexpr int NK = L::NK, NV = KV8 ? 2 : L::NV, NM = kTc2MetaRing;
  constexpr int kSlotBytes = L::kSlotBytes, kQBytes = L::kQBytes;
  constexpr int kWarpK = 16, kWarpV = 17, kWarpM = 18;  // warps 0 .. 15: softmax; 18, 19: MMA of tile 0, 1
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - raw);
  const uint32_t s_q = base;                                       // [2] Q tiles
  const uint32_t s_k = s_q + 2u * kQBytes;                      // [NK] K slots
  const uint32_t s_v = s_k + (uint32_t)NK * kSlotBytes;         // [NV] V slots
  const uint32_t s_rk = s_q + kQBytes;                          // KV8: [NK] 8-bit K slots (tile 1's Q region)
  const uint32_t s_rv = s_v + (uint32_t)NV * kSlotBytes;        // KV8: [NV] 8-bit V slots (the third V slot's place)
  const uint32_t s_meta = s_v + (uint32_t)L::NV * kSlotBytes;  // [NM] three int4 per stage
  const uint32_t s_vdesc = s_meta + (uint32_t)NM * 48;             // [NV] VStageDesc
  const uint32_t s_bar = s_vdesc + (uint32_t)L::NV * sizeof(VStageDesc);
  const uint32_t s_kfull = s_bar;                  // [NK] the K slot has landed                          (TMA)
  const uint32_t s_kempty = s_kfull + NK * 8;      // [NK] the score MMAs that read it are complete       (MMA commit)
  const uint32_t s_vfull = s_kempty + NK * 8;      // [NV] the V slot has landed                          (TMA)
  const uint32_t s_vempty = s_vfull + NV * 8;      // [NV] the P.V MMAs that read it are complete         (MMA commit)
  const uint32_t s_vdfull = s_vempty + NV * 8;     // [NV] the stage's V descriptor is posted             (K producer)
  const uint32_t s_mfull = s_vdfull + NV * 8;      // [NM] the stage's meta words are posted              (K producer)
  const uint32_t s_sready = s_mfull + NM * 8;      // [2 tiles][2] S_t holds the stage's scores            (MMA commit)
  const uint32_t s_pready = s_sready + 32;         // [2 tiles][2] P_t written, O_t rescaled, V rows clean (256 threads)
  const uint32_t s_pvdone = s_pready + 32;         // [2 tiles] the unit's last P.V_t is complete          (MMA commit)
  const uint32_t s_qready = s_pvdone + 16;         // [2 tiles] Q_t of the unit is in shared memory        (256 threads)
  const uint32_t s_pvstage = s_qready + 16;       // [2] one-tile mode: the stage's P.V is complete              (MMA commit)
  const uint32_t s_rkfull = s_pvstage + 16;       // KV8 [NK] the 8-bit K slot has landed                         (TMA)
  const uint32_t s_rkempty = s_rkfull + 16;       // KV8 [NK] the 8-bit K slot has been widened                   (256 threads)
  const uint32_t s_rvfull = s_rkempty + 16;       // KV8 [NV] the 8-bit V slot has landed                         (TMA)
  const uint32_t s_rvempty = s_rvfull + 16;       // KV8 [NV] the 8-bit V slot has been widened                   (256 threads)
  const uint32_t s_drain = s_rvempty + 16;
  const uint32_t s_slot = s_drain + 16;
  int4* g_meta = reinterpret_cast<int4*>(gen + (s_meta - base));
  VStageDesc* g_vdesc = reinterpret_cast<VStageDesc*>(gen + (s_vdesc - base));
  volatile uint32_t* g_slot = reinterpret_cast<volatile uint32_t*>(gen + (s_slot - base));
  volatile int* s_abort = reinterpret_cast<volatile int*>(gen + (s_slot + 4 - base));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // (known to be uniform)

  if (threadIdx.x == 0) {
    *s_abort = 0;
    for (int i = 0; i < NK; ++i) {
      mbar_init(s_kfull + 8 * i, KV8 ? 256 : 1);  // (KV8: filled by the widening threads, not by TMA)
      mbar_init(s_kempty + 8 * i, kOne ? 1 : 2);  // one arrival per MMA warp that reads K
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_rkfull + 8 * i, 1);
      mbar_init(s_rkempty + 8 * i, 256);
      mbar_init(s_rvfull + 8 * i, 1);
      mbar_init(s_rvempty + 8 * i, 256);
    }
    for (int i = 0; i < NV; ++i) {
      mbar_init(s_vfull + 8 * i, KV8 ? 256 : 1);
      mbar_init(s_vempty + 8 * i, kOne ? 1 : 2);
      mbar_init(s_vdfull + 8 * i, 1);
    }
    for (int i = 0; i < NM; ++i) mbar_init(s_mfull + 8 * i, 1);
    for (int i = 0; i < 4; ++i) {
      mbar_init(s_sready + 8 * i, 1);
      mbar_init(s_pready + 8 * i, 256);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_pvdone + 8 * i, 1);
      mbar_init(s_qready + 8 * i, 256);
      mbar_init(s_pvstage + 8 * i, 1);
    }
    mbar_init(s_drain, 1);
    mbar_init(s_drain + 8, 1);
    fence_mbar_init();
  }
  if (warp == kWarpM) tmem_alloc(s_slot, kTc2TmemCols);
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *g_slot;
  if (!kOne || !p.early) grid_dep_wait();  // the plan must have completed
  grid_dep_launch();                       // the next kernel of the call may queue up behind this grid

  constexpr int kList = kOne ? 0 : 1;
  const long long cap_tokens = (long long)p.MB * p.bs;

  if (kOne && p.direct_tiles > 0 && blockIdx.x == 0 && warp == kWarpM + 1) {
    // the status word, which no plan has written (any other bit of it comes from a wait of seconds, long after this)
    bool refused = false;
    for (int b = lane; b < p.B; b += 32) packed_seq(p, b, &refused);
    refused = __any_sync(0xffffffffu, refused);
    const int word = refused ? kPackedStatusRefused : 0;
    if (lane == 0) kChecked ? (void)atomicOr(&p.hdr->dec.status, word) : (void)(p.hdr->dec.status = word);  // (checked: cleared by the host)
    __syncwarp();
  }
  if (warp == kWarpK) {
    // ================================================================= K producer (and the walk over the units)
    if (lane == 0) prefetch_tmap(&tm_k);
    const int boxes_per_stage = kTc2StageTok / p.tile_rows;   // at most 8 (blocks of 16 tokens)
    const uint32_t box_rows_bytes = (uint32_t)p.tile_rows * 128;
    int it = 0;
    bool ok = true, violated = false;
    const bool direct = kOne && p.direct_tiles > 0;
    const int64_t stages_all = direct ? 0 : p.hdr->stages[kList];
    const bool pull = direct || p.hdr->pull[kList];
    const int pieces = pull || stages_all == 0 ? 0 : p.hdr->pieces[kList];
    int unit = blockIdx.x;  // where pairs are pulled: the next one
    int64_t left = 0;       // else: what is left of the CTA's piece,
    int4 at = make_int4(0, 0, 0, 0);  // and its next tile, kv head and place in the pair
    if ((int)blockIdx.x < pieces) {
      left = packed_cut(stages_all, blockIdx.x + 1, pieces) - packed_cut(stages_all, blockIdx.x, pieces);
      at = p.start[kList][blockIdx.x];
    }
    const int n_pairs = direct ? p.B * p.direct_tiles * p.Hkv : (pull ? p.hdr->pairs[kList] : 0);
    auto table_entry = [&](const int32_t* e) {
      const int v = *e;
      return checked(chk_table_entry(v, p.NB), &p.hdr->dec.status, kStatusBadTableEntry) ? v : p.NB;
    };
    // waits until K slot, V slot (and with it the V descriptor) of stage `it` are free; false when a wait gave up
    auto acquire = [&]() {
      // (KV8: the slots the copies land in are the 8-bit ones, free once they have been widened)
      return warp_wait((KV8 ? s_rkempty : s_kempty) + 8 * (it % NK), (((uint32_t)(it / NK)) & 1u) ^ 1u, s_abort) &&
             warp_wait((KV8 ? s_rvempty : s_vempty) + 8 * (it % NV), (((uint32_t)(it / NV)) & 1u) ^ 1u, s_abort);
    };
    while ((pull ? unit < n_pairs : left > 0) && ok) {
      int nxt = 0;
      PackedTile tile;
      if (direct) {
        nxt = unit + gridDim.x;
        at = make_int4(unit / p.Hkv, unit % p.Hkv, 0, 0);
        const PackedSeq q = packed_seq(p, at.x / p.direct_tiles);
        tile.b = at.x / p.direct_tiles;
        tile.c0 = at.x % p.direct_tiles * kTcRows;
        tile.first = tile.end = at.x;
        tile.r0 = q.r0;
        tile.n = q.n;
        tile.T = q.T;
        if (tile.c0 >= p.G * q.n) {
          unit = nxt;
          continue;
        }
        tile.stages = max(1, (packed_seen(p, tile, kList) + kTc2StageTok - 1) / kTc2StageTok);
      } else {
        if (pull) {
          if (lane == 0) nxt = atomicAdd(&p.hdr->next[kList], 1);
          nxt = __shfl_sync(0xffffffffu, nxt, 0);
          at = make_int4(p.order[kList][unit / p.Hkv], unit % p.Hkv, 0, 0);
        }
        tile = p.tiles[at.x];
      }
      if (!checked(chk_item(tile.b, 0, 0, tile.T, p.B, 1, cap_tokens) && chk_span(tile.r0, tile.n, 0, p.num_rows) && tile.stages > 0 &&
                       (direct || chk_index(at.x, p.max_tiles)), &p.hdr->dec.status, kStatusBadItem)) {
        *s_abort = 1;
        violated = true;
        ok = false;
        break;
      }
      const int h = at.y, s0 = max(0, at.z - kPackedUnitCost);
      const int s1 = pull ? tile.stages : max(s0, (int)min((int64_t)tile.stages, at.z + left - kPackedUnitCost));
      const int b = tile.b, c0 = tile.c0, t0 = s0 * kTc2StageTok, t1 = min(packed_seen(p, tile, kList), s1 * kTc2StageTok);
      const int lim_base = tile.T - tile.n + 1;                     // tokens the first query token sees
      const int columns = p.G * tile.n;                             // of the (sequence, kv head) pair
      const int part = s0 == 0 && s1 == tile.stages ? -1 : packed_part(p, kList, blockIdx.x, s0 == 0);
      const int t1e = t1;                                           // (the plan counts only what the last column sees)
      const int nstage = t1e > t0 ? s1 - s0 : 0;
      const int32_t* row = p.block_table + (size_t)b * p.MB;
      int blk_cur = 0;
      {
        const int tb = t0 + lane * p.tile_rows;
        if (lane < boxes_per_stage && tb < t1e) blk_cur = table_entry(row + tb / p.bs);
      }
      // a pair that sees nothing of this chunk passes one stage without tokens, which carries the bookkeeping
      // (a piece that ends in front of a pair's stages leaves the whole pair to the next one)
      for (int s = 0; s < (nstage > 0 ? nstage : (s1 > s0 ? 1 : 0)); ++s, ++it) {
        const int tok0 = t0 + s * kTc2StageTok;
        const int ntok = nstage > 0 ? min(kTc2StageTok, t1e - tok0) : 0;
        const int nbox = (ntok + p.tile_rows - 1) / p.tile_rows;
        int blk_n = 0;  // table entries of the following stage, one stage ahead of their use
        {
          const int tb = tok0 + kTc2StageTok + lane * p.tile_rows;
          if (s + 1 < nstage && lane < boxes_per_stage && tb < t1e) blk_n = table_entry(row + tb / p.bs);
        }
        if (!acquire()) {
          ok = false;
          break;
        }
        const int ks = it % NK, vs = it % NV, ms = it % NM;
        const uint32_t kfull = (KV8 ? s_rkfull : s_kfull) + 8 * ks;
        if (lane == 0) {
          const int flags = (s == 0 ? 1 : 0) | (s == (nstage > 0 ? nstage : 1) - 1 ? 2 : 0);
          g_meta[3 * ms] = make_int4(part, tile.r0, h, ntok | (flags << 16));
          g_meta[3 * ms + 1] = make_int4(tok0, lim_base, t1, c0);
          g_meta[3 * ms + 2] = make_int4(columns, 0, 0, 0);
          g_vdesc[vs].nbox = nbox;
          g_vdesc[vs].h = h;
          if (nbox > 0)
            mbar_arrive_expect_tx(kfull, (KV8 ? 1u : (uint32_t)NH) * (uint32_t)nbox * box_rows_bytes);
          else
            mbar_arrive(kfull);
        }
        __syncwarp();
        bool span_ok = true;
        if (lane < nbox) {
          const int tb = tok0 + lane * p.tile_rows;
          const int c_tok = tb % p.bs;
          const uint32_t k0 = KV8 ? s_rk + (uint32_t)ks * kTc2RawSlotBytes : s_k + (uint32_t)ks * kSlotBytes;
          const uint32_t dk = k0 + (uint32_t)lane * box_rows_bytes;
          span_ok = checked(chk_span(dk, box_rows_bytes, k0, (long long)k0 + kTc2HalfBytes) && chk_span(lane, 1, 0, 8),
                            &p.hdr->dec.status, kStatusBadSmem);
          if (span_ok) {
            tma_load_4d(dk, &tm_k, kfull, 0, c_tok, h, blk_cur);  // (KV8: the row's 128 codes; else its first 64 dims)
            if (!KV8 && NH > 1) tma_load_4d(dk + kTc2HalfBytes, &tm_k, kfull, 64, c_tok, h, blk_cur);
            g_vdesc[vs].blk[lane & 7] = blk_cur;
            g_vdesc[vs].c_tok[lane & 7] = c_tok;
          }
        }
        if (kChecked && !__all_sync(0xffffffffu, span_ok)) {  // a skipped copy leaves the stage incomplete: stop
          *s_abort = 1;
          violated = true;
          ok = false;
          break;
        }
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(s_vdfull + 8 * vs);  // the V producer takes over the stage's V boxes
          mbar_arrive(s_mfull + 8 * ms);   // the softmax threads may read the meta words
        }
        blk_cur = blk_n;
      }
      if (pull) {
        unit = nxt;
      } else {
        left -= tile.stages + kPackedUnitCost - at.z;  // (below 0 where the pair goes on in the next piece)
        at.z = 0;
        if (++at.x == tile.end) {
          if (++at.y < p.Hkv) {
            at.x = tile.first;
          } else {
            at.y = 0;
            while (left > 0 && p.before[kList][at.x + 1] == p.before[kList][at.x]) ++at.x;  // (tiles of the other lists)
          }
        }
      }
    }
    if (ok) {  // end marker: one more stage, seen by every other warp
      if (acquire()) {
        if (lane == 0) {
          g_meta[3 * (it % NM)] = make_int4(0, 0, 0, kPackedEnd);
          g_vdesc[it % NV].nbox = -1;
          mbar_arrive((KV8 ? s_rkfull : s_kfull) + 8 * (it % NK));
          mbar_arrive(s_vdfull + 8 * (it % NV));
          mbar_arrive(s_mfull + 8 * (it % NM));
        }
        ++it;
      } else {
        ok = false;
      }
    }
    if (!ok) {  // stop path: record it, then wait (bounded) until every K copy already issued has landed
      if (lane == 0 && !violated) atomicOr(&p.hdr->dec.status, kStatusWaitTimeout);
      int dummy_abort = 0;
      for (int k = 0; k < (it < NK ? it : NK); ++k) {
        const int j = it - 1 - k;
        mbar_wait_bounded((KV8 ? s_rkfull : s_kfull) + 8 * (j % NK), (uint32_t)(j / NK) & 1u, &dummy_abort, kWaitLimitNs / 8);
      }
    }
  } else if (warp == kWarpV) {
    // ================================================================= V producer
    if (lane == 0) prefetch_tmap(&tm_v);
    const uint32_t box_rows_bytes = (uint32_t)p.tile_rows * 128;
    int it = 0;
    bool ok = true;
    for (;; ++it) {
      const int vs = it % NV;
      if (!warp_wait(s_vdfull + 8 * vs, (uint32_t)(it / NV) & 1u, s_abort)) {
        ok = false;
        break;
      }
      const VStageDesc& vd = g_vdesc[vs];
      const int nbox = vd.nbox;
      const uint32_t vfull = (KV8 ? s_rvfull : s_vfull) + 8 * vs;
      if (nbox <= 0) {  // a stage without tokens, or the end marker
        if (lane == 0) mbar_arrive(vfull);
        if (nbox < 0) break;
        continue;
      }
      if (lane == 0) mbar_arrive_expect_tx(vfull, (KV8 ? 1u : (uint32_t)NH) * (uint32_t)nbox * box_rows_bytes);
      __syncwarp();
      if (lane < nbox && lane < 8) {
        const uint32_t dv = (KV8 ? s_rv + (uint32_t)vs * kTc2RawSlotBytes : s_v + (uint32_t)vs * kSlotBytes) +
                            (uint32_t)lane * box_rows_bytes;
        tma_load_4d(dv, &tm_v, vfull, 0, vd.c_tok[lane], vd.h, vd.blk[lane]);
        if (!KV8 && NH > 1) tma_load_4d(dv + kTc2HalfBytes, &tm_v, vfull, 64, vd.c_tok[lane], vd.h, vd.blk[lane]);
      }
    }
    if (!ok) {
      if (lane == 0) atomicOr(&p.hdr->dec.status, kStatusWaitTimeout);
      int dummy_abort = 0;
      for (int k = 0; k < (it < NV ? it : NV); ++k) {
        const int j = it - 1 - k;
        mbar_wait_bounded((KV8 ? s_rvfull : s_vfull) + 8 * (j % NV), (uint32_t)(j / NV) & 1u, &dummy_abort, kWaitLimitNs / 8);
      }
    }
  } else if (warp >= kWarpM && kOne) {
    // ================================================================= MMA warps, one-tile mode
    // One thread issues an MMA about every 100 cycles, so a single issuing thread needs longer for the 16 MMAs of a
    // stage than HBM needs for the stage's bytes.  With one tile the two issuing warps split the stage instead: warp
    // kWarpM issues the scores S(n) = Q . K_slot^T into S buffer n & 1 (columns 256 (n & 1); buffer 1 is what tile 1's
    // scores would occupy), warp kWarpM + 1 the values O += P(n) . V_slot.  The pipe keeps no order between two
    // threads' MMAs, so each hand-over has a barrier: S(n) overwrites P(n - 2), hence waits for P.V(n - 2) to be
    // complete (s_pvstage, one completion per stage, with or without tokens); P.V(n) waits for the softmax threads'
    // P(n).  The scores of a stage are thus computed while the softmax threads still work on the one before.
    const int t = warp - kWarpM;
    bool issued = false, ok = true;
    if (t == 0) {
      const uint32_t idesc_s = umma_idesc_16bit(kTcRows, kTc2StageTok, 0, !KV8);  // (KV8: f16 operands)
      const uint64_t dq = umma_smem_desc(s_q, 0, 1024);
      uint32_t n_q = 0;  // units with tokens (uses of the q-ready barrier)
      for (uint32_t n = 0;; ++n) {
        const int ks = n % NK, ms = n % NM;
        if (!warp_wait(s_kfull + 8 * ks, (n / NK) & 1u, s_abort)) {
          ok = false;
          break;
        }
        const int4 meta = g_meta[3 * ms];
        const bool end = meta.w & kPackedEnd;
        const int ntok = end ? 0 : (meta.w & 0xffff);
        const bool first = !end && ((meta.w >> 16) & 1);
        // The buffer's previous contents, P(n - 2), have been consumed.  Waited for on every stage, with or without
        // tokens (the end marker included): it also means that the softmax threads are past their wait for S(n - 2),
        // so this stage's completion of the score barrier n & 1 cannot overtake them.
        if (n >= 2 && !warp_wait(s_pvstage + 8 * (n & 1), ((n - 2) >> 1) & 1u, s_abort)) {
          ok = false;
          break;
        }
        if (ntok > 0) {
          if (first) {
            if (!warp_wait(s_qready, n_q & 1u, s_abort)) {
              ok = false;
              break;
            }
            ++n_q;
          }
          tc_fence_after_sync();
          if (lane == 0) {
            const uint64_t dk = umma_smem_desc(s_k + (uint32_t)ks * kSlotBytes, 0, 1024);
            const uint32_t ts = tmem + 256u * (n & 1);
#pragma unroll
            for (int hh = 0; hh < NH; ++hh)
#pragma unroll
              for (int k = 0; k < 4; ++k) {  // 16 dims = 32 bytes further along the rows; the second 64 dims = the next half
                const uint64_t off = (uint64_t)((hh * kTc2HalfBytes + k * 32) >> 4);
                umma_ss(ts, dq + off, dk + off, idesc_s, (hh | k) ? 1u : 0u);
              }
            umma_commit(s_sready + 8 * (n & 1));
            umma_commit(s_kempty + 8 * ks);
          }
          __syncwarp();
          issued = true;
        } else {
          // no scores: the turn of the barriers is taken all the same (also wakes the softmax threads for the end marker)
          if (lane == 0) {
            mbar_arrive(s_sready + 8 * (n & 1));
            mbar_arrive(s_kempty + 8 * ks);
          }
          __syncwarp();
        }
        if (end) break;
      }
    } else {
      const uint32_t idesc_o = umma_idesc_16bit(kTcRows, D, 1, !KV8);
      for (uint32_t n = 0;; ++n) {
        const int vs = n % NV, ms = n % NM;
        if (!warp_wait(s_mfull + 8 * ms, (n / NM) & 1u, s_abort)) {
          ok = false;
          break;
        }
        const int4 meta = g_meta[3 * ms];
        if (meta.w & kPackedEnd) break;
        const int ntok = meta.w & 0xffff;
        const bool first = (meta.w >> 16) & 1, last = (meta.w >> 17) & 1;
        // the V slot first (normally there already), so that nothing but the MMAs follows the softmax threads' hand-over
        if ((ntok > 0 && !warp_wait(s_vfull + 8 * vs, (n / NV) & 1u, s_abort)) ||
            !warp_wait(s_pready + 8 * (n & 1), (n >> 1) & 1u, s_abort)) {
          ok = false;
          break;
        }
        if (ntok > 0) {
          tc_fence_after_sync();
          if (lane == 0) {
            const uint64_t dv = umma_smem_desc(s_v + (uint32_t)vs * kSlotBytes, kTc2HalfBytes, 1024);
            const uint32_t tp = tmem + 256u * (n & 1);
#pragma unroll
            for (int k = 0; k < kTc2StageTok / 16; ++k)  // 16 tokens: 8 columns of P, 16 rows of 128 bytes of V in either half
              umma_ts(tmem + 128, tp + 8 * k, dv + (uint64_t)(k * (2048 >> 4)), idesc_o, (first && k == 0) ? 0u : 1u);
            if (last) umma_commit(s_pvdone);
            umma_commit(s_pvstage + 8 * (n & 1));
            umma_commit(s_vempty + 8 * vs);
          }
          __syncwarp();
          issued = true;
        } else {
          if (lane == 0) {
            if (last) mbar_arrive(s_pvdone);  // a unit without tokens: nothing to wait for
            mbar_arrive(s_pvstage + 8 * (n & 1));
            mbar_arrive(s_vempty + 8 * vs);
          }
          __syncwarp();
        }
      }
    }
    if (!ok && lane == 0) atomicOr(&p.hdr->dec.status, kStatusWaitTimeout);
    if (!ok && issued) {  // the tensor memory must not be released under MMAs in flight
      if (lane == 0) umma_commit(s_drain + 8 * t);
      __syncwarp();
      int dummy = 0;
      mbar_wait_bounded(s_drain + 8 * t, 0u, &dummy, kWaitLimitNs / 8);
    }
  } else if (warp >= kWarpM) {
    // ================================================================= MMA warps: warp kWarpM + t issues tile t's MMAs
    // One thread issues an MMA about every 110 to 130 cycles whatever its size (measured: M128 N64 or N128 K16, either
    // operand source), twice what the pipe needs for N = 128, and the pipe overlaps the MMAs of two threads (two
    // issuers: one N = 128 MMA per 70 cycles).  So each tile has an issuing warp of its own; the order inside a tile,
    // P.V_t(n - 1) before S_t(n), is the program order of its thread, and the tiles need no order between them.
    const int t = warp - kWarpM;
    const uint32_t idesc_s = umma_idesc_16bit(kTcRows, kTc2StageTok, 0, true);
    const uint32_t idesc_o = umma_idesc_16bit(kTcRows, D, 1, true);
    const uint32_t ts = tmem + 256u * t;
    const uint64_t dq = umma_smem_desc(s_q + (uint32_t)t * kQBytes, 0, 1024);
    uint32_t n_q = 0;  // units in which the tile had rows and tokens (uses of its q-ready barrier)
    bool issued = false, ok = true;
    // what is known about the stage whose P.V MMAs are still to be issued
    bool p_valid = false, p_act = false, p_first = false, p_last = false;
    int p_ntok = 0;
    uint32_t p_n = 0;
    for (uint32_t n = 0;; ++n) {
      const int ks = n % NK, ms = n % NM;
      if (!warp_wait(s_kfull + 8 * ks, (n / NK) & 1u, s_abort)) {
        ok = false;
        break;
      }
      const int4 meta = g_meta[3 * ms], meta2 = g_meta[3 * ms + 1];
      const int columns = g_meta[3 * ms + 2].x;
      const bool end = meta.w & kPackedEnd;
      const int ntok = end ? 0 : (meta.w & 0xffff);
      const bool first = !end && ((meta.w >> 16) & 1), last = !end && ((meta.w >> 17) & 1);
      const bool act = !end && (t == 0 || meta2.w + kTcRows < columns);  // a unit always has rows in its first tile
      // Everything that is normally there already is waited for first (the pending stage's V slot, the other tile's
      // turn: see below), so that nothing but the MMAs themselves follows the softmax threads' hand-over.
      if (p_valid && p_act && p_ntok > 0 && !warp_wait(s_vfull + 8 * (p_n % NV), (p_n / NV) & 1u, s_abort)) {
        ok = false;
        break;
      }
      // The tiles take turns, half a stage apart: S_0(n), S_1(n), S_0(n + 1), ... in this order, so that one tile's
      // softmax runs beside the other tile's MMAs (P.V of the stage before, then these scores) instead of both tiles
      // doing the same thing at once.  Tile 1 waits for tile 0's scores of this stage, tile 0 for tile 1's of the
      // stage before -- on every stage, with or without work, so that neither warp can get two turns ahead of the
      // other on a barrier pair.
      if (t == 1 ? !warp_wait(s_sready + 8 * (n & 1), (n >> 1) & 1u, s_abort)
                 : (n > 0 && !warp_wait(s_sready + 8 * (2 + ((n - 1) & 1)), ((n - 1) >> 1) & 1u, s_abort))) {
        ok = false;
        break;
      }
      // ---- P.V of the pending stage: waits for the tile's softmax threads, then issues (or just takes the turn)
      if (p_valid) {
        const int vs = p_n % NV;
        if (!warp_wait(s_pready + 8 * (2 * t + (p_n & 1)), (p_n >> 1) & 1u, s_abort)) {
          ok = false;
          break;
        }
        if (p_act && p_ntok > 0) {
          tc_fence_after_sync();
          if (lane == 0) {
            const uint64_t dv = umma_smem_desc(s_v + (uint32_t)vs * kSlotBytes, kTc2HalfBytes, 1024);
#pragma unroll
            for (int k = 0; k < kTc2StageTok / 16; ++k)  // 16 tokens: 8 columns of P, 16 rows of 128 bytes of V in either half
              umma_ts(ts + 128, ts + 8 * k, dv + (uint64_t)(k * (2048 >> 4)), idesc_o, (p_first && k == 0) ? 0u : 1u);
            if (p_last) umma_commit(s_pvdone + 8 * t);
            umma_commit(s_vempty + 8 * vs);  // (one of the two arrivals that free the V slot)
          }
          __syncwarp();
          issued = true;
        } else {
          if (lane == 0) {
            if (p_act && p_last) mbar_arrive(s_pvdone + 8 * t);  // a unit without tokens: nothing to wait for
            mbar_arrive(s_vempty + 8 * vs);
          }
          __syncwarp();
        }
      }
      // ---- scores of this stage
      if (act && ntok > 0) {
        if (first) {
          if (!warp_wait(s_qready + 8 * t, n_q & 1u, s_abort)) {
            ok = false;
            break;
          }
          ++n_q;
        }
        tc_fence_after_sync();
        if (lane == 0) {
          const uint64_t dk = umma_smem_desc(s_k + (uint32_t)ks * kSlotBytes, 0, 1024);
#pragma unroll
          for (int hh = 0; hh < NH; ++hh)
#pragma unroll
            for (int k = 0; k < 4; ++k) {  // 16 dims = 32 bytes further along the rows; the second 64 dims = the next half
              const uint64_t off = (uint64_t)((hh * kTc2HalfBytes + k * 32) >> 4);
              umma_ss(ts, dq + off, dk + off, idesc_s, (hh | k) ? 1u : 0u);
            }
          umma_commit(s_sready + 8 * (2 * t + (n & 1)));
          umma_commit(s_kempty + 8 * ks);  // (one of the two arrivals that free the K slot)
        }
        __syncwarp();
        issued = true;
      } else {
        // no scores for this tile: the turn of its barriers is taken all the same (also wakes the softmax threads
        // for the end marker)
        if (lane == 0) {
          mbar_arrive(s_sready + 8 * (2 * t + (n & 1)));
          mbar_arrive(s_kempty + 8 * ks);
        }
        __syncwarp();
      }
      if (end) break;
      p_valid = true;
      p_act = act;
      p_first = first;
      p_last = last;
      p_ntok = ntok;
      p_n = n;
    }
    if (!ok && lane == 0) atomicOr(&p.hdr->dec.status, kStatusWaitTimeout);
    if (!ok && issued) {  // the tensor memory must not be released under MMAs in flight
      if (lane == 0) umma_commit(s_drain + 8 * t);
      __syncwarp();
      int dummy = 0;
      mbar_wait_bounded(s_drain + 8 * t, 0u, &dummy, kWaitLimitNs / 8);
    }
  } else {
    // ================================================================= softmax warps
    // Tile t = warps 8 t .. 8 t + 7.  Warp (q = warp & 3, hf = (warp >> 2) & 1) owns the 16 score rows
    // 32 q + 16 hf .. + 15 of the tile (a warp reaches the 32 tensor-memory lanes of its quarter q only) and reads
    // them in the 16-lane shape: lane (g, tq) holds rows g and g + 8, columns 8 i + 2 tq, + 1 -- two threads would be
    // too few per row to hide the latency of the row's chain, four share it here and combine with quad shuffles.
    const int t = warp >> 3, q4 = warp & 3, hf = (warp >> 2) & 1;
    const int g = lane >> 2, tq = lane & 3;
    const int row0 = 32 * q4 + 16 * hf + g;  // this thread's rows of the tile: row0 and row0 + 8
    const uint32_t trow = tmem + ((uint32_t)(32 * q4 + 16 * hf) << 16) + 256u * t;  // the warp's lanes, the tile's columns
    const int tid_t = threadIdx.x & 255;     // index among the tile's 256 threads
    // Score column (query token x head) of a tile's row r: column 4 (r % 32) + r / 32 of the tile, so that the columns
    // of a tile that is not full spread over the four lane quarters -- the warps with hf = 0 take rows before those with
    // hf = 1, one busy warp per scheduler -- and a warp none of whose rows is a column skips the stage's arithmetic.
    auto tile_col = [](int r) { return 4 * (r & 31) + (r >> 5); };
    uint8_t* q_gen = gen + (size_t)t * kQBytes;
    float m_ref[2] = {-INFINITY, -INFINITY};  // reference maximum per row (scaled, log2 domain)
    float l_part[2] = {0.f, 0.f};             // this thread's share of the row's sum of weights
    int lim_row[2] = {0, 0};
    // Units in which this tile had rows, times kUnit; below that, 127 + the binary orders that the warp's rows of Q were lowered by
    // (load_q).  One register for both, and one number for all rows of the warp: kept apart, or by rows, prompts over the 8-bit cache
    // took 11 and 16 % longer than without (this form: 3 to 4 %).
    constexpr uint32_t kUnit = 512;
    uint32_t n_unit = 127;
    bool ok = true;
    bool q_ahead = false;  // the Q rows of the unit that starts with the next stage are in shared memory already
    // Q of the tile's columns from c0_ on, of a sequence whose rows of q begin at row0_, into the swizzled K-major tile
    // ([half][row][64 dims], 16-byte chunk ^= row & 7): a warp writes its own 16 rows, two lanes a row; then the q-ready
    // arrival.  KV8: f16 ends at 65504 and has 11 bits down to 2^-14, bf16 goes far beyond, so a warp's rows are moved by the power of
    // two that brings the largest finite one of their values to 2^15, which the scale of their scores takes back.  A value x is off by at most
    // 2^-11 |x|, or half a step of the smallest f16 numbers: 2^-40 of that largest one, 2^-125 where that is below 2^-85.
    auto load_q = [&](int row0_, int h_, int c0_, int columns_) {
      const int r_ = 32 * q4 + 16 * hf + (lane >> 1), part_ = lane & 1;
      const int col_ = c0_ + t * kTcRows + tile_col(r_);
      const int qi_ = col_ / p.G, head_ = col_ - qi_ * p.G;
      const bool real_ = col_ < columns_;
      const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)(row0_ + (real_ ? qi_ : 0)) * p.q_stride +
                                                        (int64_t)(h_ * p.G + (real_ ? head_ : 0)) * D + part_ * (D / 2));
      uint4 w_[D / 16];
#pragma unroll
      for (int c = 0; c < D / 16; ++c) w_[c] = real_ ? src[c] : make_uint4(0u, 0u, 0u, 0u);
      float factor = 1.f;
      if (KV8) {
        uint32_t top = 0u;  // the largest magnitude, as bits: of the even and of the odd dims, then of the warp's rows
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
          top = __vmaxu2(top, __vmaxu2(__vmaxu2(w_[c].x & 0x7fff7fffu, w_[c].y & 0x7fff7fffu),
                                       __vmaxu2(w_[c].z & 0x7fff7fffu, w_[c].w & 0x7fff7fffu)));
        top = max(top & 0xffffu, top >> 16);
        if (top >= 0x7f80u) top = 0u;  // (what is not finite stays so, and must not move its neighbours)
        top = __reduce_max_sync(0xffffffffu, top);
        const int e = (int)(top >> 7) - 127;  // 2^e <= the largest value < 2^(e + 1)
        // (not below -100, so that the scores and their scale stay far from the ends of fp32)
        const int shift = e > 15 ? e - 15 : (e < 15 && top ? max(e - 15, -100) : 0);
        factor = __uint_as_float((uint32_t)(127 - shift) << 23);
        n_unit = (n_unit & ~(kUnit - 1)) | (uint32_t)(127 + shift);
      }
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        uint4 v = w_[c];
        if (KV8) {
          auto narrow = [&](uint32_t x) { return pack_f16x2(bf16_lo(x) * factor, bf16_hi(x) * factor); };
          v = make_uint4(narrow(v.x), narrow(v.y), narrow(v.z), narrow(v.w));
        }
        const int cc = part_ * (D / 16) + c;
        *reinterpret_cast<uint4*>(q_gen + (size_t)(cc >> 3) * kTc2HalfBytes + (size_t)r_ * 128 + (((cc & 7) ^ (r_ & 7)) << 4)) = v;
      }
      fence_proxy_async_smem();  // the tile is read by the MMAs through the async proxy
      mbar_arrive(s_qready + 8 * t);
    };
    if (KV8 && t == 1) {
      // ================================================================= widening warps (8-bit cache, one-tile mode)
      // Stage n of the 8-bit rings becomes stage n of the 16-bit slots (stages without tokens and the end marker take
      // their turns too).  A unit of work is (token row r, 16-byte chunk c of the row's 128 codes): one 16-byte load,
      // sixteen codes widened, two 16-byte stores into the row's 64-dim half c / 4; 1024 units per slot, four per
      // thread.  K first: the scores need it a stage earlier than P.V needs V.
      auto widen = [&](const uint8_t* rsrc, uint8_t* sdst, int ntok_) {
#pragma unroll
        for (int i = 0; i < kTc2StageTok * 8 / 256; ++i) {
          const int u = i * 256 + tid_t;
          const int r = u >> 3, c = u & 7;
          if (r >= ntok_) continue;  // rows beyond the stage's tokens are never used (masked scores, cleared V rows)
          const uint4 w = *reinterpret_cast<const uint4*>(rsrc + (size_t)r * 128 + ((c ^ (r & 7)) << 4));
          uint8_t* drow = sdst + (size_t)(c >> 2) * kTc2HalfBytes + (size_t)r * 128;
          *reinterpret_cast<uint4*>(drow + (((2 * (c & 3)) ^ (r & 7)) << 4)) =
              make_uint4(e4m3x2_to_f16x2<kSelB0B1>(w.x), e4m3x2_to_f16x2<kSelB2B3>(w.x), e4m3x2_to_f16x2<kSelB0B1>(w.y),
                         e4m3x2_to_f16x2<kSelB2B3>(w.y));
          *reinterpret_cast<uint4*>(drow + (((2 * (c & 3) + 1) ^ (r & 7)) << 4)) =
              make_uint4(e4m3x2_to_f16x2<kSelB0B1>(w.z), e4m3x2_to_f16x2<kSelB2B3>(w.z), e4m3x2_to_f16x2<kSelB0B1>(w.w),
                         e4m3x2_to_f16x2<kSelB2B3>(w.w));
        }
      };
      for (uint32_t n = 0;; ++n) {
        const int ks = n % NK, vs = n % NV, ms = n % NM;
        // the 8-bit K slot has landed (its meta words were written before its barrier was armed), the 16-bit one is free
        if (!warp_wait(s_rkfull + 8 * ks, (n / NK) & 1u, s_abort) ||
            !warp_wait(s_kempty + 8 * ks, ((n / NK) & 1u) ^ 1u, s_abort)) {
          ok = false;
          break;
        }
        const int4 meta = g_meta[3 * ms];
        const bool end = meta.w & kPackedEnd;
        const int ntok = end ? 0 : (meta.w & 0xffff);
        if (ntok > 0) {
          widen(gen + (s_rk - base) + (size_t)ks * kTc2RawSlotBytes, gen + (s_k - base) + (size_t)ks * kSlotBytes, ntok);
          fence_proxy_async_smem();  // the widened slot is read by the MMAs through the async proxy
        }
        mbar_arrive(s_kfull + 8 * ks);
        mbar_arrive(s_rkempty + 8 * ks);
        if (end) break;
        if (!warp_wait(s_rvfull + 8 * vs, (n / NV) & 1u, s_abort) ||
            !warp_wait(s_vempty + 8 * vs, ((n / NV) & 1u) ^ 1u, s_abort)) {
          ok = false;
          break;
        }
        if (ntok > 0) {
          widen(gen + (s_rv - base) + (size_t)vs * kTc2RawSlotBytes, gen + (s_v - base) + (size_t)vs * kSlotBytes, ntok);
          fence_proxy_async_smem();
        }
        mbar_arrive(s_vfull + 8 * vs);
        mbar_arrive(s_rvempty + 8 * vs);
      }
    }
    for (uint32_t n = 0; !(kOne && t == 1); ++n) {  // (one-tile mode: the warps of tile 1 have nothing else to do)
      const int ms = n % NM;
      if (!warp_wait(s_mfull + 8 * ms, (n / NM) & 1u, s_abort)) {
        ok = false;
        break;
      }
      const int4 meta = g_meta[3 * ms], meta2 = g_meta[3 * ms + 1];
      const int columns = g_meta[3 * ms + 2].x;
      const bool end = meta.w & kPackedEnd;
      const int ntok = end ? 0 : (meta.w & 0xffff);
      const bool first = !end && ((meta.w >> 16) & 1), last = !end && ((meta.w >> 17) & 1);
      const int h = meta.z, c0 = meta2.w, lim_base = meta2.y;
      const bool act = !end && (t == 0 || c0 + kTcRows < columns);
      const int col0 = c0 + t * kTcRows + tile_col(row0);  // score column of row0; that of row0 + 8: col0 + 32
      const bool warp_rows = c0 + t * kTcRows + tile_col(32 * q4 + 16 * hf) < columns;  // the warp's first column exists
      if (first && act) {
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) {
          m_ref[rr] = -INFINITY;
          l_part[rr] = 0.f;
          lim_row[rr] = lim_base + (col0 + 32 * rr) / p.G;
        }
        if (ntok > 0 && !q_ahead) load_q(meta.y, h, c0, columns);
        q_ahead = false;
        n_unit += kUnit;
      }
      if (!warp_wait(s_sready + 8 * (2 * t + (n & 1)), (n >> 1) & 1u, s_abort)) {
        ok = false;
        break;
      }
      if (end) break;
      if (act && ntok > 0 && warp_rows) {
        tc_fence_after_sync();
        // Two passes over the stage's scores, 64 tokens at a time (32 registers): the row maxima first, then, with the
        // reference maxima known, the weights.  Reading the scores twice costs little (tensor memory is close) and
        // keeps the threads clear of spills.  sh[4 i + 2 rr + c] = score of row (row0 + 8 rr), token 64 h2 + 8 i + 2 tq + c.
        // tokens [0, e) of the stage are visible to the row
        const int e0 = min(min(meta2.z, lim_row[0]) - meta2.x, ntok), e1 = min(min(meta2.z, lim_row[1]) - meta2.x, ntok);
        const bool masked = __any_sync(0xffffffffu, min(e0, e1) < kTc2StageTok);
        const uint32_t srow = trow + (kOne ? 256u * (n & 1) : 0u);  // the stage's S (and P) columns
        auto load_half = [&](int h2, uint32_t (&sh)[32]) {
          tmem_ld_16x256b_x8(srow + 64 * h2, sh);
          tmem_ld_wait();
          if (masked) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const int j = 64 * h2 + 8 * i + 2 * tq + c;
                if (j >= e0) sh[4 * i + c] = 0xff800000u;  // -inf
                if (j >= e1) sh[4 * i + 2 + c] = 0xff800000u;
              }
          }
        };
        const float scale = KV8 ? p.scale_log2e * __uint_as_float(n_unit << 23) : p.scale_log2e;
        float mxr[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
          uint32_t sh[32];
          load_half(h2, sh);
#pragma unroll
          for (int rr = 0; rr < 2; ++rr) {
            float ma = mxr[rr], mb = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {  // three-input maximum: two scores per instruction, two chains
              ma = fmax3(ma, __uint_as_float(sh[4 * i + 2 * rr]), __uint_as_float(sh[4 * i + 2 * rr + 1]));
              mb = fmax3(mb, __uint_as_float(sh[4 * i + 4 + 2 * rr]), __uint_as_float(sh[4 * i + 4 + 2 * rr + 1]));
            }
            mxr[rr] = fmaxf(ma, mb);
          }
        }
        float alpha[2] = {1.f, 1.f}, neg_mu[2];
        bool raise_any = false;
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) {
          float mx = mxr[rr];
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
          mx *= scale;  // positive
          // reference maximum: raised only when the row maximum is more than kTcRescaleStep above it
          const bool raise = m_ref[rr] != -INFINITY && mx > m_ref[rr] + kTcRescaleStep;
          if (m_ref[rr] == -INFINITY) {
            m_ref[rr] = mx;  // nothing accumulated for this row so far
          } else if (raise) {
            alpha[rr] = ex2(m_ref[rr] - mx);
            m_ref[rr] = mx;
          }
          raise_any |= raise;
          neg_mu[rr] = m_ref[rr] == -INFINITY ? 0.f : -m_ref[rr];
        }
        if (__any_sync(0xffffffffu, raise_any)) {
          // P.V of the previous stage was issued before this stage's score MMAs, so it is complete: O may be rescaled
          // (one-tile mode: another thread issues it, so its own barrier is waited on; never on a unit's first stage)
          if (kOne && !warp_wait(s_pvstage + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1u, s_abort)) {
            ok = false;
            break;
          }
          if (kOne) tc_fence_after_sync();
#pragma unroll 1
          for (int c2 = 0; c2 < NH; ++c2) {
            uint32_t o[32];
            tmem_ld_16x256b_x8(trow + 128 + 64 * c2, o);
            tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * alpha[(j >> 1) & 1]);
            tmem_st_16x256b_x8(trow + 128 + 64 * c2, o);
          }
          tmem_st_wait();
          l_part[0] *= alpha[0];
          l_part[1] *= alpha[1];
        }
        const float2 scale2 = make_float2(scale, scale);
        const float2 nm0 = make_float2(neg_mu[0], neg_mu[0]), nm1 = make_float2(neg_mu[1], neg_mu[1]);
        float2 add0 = {0.f, 0.f}, add1 = {0.f, 0.f};
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {  // 64 tokens at a time: 16 packed words of P per thread
          uint32_t sh[32];
          load_half(h2, sh);
          // (P of the first 64 tokens lands on score columns 0 .. 31, read by now; the second 64 tokens' scores, still
          // to be read, are columns 64 .. 127)
          uint32_t pw[16];  // pw[2 i + rr]: row (row0 + 8 rr), tokens 64 h2 + 8 i + 2 tq, + 1 = P column 32 h2 + 4 i + tq
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int r = 4 * i;
            const float2 x0 = ffma2(make_float2(__uint_as_float(sh[r]), __uint_as_float(sh[r + 1])), scale2, nm0);
            const float2 x1 = ffma2(make_float2(__uint_as_float(sh[r + 2]), __uint_as_float(sh[r + 3])), scale2, nm1);
            const float2 w0 = make_float2(ex2(x0.x), ex2(x0.y)), w1 = make_float2(ex2(x1.x), ex2(x1.y));
            add0 = fadd2(add0, w0);
            add1 = fadd2(add1, w1);
            pw[2 * i] = KV8 ? pack_f16x2(w0.x, w0.y) : pack_bf16x2(w0.x, w0.y);
            pw[2 * i + 1] = KV8 ? pack_f16x2(w1.x, w1.y) : pack_bf16x2(w1.x, w1.y);
          }
          tmem_st_16x128b_x8(srow + 32 * h2, pw);
        }
        l_part[0] += add0.x + add0.y;
        l_part[1] += add1.x + add1.y;
        tmem_st_wait();
      }
      if (act && ntok > 0) {
        if (ntok < kTc2StageTok) {
          // V rows beyond the stage's tokens may hold anything (NaN included): clear them once the slot has landed
          const int vs = n % NV;
          if (!warp_wait(s_vfull + 8 * vs, (n / NV) & 1u, s_abort)) {
            ok = false;
            break;
          }
          uint8_t* vgen = gen + (s_v - base) + (size_t)vs * kSlotBytes;
          for (int idx = tid_t; idx < (kTc2StageTok - ntok) * (D / 8); idx += 256) {
            const int r = ntok + idx / (D / 8), c = idx % (D / 8);
            *reinterpret_cast<uint4*>(vgen + (size_t)(c >> 3) * kTc2HalfBytes + (size_t)r * 128 + ((c & 7) << 4)) =
                make_uint4(0u, 0u, 0u, 0u);
          }
          fence_proxy_async_smem();  // the cleared rows are read by the MMA through the async proxy
        }
        tc_fence_before_sync();
        __syncwarp();
      }
      mbar_arrive(s_pready + 8 * (2 * t + (n & 1)));

      if (last && act) {
        // The unit's last score MMAs are complete, so the tile's Q rows are free: when the next stage opens a unit
        // with rows in this tile, its Q goes to shared memory now and the score MMAs of that stage need not wait
        // for the epilogue below.
        {
          const int ms1 = (n + 1) % NM;
          if (!warp_wait(s_mfull + 8 * ms1, ((n + 1) / NM) & 1u, s_abort)) {
            ok = false;
            break;
          }
          const int4 nm = g_meta[3 * ms1], nm2 = g_meta[3 * ms1 + 1];
          const int ncol = g_meta[3 * ms1 + 2].x;
          if (!(nm.w & kPackedEnd) && (nm.w & 0xffff) > 0 && (t == 0 || nm2.w + kTcRows < ncol)) {
            load_q(nm.y, nm.z, nm2.w, ncol);
            q_ahead = true;
          }
        }
        // ---- the unit is complete: normalise the rows of O and write them
        const int part = meta.x;  // first partial row of the unit, or -1: the rows are complete
        // the use of the tile's pv-done barrier that is the unit's
        if (!warp_wait(s_pvdone + 8 * t, (n_unit / kUnit - 1) & 1u, s_abort)) {
          ok = false;
          break;
        }
        tc_fence_after_sync();
        const bool unit_has_tokens = ntok > 0;  // (a unit without tokens is one stage: nothing is in O)
        float inv[2], lse[2];
        __nv_bfloat16* orow[2];
        float* prow[2];
        bool write_row[2];
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) {
          float l = l_part[rr];
          l += __shfl_xor_sync(0xffffffffu, l, 1);
          l += __shfl_xor_sync(0xffffffffu, l, 2);
          // l = 0: the row saw no token of this chunk; the 8-bit cache's V scale (and widening factor) comes in here
          inv[rr] = (l > 0.f ? 1.f / l : 0.f) * (KV8 ? p.v_scale : 1.f);
          lse[rr] = l > 0.f ? m_ref[rr] + lg2(l) : -INFINITY;
          const int col = col0 + 32 * rr;
          const int qi = col / p.G, head = col - qi * p.G;
          write_row[rr] = col < columns &&
                          checked(part < 0 || chk_index(part + col - c0, p.max_part_rows), &p.hdr->dec.status, kStatusBadIndex);
          orow[rr] = p.out + (int64_t)(meta.y + qi) * p.out_stride + (int64_t)(h * p.G + head) * D;
          prow[rr] = p.part_o + (int64_t)(part + col - c0) * D;
          if (write_row[rr] && tq == 0 && part >= 0) p.part_lse[part + col - c0] = lse[rr];
        }
#pragma unroll 1
        for (int c2 = 0; c2 < (warp_rows ? NH : 0); ++c2) {
          uint32_t o[32];  // o[4 i + 2 rr + c] = row (row0 + 8 rr), dim 64 c2 + 8 i + 2 tq + c
          if (unit_has_tokens) {
            tmem_ld_16x256b_x8(trow + 128 + 64 * c2, o);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = 0u;
          }
#pragma unroll
          for (int rr = 0; rr < 2; ++rr) {
            if (!write_row[rr]) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float a = __uint_as_float(o[4 * i + 2 * rr]) * inv[rr], c = __uint_as_float(o[4 * i + 2 * rr + 1]) * inv[rr];
              const int dim = 64 * c2 + 8 * i + 2 * tq;
              if (part < 0)
                *reinterpret_cast<uint32_t*>(orow[rr] + dim) = pack_bf16x2(a, c);
              else
                *reinterpret_cast<float2*>(prow[rr] + dim) = make_float2(a, c);
            }
          }
          __syncwarp();  // the tensor-memory loads are warp-wide: reconverge before the next one
        }
        tc_fence_before_sync();  // the next unit's first P.V overwrites O: ordered behind these reads by p-ready
      }
    }
    if (!ok && lane == 0) atomicOr(&p.hdr->dec.status, kStatusWaitTimeout);
  }
  // ---- common exit: release the tensor memory once every warp is done with it
  tc_fence_before_sync();
  __syncthreads();
  if (warp == kWarpM) tmem_dealloc(tmem, kTc2TmemCols);
  if (kOne && p.early) grid_dep_wait();  // (this grid's end says that the one in front of it has ended, too)
}


}  // namespace ooco
