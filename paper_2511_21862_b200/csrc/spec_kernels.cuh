// Kernels of the operators around the attention of a speculative decoding step: slot planning, rotary
// positions with the cache append, verification of the drafts, moving the accepted branch together.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "cta_util.cuh"
#include "ptx.cuh"

namespace ooco {

constexpr int kSlotsStatusBadBlock = 4, kSlotsStatusRefused = 128;

// ------------------------------------------------------------------------------------ slot planning
struct SlotsParams {
  const int32_t *context_lens, *new_lens, *blocks_held, *free_ids, *free_head, *parents;
  int32_t *block_table, *blocks_held_out, *free_head_out, *slot_map, *positions, *first_token, *granted, *total;
  int32_t* status;     // may be NULL
  int32_t* ws_from;    // [B] index into free_ids of the sequence's first new block
  int32_t* ws_held;    // [B] blocks held before the call (blocks_held may be updated in place)
  int32_t B, bs_log2, NB, MB, num_free, row_len, num_rows;
};

constexpr int kSlotsThreads = kScanThreads;

// One CTA: two prefix sums over the sequences (tokens, missing blocks), who is granted, and the per-sequence
// outputs.  Latency-bound: two block-wide scans per 1024 sequences.  The rows of a small call are filled by the same CTA, which
// saves a launch: 64 sequences of 16 tree nodes take 6.3 us.
__device__ __forceinline__ void slots_scan_body(const SlotsParams& p) {
  __shared__ long long s_warp[32];
  __shared__ int s_taken;
  const int tid = threadIdx.x;
  const long long cap = (long long)p.MB << p.bs_log2;
  const int head0 = max(0, *p.free_head);
  if (tid == 0) s_taken = 0;
  long long run_tok = 0, run_need = 0;
  bool refused_any = false;
  for (int base = 0; base < p.B; base += kSlotsThreads) {
    const int b = base + tid;
    const bool live = b < p.B;
    const long long ctx = live ? max(0, p.context_lens[b]) : 0, add = live ? max(0, p.new_lens[b]) : 0;
    const int held = live ? min(max(0, p.blocks_held[b]), p.MB) : 0;
    long long sum_tok, sum_need;
    const long long tok_hi = run_tok + block_scan(add, s_warp, &sum_tok);
    const bool fits = ctx + add <= cap && ctx <= ((long long)held << p.bs_log2) &&
                      (add == 0 || (p.row_len ? add <= p.row_len : tok_hi <= p.num_rows));
    const long long want = (ctx + add + (1 << p.bs_log2) - 1) >> p.bs_log2;
    const int need = live && fits && want > held ? (int)(want - held) : 0;
    const long long need_hi = run_need + block_scan(need, s_warp, &sum_need);
    const bool ok = fits && (need == 0 || head0 + need_hi <= p.num_free);
    if (live) {
      const long long f = p.row_len ? (long long)b * p.row_len : tok_hi - add;
      p.first_token[b] = (int)min(f, (long long)p.num_rows);
      p.granted[b] = ok ? (int)add : 0;
      p.total[b] = (int)(ctx + (ok ? add : 0));
      p.ws_from[b] = ok ? (int)(head0 + need_hi - need) : 0;
      p.ws_held[b] = held;
      p.blocks_held_out[b] = held + (ok ? need : 0);
      if (ok && need > 0) atomicMax(&s_taken, (int)need_hi);
      refused_any |= !ok;
    }
    run_tok += sum_tok;
    run_need += sum_need;
  }
  const bool refused = __syncthreads_or(refused_any);
  if (tid == 0) {
    p.first_token[p.B] = p.row_len ? p.num_rows : (int)min(run_tok, (long long)p.num_rows);
    *p.free_head_out = head0 + s_taken;
    if (refused && p.status) atomicOr(p.status, kSlotsStatusRefused);
  }
}

// Slots and positions, four consecutive rows per thread; the row of a block's first token also writes the
// block-table entry of a newly taken block (every such block starts with a new token).
__device__ __forceinline__ void slots_fill_body(const SlotsParams& p, int block, int nblocks) {
  const int groups = p.num_rows / 4 + (p.num_rows % 4 ? 1 : 0);
  const bool vec = (((uintptr_t)p.slot_map | (uintptr_t)p.positions) & 15) == 0;
  const int used = p.row_len ? p.num_rows : p.first_token[p.B];
  bool bad = false;
  auto store_rows = [&](int r0, int n, const int (&slot)[4], const int (&pos)[4]) {
    if (vec && n == 4) {
      *reinterpret_cast<int4*>(p.slot_map + r0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
      *reinterpret_cast<int4*>(p.positions + r0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
      return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < n) {
        p.slot_map[r0 + k] = slot[k];
        p.positions[r0 + k] = pos[k];
      }
  };
  // Each CTA has consecutive rows: a thread's next rows are mostly those of the same sequence or the one behind it, and the
  // search over the sequences is rarely needed.  Bound by the rows' stores: 256 packed prompts, 8.4 M rows of which 5.2 M are
  // used, take 21.8 us, scan included (67 MB of rows, 10.4 us at the measured copy rate; 25.6 us with a search for every
  // four rows).
  const long long per = (groups + nblocks - 1) / nblocks, g_hi = min((long long)groups, (block + 1) * per);
  int b = 0;
  for (long long gi = block * per + threadIdx.x; gi < g_hi; gi += blockDim.x) {
    const int r0 = (int)(4 * gi);
    int slot[4] = {-1, -1, -1, -1}, pos[4] = {-1, -1, -1, -1};
    const int n = min(4, p.num_rows - r0);
    if (r0 < used) {
      if (p.row_len) {
        b = r0 / p.row_len;
      } else {
        // largest b with first_token[b] <= r0 (rows increase, so it is not below the last one)
        int lo = b, hi = p.B;
        for (int k = 0; k < 2 && lo + 1 < hi; ++k) {
          if (p.first_token[lo + 1] <= r0) ++lo; else hi = lo + 1;
        }
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (p.first_token[mid] <= r0) lo = mid; else hi = mid;
        }
        b = lo;
      }
      const int seq_lo = p.row_len ? b * p.row_len : p.first_token[b];
      const int seq_hi = p.row_len ? seq_lo + p.row_len : p.first_token[b + 1];
      const int i0 = r0 - seq_lo;
      if (!p.parents && r0 + 4 <= seq_hi && i0 + 4 <= p.granted[b]) {
        // four granted tokens of one sequence: at most two blocks
        const int t0 = p.context_lens[b] > 0 ? p.context_lens[b] + i0 : i0, held = p.ws_held[b], from = p.ws_from[b];
        const int ia = t0 >> p.bs_log2, ib = (t0 + 3) >> p.bs_log2, mask = (1 << p.bs_log2) - 1;
        int32_t* row = p.block_table + (size_t)b * p.MB;
        const int blk_a = ia < held ? row[ia] : p.free_ids[from + ia - held];
        int blk_b = blk_a;
        if (ib != ia) {
          blk_b = ib < held ? row[ib] : p.free_ids[from + ib - held];
          if (ib >= held) row[ib] = blk_b;
        } else if (ia >= held && (t0 & mask) == 0) {
          row[ia] = blk_a;
        }
        const bool ok_a = blk_a >= 0 && blk_a < p.NB, ok_b = blk_b >= 0 && blk_b < p.NB;
        bad |= !ok_a || !ok_b;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int t = t0 + k;
          const bool first_blk = (t >> p.bs_log2) == ia;
          pos[k] = t;
          slot[k] = (first_blk ? ok_a : ok_b) ? ((first_blk ? blk_a : blk_b) << p.bs_log2) + (t & mask) : -1;
        }
        store_rows(r0, n, slot, pos);
        continue;
      }
      int cur = -1, row_lo = 0, row_hi = 0, ctx = 0, held = 0, from = 0, granted = 0, add = 0, blk_at = -1, blk = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int r = r0 + k;
        if (k >= n || r >= used) break;
        if (cur >= 0 && r >= row_hi) ++b;
        while (cur != b) {  // (packed: sequences without new tokens are passed over)
          row_lo = p.row_len ? b * p.row_len : p.first_token[b];
          row_hi = p.row_len ? row_lo + p.row_len : p.first_token[b + 1];
          cur = b;
          if (r >= row_hi) {
            ++b;
            continue;
          }
          ctx = max(0, p.context_lens[b]);
          add = max(0, p.new_lens[b]);
          granted = p.granted[b];
          held = p.ws_held[b];
          from = p.ws_from[b];
          blk_at = -1;
        }
        const int i = r - row_lo;
        if (i >= add) continue;  // padding
        int at = i;              // distance from the end of the context: index, or depth in the tree
        if (p.parents) {
          at = 0;
          for (int j = i, up = p.parents[row_lo + i]; up >= 0 && up < j; j = up, up = p.parents[row_lo + up]) ++at;
        }
        pos[k] = (int)min((long long)ctx + at, 0x7fffffffLL);
        if (i >= granted) continue;
        const int t = ctx + i, idx = t >> p.bs_log2, off = t & ((1 << p.bs_log2) - 1);
        if (idx != blk_at) {
          blk = idx < held ? p.block_table[(size_t)b * p.MB + idx] : p.free_ids[from + idx - held];
          blk_at = idx;
        }
        if (idx >= held && off == 0) p.block_table[(size_t)b * p.MB + idx] = blk;
        if (blk >= 0 && blk < p.NB) slot[k] = (blk << p.bs_log2) + off;
        else bad = true;
      }
    }
    store_rows(r0, n, slot, pos);
  }
  if (bad && p.status) atomicOr(p.status, kSlotsStatusBadBlock);
}

__global__ void __launch_bounds__(kSlotsThreads) slots_scan_kernel(const SlotsParams p, const int fill) {
  grid_dep_wait();
  grid_dep_launch();
  slots_scan_body(p);
  if (fill) {
    __syncthreads();  // the scan's outputs, written by this CTA, are read back
    slots_fill_body(p, 0, 1);
  }
}
__global__ void __launch_bounds__(256) slots_fill_kernel(const SlotsParams p) {
  grid_dep_wait();
  grid_dep_launch();
  slots_fill_body(p, blockIdx.x, gridDim.x);
}

// ------------------------------------------------------------------------------------ rotary positions + append
// A unit of work is 16 dims of one head of one token, two 16-byte pieces that a thread reads, turns and writes:
// with the halves layout the pieces of dims 8 c .. and rot / 2 + 8 c .. (the two members of eight pairs), else 32
// consecutive bytes.  Bound by HBM (every q, k, v value is read and written once); the cosines and sines of a
// token, the only costly arithmetic (one 64-bit product and reduction each), are formed once per token and shared
// by all its heads through shared memory.  16384 tokens of 64 + 8 heads: 116 to 122 us, 5.5 to 5.8 TB/s (0.85 to 0.90 of
// the measured copy rate), into the 8-bit cache 122; 40 tokens of 32 + 8 heads: 3 us (8-bit 3.5), a launch and one trip to memory.
template <int D, bool KV8>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const RopeParams p, const int interleaved) {
  constexpr int UPH = D / 16;  // units per head
  __shared__ float2 s_cs[kRopeMaxTile][D / 2];
  __shared__ int s_pos[kRopeMaxTile], s_slot[kRopeMaxTile];
  grid_dep_wait();
  grid_dep_launch();
  const int heads = p.Hq + 2 * p.Hkv, per_tok = heads * UPH, rot_units = p.half / 8;
  for (int t0 = blockIdx.x * p.tile; t0 < p.T; t0 += gridDim.x * p.tile) {
    const int nt = min(p.tile, p.T - t0);
    for (int i = threadIdx.x; i < nt * p.half; i += kRopeThreads) {
      const int tk = i / p.half, j = i - tk * p.half;
      // angle / (2 pi) reduced to [-1/2, 1/2] in 64 bits: far positions lose nothing
      const double turns = (double)p.positions[t0 + tk] * (double)p.inv_freq[j] * 0.15915494309189533577;
      float s, c;
      sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
      s_cs[tk][j] = make_float2(c * p.magnitude, s * p.magnitude);
    }
    if ((int)threadIdx.x < nt) {
      s_pos[threadIdx.x] = p.positions[t0 + threadIdx.x];
      s_slot[threadIdx.x] = p.slots[t0 + threadIdx.x];
    }
    __syncthreads();
    const int n = nt * per_tok;
    for (int u0 = threadIdx.x; u0 < n; u0 += kRopeThreads * kRopeBatch) {
      uint4 a[kRopeBatch], b[kRopeBatch];
      int tk[kRopeBatch], head[kRopeBatch], c[kRopeBatch], d_lo[kRopeBatch], d_hi[kRopeBatch];
#pragma unroll
      for (int i = 0; i < kRopeBatch; ++i) {
        const int u = u0 + i * kRopeThreads;
        tk[i] = -1;
        if (u >= n) continue;
        const int tok = u / per_tok, e = u - tok * per_tok;
        if (s_pos[tok] < 0) continue;  // padding
        tk[i] = tok;
        head[i] = e / UPH;
        c[i] = e % UPH;
        const bool turned_halves = !interleaved && c[i] < rot_units;
        d_lo[i] = turned_halves ? 8 * c[i] : 16 * c[i];
        d_hi[i] = turned_halves ? p.half + 8 * c[i] : 16 * c[i] + 8;
        const size_t t = (size_t)(t0 + tok);
        const uint16_t* src = head[i] < p.Hq           ? p.q + t * p.q_stride + (size_t)head[i] * D
                              : head[i] < p.Hq + p.Hkv ? p.k + t * p.k_stride + (size_t)(head[i] - p.Hq) * D
                                                       : p.v + t * p.v_stride + (size_t)(head[i] - p.Hq - p.Hkv) * D;
        a[i] = *reinterpret_cast<const uint4*>(src + d_lo[i]);
        b[i] = *reinterpret_cast<const uint4*>(src + d_hi[i]);
      }
#pragma unroll
      for (int i = 0; i < kRopeBatch; ++i) {
        if (tk[i] < 0) continue;
        const bool is_q = head[i] < p.Hq, is_v = head[i] >= p.Hq + p.Hkv;
        float x[8], y[8];
        unpack8(a[i], x);
        unpack8(b[i], y);
        if (!is_v && c[i] < rot_units) {
          const float2* cs = &s_cs[tk[i]][8 * c[i]];
          if (interleaved) {
#pragma unroll
            for (int m = 0; m < 4; ++m) {
              const float2 w0 = cs[m], w1 = cs[4 + m];
              const float x0 = x[2 * m], y0 = y[2 * m];
              x[2 * m] = x0 * w0.x - x[2 * m + 1] * w0.y;
              x[2 * m + 1] = x[2 * m + 1] * w0.x + x0 * w0.y;
              y[2 * m] = y0 * w1.x - y[2 * m + 1] * w1.y;
              y[2 * m + 1] = y[2 * m + 1] * w1.x + y0 * w1.y;
            }
          } else {
#pragma unroll
            for (int m = 0; m < 8; ++m) {
              const float2 w = cs[m];
              const float x0 = x[m];
              x[m] = x0 * w.x - y[m] * w.y;
              y[m] = y[m] * w.x + x0 * w.y;
            }
          }
        }
        if (is_q) {
          uint16_t* dst = p.q_out + (size_t)(t0 + tk[i]) * p.q_out_stride + (size_t)head[i] * D;
          *reinterpret_cast<uint4*>(dst + d_lo[i]) = pack8_bf16(x);
          *reinterpret_cast<uint4*>(dst + d_hi[i]) = pack8_bf16(y);
        } else {
          const int slot = s_slot[tk[i]];
          if (slot < 0 || slot >= p.num_slots) continue;
          const int h = head[i] - p.Hq - (is_v ? p.Hkv : 0);
          const int64_t at = (int64_t)(slot >> p.bs_log2) * p.bstr + (int64_t)h * p.hstr +
                             (int64_t)(slot & ((1 << p.bs_log2) - 1)) * p.tstr;
          uint8_t* cache = is_v ? p.v_cache : p.k_cache;
          if (KV8) {
            const float sc = is_v ? p.v_scale : p.k_scale;
            *reinterpret_cast<uint2*>(cache + at + d_lo[i]) = pack8_e4m3(x, sc);
            *reinterpret_cast<uint2*>(cache + at + d_hi[i]) = pack8_e4m3(y, sc);
          } else {
            *reinterpret_cast<uint4*>(cache + 2 * (at + d_lo[i])) = is_v ? a[i] : pack8_bf16(x);
            *reinterpret_cast<uint4*>(cache + 2 * (at + d_hi[i])) = is_v ? b[i] : pack8_bf16(y);
          }
        }
      }
    }
    __syncthreads();  // the tile's cosines are consumed before the next tile's are written
  }
}

// ------------------------------------------------------------------------------------ verification
struct VerifyParams {
  const float *target, *draft, *uniforms;
  const int32_t *tokens, *parents, *tree_sizes;
  int32_t *path, *out_tokens, *num_accepted;
  int64_t t_seq, t_node, d_seq, d_node;
  int32_t B, N, V;
};

constexpr int kVerifyThreads = 512, kVerifyMaxCluster = 16;  // most threads of a CTA, most CTAs of a cluster
constexpr int kVerifyTile = 512;  // values whose weights are summed by one warp at a time: 16 per lane
constexpr int kVerifyMaxTiles = (1 << 20) / kVerifyTile;

// ---- double-float arithmetic: an unevaluated sum hi + lo of two fp32 values, 2^-46 relative or better for the sums of
// non-negative terms formed here.  fp64 instructions issue at about 1 / 60 of the fp32 rate on this part (measured: a
// pass in fp64 took 0.45 weights per cycle and SM, 1/6 of what HBM delivers).
struct Df {
  float hi, lo;
};
__device__ __forceinline__ Df two_sum(float a, float b) {  // exact (error-free transformation, Knuth)
  const float s = __fadd_rn(a, b), bb = __fsub_rn(s, a);
  return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, bb)), __fsub_rn(b, bb))};
}
__device__ __forceinline__ Df df_add(Df a, Df b) {
  const Df s = two_sum(a.hi, b.hi);
  const float e = __fadd_rn(s.lo, __fadd_rn(a.lo, b.lo)), h = __fadd_rn(s.hi, e);
  return {h, __fsub_rn(e, __fsub_rn(h, s.hi))};
}
__device__ __forceinline__ bool df_greater(Df a, Df b) { return a.hi > b.hi || (a.hi == b.hi && a.lo > b.lo); }
__device__ __forceinline__ Df df_times(Df a, float b) {
  const float m = __fmul_rn(a.hi, b), e = __fmaf_rn(a.lo, b, __fmaf_rn(a.hi, b, -m)), h = __fadd_rn(m, e);
  return {h, __fsub_rn(e, __fsub_rn(h, m))};
}
__device__ __forceinline__ Df df_shfl(Df v, int src) {
  return {__shfl_sync(0xffffffffu, v.hi, src), __shfl_sync(0xffffffffu, v.lo, src)};
}
__device__ __forceinline__ Df df_shfl_up1(Df v) {
  return {__shfl_up_sync(0xffffffffu, v.hi, 1), __shfl_up_sync(0xffffffffu, v.lo, 1)};
}
// A draft probability: NaN counts as 0, like a negative value (of the target's, df_weight and the sums below see to that).
__device__ __forceinline__ float draft_prob(float q) { return fmaxf(q, 0.f); }
// max(p - s q, 0); NaN counts as 0
__device__ __forceinline__ Df df_weight(float p, float q, Df s) {
  const float m = __fmul_rn(s.hi, q);                                  // s q = m + e
  const float e = __fmaf_rn(s.lo, q, __fmaf_rn(s.hi, q, -m));
  const Df d = two_sum(p, -m);
  const float l = __fsub_rn(d.lo, e), h = __fadd_rn(d.hi, l);
  return h > 0.f ? Df{h, __fsub_rn(l, __fsub_rn(h, d.hi))} : Df{0.f, 0.f};
}
__device__ __forceinline__ Df df_shfl_xor(Df v, int o) {
  return {__shfl_xor_sync(0xffffffffu, v.hi, o), __shfl_xor_sync(0xffffffffu, v.lo, o)};
}
__device__ __forceinline__ Df df_warp_scan(Df v, int lane) {  // inclusive
  for (int o = 1; o < 32; o <<= 1) {
    const Df u = {__shfl_up_sync(0xffffffffu, v.hi, o), __shfl_up_sync(0xffffffffu, v.lo, o)};
    if (lane >= o) v = df_add(v, u);
  }
  return v;
}

// What CTA 0 tells the cluster to do next.
struct VerifyCommand {
  int op;       // 0 stop, 1 sum the weights of `node`, 2 sum them and draw the last token
  int node;
  int drops;    // without draft probabilities: refused siblings whose tokens have left the weights
  int count;    // drafts accepted so far
  Df spent;     // S: weights are max(p - S q, 0)
  float u;      // uniform number of the last token
  int pad;
};

// One cluster of CTAs per sequence.  CTA 0 walks down the tree (a warp, from the few values per node that it
// gathered at the start); whenever the mass of the weights is needed (a refusal with draft probabilities, the last
// token) it sends a command to the cluster, every CTA sums its share of the vocabulary, and all exchange their sums
// through distributed shared memory.  Only rows that such a pass needs are read: one or two per sequence, however
// many nodes there are.  Bound by HBM for many sequences (two rows of V fp32 values each), by latency for few
// (gather, walk, pass and draw follow one another), which is why a sequence is spread over several CTAs then.  128
// sequences of 16 nodes and 128256 values: 50.5 us (chosen drafts 37.6), 4 of 5 nodes and 152064 values: 11.7 us (12.2).  The first reads 99 MB (15 us): a
// third of a warp's time goes by at the cluster's barriers while CTA 0 gathers and walks, the issue slots are 46 % busy with
// the two-float sums, and sequences that need a second pass are the tail.
//
// Weights and their sums are double-floats: the drawn index depends on a cumulative sum of up to 2^20 weights, and an
// fp32 sum would move its borders by more than the smallest weights.
__global__ void __launch_bounds__(kVerifyThreads, 2) verify_kernel(const VerifyParams p, const int cluster) {
  __shared__ int s_token[kTreeMaxNodes], s_parent[kTreeMaxNodes];
  __shared__ float s_p[kTreeMaxNodes], s_q[kTreeMaxNodes], s_u[kTreeMaxNodes];
  __shared__ uint8_t s_drop[kTreeMaxNodes];
  __shared__ int s_drop_tok[kTreeMaxNodes];          // tokens that have left the weights (same in every CTA)
  __shared__ VerifyCommand s_cmd;
  __shared__ Df s_part[kVerifyMaxCluster];           // sum of each CTA's share
  __shared__ Df s_tile[kVerifyMaxTiles];
  __shared__ uint32_t s_bits[(1 << 20) / 32 / 8 + 1];
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5, threads = blockDim.x, warps = threads >> 5;
  const int rank = cluster > 1 ? (int)cluster_rank() : 0;
  const int b = blockIdx.x / cluster;
  grid_dep_wait();
  grid_dep_launch();
  if (cluster > 1) cluster_arrive();  // (waited for before the first write to another CTA's memory)
  const int N = p.N, V = p.V;
  const int n = p.tree_sizes ? min(max(0, p.tree_sizes[b]), N) : N;
  const float* target = p.target + (int64_t)b * p.t_seq;
  const float* draft = p.draft ? p.draft + (int64_t)b * p.d_seq : nullptr;
  // this CTA's share of the vocabulary, in whole tiles
  const int tiles_all = (V + kVerifyTile - 1) / kVerifyTile, per = (tiles_all + cluster - 1) / cluster;
  const int tile0 = min(tiles_all, rank * per), ntile = min(tiles_all, tile0 + per) - tile0;
  const int v_lo = tile0 * kVerifyTile, v_hi = min(V, v_lo + ntile * kVerifyTile);

  if (rank == 0) {
    for (int i = tid; i < N; i += threads) {
      int par = -1, x = -1;
      float pp = 0.f, qq = 0.f;
      if (i > 0 && i < n) {
        par = p.parents ? p.parents[(size_t)b * N + i] : i - 1;
        x = p.tokens[(size_t)b * N + i];
        if (par >= i || par < 0 || x < 0 || x >= V) par = -1;
        if (par >= 0) {
          pp = target[(int64_t)par * p.t_node + x];
          if (draft) qq = draft[(int64_t)par * p.d_node + x];
        }
      }
      s_parent[i] = par;
      s_token[i] = x;
      s_p[i] = pp;
      s_q[i] = draft_prob(qq);
      s_u[i] = i < n ? p.uniforms[(size_t)b * N + i] : 0.f;
      s_drop[i] = 0;
      p.path[(size_t)b * N + i] = i == 0 && n > 0 ? 0 : -1;
      p.out_tokens[(size_t)b * N + i] = -1;
    }
  }
  __syncthreads();
  if (cluster > 1) cluster_wait();

  // the walk's state, in warp 0 of CTA 0 (the same in every lane)
  int cur = 0, last = 0, count = 0;
  Df spent = {0.f, 0.f}, mass = {1.f, 0.f};
  const float u_last = rank == 0 && n > 0 ? s_u[0] : 0.f;

  for (;;) {
    if (rank == 0 && wid == 0) {
      int op = n > 0 ? 2 : 0, drops = 0;
      while (n > 0) {
        int next = N;  // the next child of `cur`
        for (int c0 = (last + 1) & ~31; c0 < n && next == N; c0 += 32) {
          const int i = c0 + lane;
          const uint32_t hit = __ballot_sync(0xffffffffu, i > last && i < n && s_parent[i] == cur);
          if (hit) next = c0 + __ffs(hit) - 1;
        }
        if (next == N) break;
        last = next;
        const int x = s_token[next];
        Df w = {s_p[next], 0.f}, bar = df_times(mass, s_u[next]);
        if (draft) {
          const float q = s_q[next];
          w = df_weight(w.hi, q, spent);
          bar = df_times(bar, q);
        } else {
          bool gone = false;  // the token was refused already
          for (int c0 = 0; c0 < next; c0 += 32)
            gone |= __any_sync(0xffffffffu, c0 + lane < next && s_drop[c0 + lane] && s_token[c0 + lane] == x);
          if (gone || !(w.hi > 0.f)) w.hi = 0.f;
        }
        if (df_greater(w, bar)) {
          cur = next;
          spent = Df{0.f, 0.f};
          mass = Df{1.f, 0.f};
          ++count;
          for (int i = lane; i < n; i += 32) s_drop[i] = 0;
          __syncwarp();
          if (lane == 0) {
            p.path[(size_t)b * N + count] = next;
            p.out_tokens[(size_t)b * N + count - 1] = x;
          }
        } else if (draft) {
          spent = df_add(spent, mass);
          // another sibling to ask needs the new mass; without one the pass is the last
          bool more = false;
          for (int c0 = (last + 1) & ~31; c0 < n; c0 += 32)
            more |= __any_sync(0xffffffffu, c0 + lane > last && c0 + lane < n && s_parent[c0 + lane] == cur);
          if (more) op = 1;
          break;
        } else {
          mass = df_add(mass, Df{-w.hi, -w.lo});
          if (lane == 0) s_drop[next] = 1;
          __syncwarp();
        }
      }
      if (!draft && op == 2) {  // the refused siblings' tokens, for every CTA
        for (int c0 = 0; c0 < n; c0 += 32) {
          const bool d = c0 + lane < n && s_drop[c0 + lane];
          const uint32_t m = __ballot_sync(0xffffffffu, d);
          const int at = drops + __popc(m & ((1u << lane) - 1));
          if (d)
            for (int r = 0; r < cluster; ++r) {
              if (cluster > 1) st_cluster(map_cluster(smem_u32(&s_drop_tok[at]), r), s_token[c0 + lane]);
              else s_drop_tok[at] = s_token[c0 + lane];
            }
          drops += __popc(m);
        }
      }
      if (lane < cluster) {
        if (cluster > 1) {
          const uint32_t at = map_cluster(smem_u32(&s_cmd), lane);
          st_cluster(at, op);
          st_cluster(at + 4, cur);
          st_cluster(at + 8, drops);
          st_cluster(at + 12, count);
          st_cluster(at + 16, spent.hi);
          st_cluster(at + 20, spent.lo);
          st_cluster(at + 24, u_last);
        } else {
          s_cmd.op = op;
          s_cmd.node = cur;
          s_cmd.drops = drops;
          s_cmd.count = count;
          s_cmd.spent = spent;
          s_cmd.u = u_last;
        }
      }
      if (lane == 0) p.num_accepted[b] = count;
    }
    __syncwarp();
    if (cluster > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
    const int op = s_cmd.op;
    if (op == 0) return;
    const float* pr = target + (int64_t)s_cmd.node * p.t_node;
    const float* qr = draft ? draft + (int64_t)s_cmd.node * p.d_node : nullptr;
    Df S = s_cmd.spent;
    if (S.hi == 0.f) qr = nullptr;
    int drops = s_cmd.drops;

    for (int attempt = 0;; ++attempt) {
      if (drops > 0) {
        for (int i = tid; i < (v_hi - v_lo + 31) / 32; i += threads) s_bits[i] = 0u;
        __syncthreads();
        for (int i = tid; i < drops; i += threads) {
          const int x = s_drop_tok[i] - v_lo;
          if (x >= 0 && x < v_hi - v_lo) atomicOr(&s_bits[x >> 5], 1u << (x & 31));
        }
        __syncthreads();
      }
      auto weight = [&](int v, float pv, float qv) {
        Df w = qr ? df_weight(pv, qv, S) : Df{pv > 0.f ? pv : 0.f, 0.f};
        if (drops > 0 && (s_bits[(v - v_lo) >> 5] >> ((v - v_lo) & 31) & 1u)) w = Df{0.f, 0.f};
        return w;
      };
      auto add_to = [](Df& s, Df w) {  // (the low parts may grow a little: they are folded in by the next df_add)
        const Df a = two_sum(s.hi, w.hi);
        s = Df{a.hi, __fadd_rn(s.lo, __fadd_rn(a.lo, w.lo))};
      };
      // Sums of the tiles' weights.  kKind: 0 the target's values (3: without the tokens that left), 1 p - q (one refusal: s = 1, the difference needs no
      // product), 2 p - s q.  The weights are added as they come, without bringing hi and lo apart first.
      auto sum_tiles = [&](auto kind) {
        constexpr int kKind = decltype(kind)::value;
        for (int k = wid; k < ntile; k += warps) {
          const int v0 = v_lo + k * kVerifyTile + lane;
          Df s0 = {0.f, 0.f}, s1 = {0.f, 0.f};
          if (v0 - lane + kVerifyTile <= v_hi) {
            float pv[16], qv[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) pv[e] = pr[v0 + 32 * e];
            if (kKind == 1 || kKind == 2) {
#pragma unroll
              for (int e = 0; e < 16; ++e) qv[e] = qr[v0 + 32 * e];
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              Df w;
              bool some;
              if (kKind == 0 || kKind == 3) {
                w = Df{pv[e], 0.f};
                some = pv[e] > 0.f && !(kKind == 3 && (s_bits[(kVerifyTile / 32) * k + e] >> lane & 1u));
              } else if (kKind == 1) {
                w = two_sum(pv[e], -draft_prob(qv[e]));
                some = w.hi > 0.f;
              } else {
                const float q = draft_prob(qv[e]), m = __fmul_rn(S.hi, q);
                w = two_sum(pv[e], -m);
                w.lo = __fsub_rn(w.lo, __fmaf_rn(S.lo, q, __fmaf_rn(S.hi, q, -m)));
                some = __fadd_rn(w.hi, w.lo) > 0.f;
              }
              add_to(e & 1 ? s1 : s0, some ? w : Df{0.f, 0.f});
            }
          } else {
            for (int v = v0; v < min(v_hi, v0 - lane + kVerifyTile); v += 32) add_to(s0, weight(v, pr[v], draft_prob(qr ? qr[v] : 0.f)));
          }
          Df s = df_add(s0, s1);
          for (int o = 16; o; o >>= 1) s = df_add(s, df_shfl_xor(s, o));
          if (lane == 0) s_tile[k] = s;
        }
      };
      if (!qr && drops > 0)
        sum_tiles(std::integral_constant<int, 3>{});
      else if (!qr)
        sum_tiles(std::integral_constant<int, 0>{});
      else if (S.hi == 1.f && S.lo == 0.f)
        sum_tiles(std::integral_constant<int, 1>{});
      else
        sum_tiles(std::integral_constant<int, 2>{});
      __syncthreads();
      if (wid == 0) {  // the share's sum, to every CTA of the cluster
        Df s = {0.f, 0.f};
        for (int k = lane; k < ntile; k += 32) s = df_add(s, s_tile[k]);
        for (int o = 16; o; o >>= 1) s = df_add(s, df_shfl_xor(s, o));
        if (lane < cluster) {
          if (cluster > 1) {
            const uint32_t at = map_cluster(smem_u32(&s_part[rank]), lane);
            st_cluster(at, s.hi);
            st_cluster(at + 4, s.lo);
          } else {
            s_part[0] = s;
          }
        }
      }
      __syncwarp();
      if (cluster > 1) {
        cluster_arrive();
        cluster_wait();
      } else {
        __syncthreads();
      }
      // shares' sums in order, one per lane (the same in every warp of every CTA)
      const Df part = lane < cluster ? s_part[lane] : Df{0.f, 0.f};
      const Df part_upto = df_warp_scan(part, lane), sum = df_shfl(part_upto, 31);
      if (op == 1) {  // the walk goes on with the new mass
        mass = sum;
        break;
      }
      if (!(sum.hi > 0.f && sum.hi <= 1e30f)) {
        if (attempt == 0) {  // nothing is left: the target's own row
          S = Df{0.f, 0.f};
          qr = nullptr;
          drops = 0;
          if (cluster > 1) {  // the sums of this attempt have been read before they are written again
            cluster_arrive();
            cluster_wait();
          } else {
            __syncthreads();
          }
          continue;
        }
        if (rank == 0 && tid == 0) p.out_tokens[(size_t)b * N + s_cmd.count] = 0;
        return;
      }
      if (wid != 0) return;
      // ---- draw: the first lane whose cumulative sum exceeds the target value, of the CTAs' shares, of runs of tiles,
      // of the tiles of a run, of runs of 16 values, of those values.  Where rounding leaves the target beyond all
      // sums, the last one with weight is taken.
      Df t = df_times(sum, s_cmd.u);
      auto first_over = [&](Df upto, bool some) {
        uint32_t m = __ballot_sync(0xffffffffu, some && df_greater(upto, t));
        if (m) return __ffs(m) - 1;
        m = __ballot_sync(0xffffffffu, some);
        return m ? 31 - __clz(m) : 0;
      };
      // moves the origin to the start of the range that lane `src` holds; `upto` are the lanes' inclusive sums
      auto enter = [&](Df upto, int src) {
        Df before = df_shfl_up1(upto);
        if (lane == 0) before = Df{0.f, 0.f};
        before = df_shfl(before, src);
        t = df_add(t, Df{-before.hi, -before.lo});
      };
      int src = first_over(part_upto, part.hi > 0.f);
      if (src != rank) return;
      enter(part_upto, src);
      const int run = (ntile + 31) / 32;
      Df s = {0.f, 0.f};
      for (int k = lane * run; k < min(ntile, lane * run + run); ++k) s = df_add(s, s_tile[k]);
      Df upto = df_warp_scan(s, lane);
      src = first_over(upto, s.hi > 0.f);
      enter(upto, src);
      int tile = src * run;
      for (int k0 = tile;; k0 += 32) {  // (one round unless a share has over 1024 tiles)
        const int k_hi = min(ntile, src * run + run);
        s = k0 + lane < k_hi ? s_tile[k0 + lane] : Df{0.f, 0.f};
        upto = df_warp_scan(s, lane);
        const int f = first_over(upto, s.hi > 0.f);
        const bool over = df_greater(df_shfl(upto, 31), t);
        tile = k0 + f;
        if (over || k0 + 32 >= k_hi) {
          enter(upto, f);
          break;
        }
        const Df all = df_shfl(upto, 31);
        t = df_add(t, Df{-all.hi, -all.lo});
      }
      const int v0 = v_lo + tile * kVerifyTile;
      float pv[16], qv[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int v = v0 + 16 * lane + e;
        pv[e] = v < v_hi ? pr[v] : 0.f;
        qv[e] = qr && v < v_hi ? qr[v] : 0.f;
      }
      s = Df{0.f, 0.f};
      Df s1 = {0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const int v = v0 + 16 * lane + e;
        if (v < v_hi) add_to(s, weight(v, pv[e], draft_prob(qv[e])));
        if (v + 1 < v_hi) add_to(s1, weight(v + 1, pv[e + 1], draft_prob(qv[e + 1])));
      }
      s = df_add(s, s1);
      upto = df_warp_scan(s, lane);
      src = first_over(upto, s.hi > 0.f);
      enter(upto, src);
      const int run_lo = v0 + 16 * src, v = run_lo + lane;
      s = lane < 16 && v < v_hi ? weight(v, pr[v], draft_prob(qr ? qr[v] : 0.f)) : Df{0.f, 0.f};
      src = first_over(df_warp_scan(s, lane), s.hi > 0.f);
      if (lane == 0) p.out_tokens[(size_t)b * N + s_cmd.count] = min(run_lo + src, V - 1);
      return;
    }
    // (op 1) the next command is written by CTA 0 after it has read the sums; the other CTAs read theirs before
    // they wait for it, and their parts are not written again before that
  }
}

// ------------------------------------------------------------------------------------ accepted branch
struct KeepParams {
  uint8_t *k_cache, *v_cache;
  const int32_t *block_table, *base_lens, *path, *num_accepted;
  int32_t* context_lens_out;  // may be NULL
  int64_t bstr, hstr, tstr;   // bytes
  int32_t B, N, Hkv, row_vecs, bs_log2, NB, MB;  // row_vecs: 16-byte pieces of a row
};

constexpr int kKeepThreads = 128, kKeepBatch = 8;

// A thread owns one 16-byte column of a sequence (cache, head, piece of the row) through all moves: entries of the
// path increase, so a move's source is never below its target, and a source that has not been read yet is never a
// target of an earlier move; a batch of moves is read before it is written.  HBM-bound (each row read and written
// once): 512 sequences, 8 heads, up to 31 moves of 256-byte rows, take 16.8 us, 4.7 TB/s (8-bit: 8.2); for few sequences the chain path ->
// table -> rows is what it takes (8 sequences: 2.8 us).
__global__ void __launch_bounds__(kKeepThreads) keep_path_kernel(const KeepParams p) {
  __shared__ int64_t s_src[kTreeMaxNodes], s_dst[kTreeMaxNodes];
  __shared__ int s_count, s_path[kTreeMaxNodes];
  grid_dep_wait();
  grid_dep_launch();
  const int b = blockIdx.x, tid = threadIdx.x;
  const long long cap = (long long)p.MB << p.bs_log2;
  const int acc = min(max(0, p.num_accepted[b]), p.N - 1);
  const int32_t* path = p.path + (size_t)b * p.N;
  if (tid == 0) s_count = acc + 1;
  __syncthreads();
  for (int j = tid; j < p.N; j += kKeepThreads) {  // how far the branch is well formed (entries are read beside the count)
    const int node = path[j], before = j ? path[j - 1] : -1;
    s_path[j] = node;
    if (j <= acc && (node <= before || node >= p.N || (j == 0 && node != 0))) atomicMin(&s_count, j);
  }
  __syncthreads();
  const int count = s_count;
  const long long base = max(0, p.base_lens[b]);
  if (blockIdx.y == 0 && tid == 0 && p.context_lens_out) p.context_lens_out[b] = (int)min(base + count, 0x7fffffffLL);
  for (int j = tid; j < count; j += kKeepThreads) {
    int64_t src = -1, dst = -1;
    const long long ts = base + s_path[j], td = base + j;
    if (ts != td && ts < cap) {
      const int bsrc = p.block_table[(size_t)b * p.MB + (ts >> p.bs_log2)];
      const int bdst = p.block_table[(size_t)b * p.MB + (td >> p.bs_log2)];
      const int mask = (1 << p.bs_log2) - 1;
      if (bsrc >= 0 && bsrc < p.NB && bdst >= 0 && bdst < p.NB) {
        src = (int64_t)bsrc * p.bstr + (ts & mask) * p.tstr;
        dst = (int64_t)bdst * p.bstr + (td & mask) * p.tstr;
      }
    }
    s_src[j] = src;
    s_dst[j] = dst;
  }
  __syncthreads();
  const int cols = 2 * p.Hkv * p.row_vecs;
  for (int c = blockIdx.y * kKeepThreads + tid; c < cols; c += gridDim.y * kKeepThreads) {
    const int piece = c % p.row_vecs, hk = c / p.row_vecs, h = hk % p.Hkv;
    uint8_t* cache = (hk >= p.Hkv ? p.v_cache : p.k_cache) + (int64_t)h * p.hstr + 16 * piece;
    for (int j0 = 1; j0 < count; j0 += kKeepBatch) {
      uint4 w[kKeepBatch];
#pragma unroll
      for (int i = 0; i < kKeepBatch; ++i)
        if (j0 + i < count && s_src[j0 + i] >= 0) w[i] = *reinterpret_cast<const uint4*>(cache + s_src[j0 + i]);
#pragma unroll
      for (int i = 0; i < kKeepBatch; ++i)
        if (j0 + i < count && s_src[j0 + i] >= 0) *reinterpret_cast<uint4*>(cache + s_dst[j0 + i]) = w[i];
    }
  }
}

}  // namespace ooco
