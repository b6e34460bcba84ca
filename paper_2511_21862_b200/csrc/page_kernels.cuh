// Kernels that share and give back pages of the cache between sequences: block tables, holder counts, the free list.
// Whole-number bookkeeping, bound by latency: a few dependent trips to memory, so each call is one launch, one CTA or one
// thread-block cluster whose barriers order the phases.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "cta_util.cuh"
#include "ptx.cuh"

namespace ooco {

constexpr int kPagesStatusBadBlock = 4, kPagesStatusRefused = 128;
constexpr int kPagesThreads = 1024, kPagesWarps = kPagesThreads / 32, kPagesMaxCluster = 16;
constexpr int kPagesSegment = 256;  // table entries of one row that a warp handles at a time, 8 per lane

struct PagesParams {
  const int32_t *parents;          // fork: the parents; release: the rows
  const int32_t *children;         // fork only
  const int32_t *lens;             // fork: shared_lens, release: keep_lens; may be NULL
  const int32_t *context_lens, *blocks_held, *free_head, *shares;
  int32_t *block_table, *free_ids;
  int32_t *context_lens_out, *blocks_held_out, *free_head_out, *shares_out;  // equal to the inputs where in place
  int32_t *copy_src, *copy_dst, *granted, *status;
  int32_t *ws_a, *ws_b;            // [n] fork: full blocks of each fork (-1: refused), -; release: first and end entry given back
  int32_t n, B, NB, MB, bs_log2, num_free;
};

__device__ __forceinline__ void pages_flag(const PagesParams& p, int bit) {
  if (p.status) atomicOr(p.status, bit);
}
__device__ __forceinline__ void pages_sync(int cluster) {
  if (cluster > 1) {
    cluster_arrive();
    cluster_wait();
  } else {
    __syncthreads();
  }
}

// The outputs that are not in place start as copies of the inputs.
__device__ __forceinline__ void pages_copy_state(const PagesParams& p, int tid, int threads) {
  if (p.shares_out != p.shares) {
    const bool wide = !(((uintptr_t)p.shares | (uintptr_t)p.shares_out) & 15);
    const int n4 = wide ? p.NB / 4 : 0;
    for (int i = tid; i < n4; i += threads) reinterpret_cast<int4*>(p.shares_out)[i] = reinterpret_cast<const int4*>(p.shares)[i];
    for (int i = 4 * n4 + tid; i < p.NB; i += threads) p.shares_out[i] = p.shares[i];
  }
  if (p.context_lens_out != p.context_lens)
    for (int i = tid; i < p.B; i += threads) p.context_lens_out[i] = p.context_lens[i];
  if (p.blocks_held_out != p.blocks_held)
    for (int i = tid; i < p.B; i += threads) p.blocks_held_out[i] = p.blocks_held[i];
}

// Bit maps over the rows in shared memory: rows named (once), named again, and (fork) named as parents.
struct RowMaps {
  uint32_t *once, *again, *parent;
  int words;
};
__device__ __forceinline__ RowMaps row_maps(uint32_t* smem, int B, bool with_parents) {
  RowMaps m;
  m.words = (B + 31) / 32;
  m.once = smem;
  m.again = smem + m.words;
  m.parent = smem + 2 * m.words;
  for (int i = threadIdx.x; i < m.words * (with_parents ? 3 : 2); i += kPagesThreads) smem[i] = 0u;
  __syncthreads();
  return m;
}
__device__ __forceinline__ void mark_row(const RowMaps& m, int row, int B) {
  if (row < 0 || row >= B) return;
  const uint32_t bit = 1u << (row & 31);
  if (atomicOr(&m.once[row >> 5], bit) & bit) atomicOr(&m.again[row >> 5], bit);
}
__device__ __forceinline__ bool has_row(const uint32_t* map, int row) { return (map[row >> 5] >> (row & 31)) & 1u; }

// ------------------------------------------------------------------------------------ fork
// CTA 0 decides who is granted (a prefix sum of the needed blocks over the forks) and writes what there is one of per
// fork, while the other CTAs copy the state that is not updated in place; then all copy table entries and count holders,
// a warp per (fork, 256 entries).  Counts are whole numbers: the order of the atomics does not matter.
__global__ void __launch_bounds__(kPagesThreads, 1) fork_pages_kernel(const PagesParams p, const int cluster) {
  extern __shared__ uint32_t s_maps[];
  __shared__ long long s_warp[32];
  const int tid = threadIdx.x, lane = tid & 31;
  const int rank = cluster > 1 ? (int)cluster_rank() : 0;
  grid_dep_wait();
  grid_dep_launch();
  pages_copy_state(p, rank * kPagesThreads + tid, cluster * kPagesThreads);
  if (cluster > 1) cluster_arrive();  // (CTA 0 waits for the copies before it writes the children's lengths)
  if (rank == 0) {
    const RowMaps m = row_maps(s_maps, p.B, true);
    for (int c = tid; c < p.n; c += kPagesThreads) {
      mark_row(m, p.children[c], p.B);
      const int par = p.parents[c];
      if (par >= 0 && par < p.B) atomicOr(&m.parent[par >> 5], 1u << (par & 31));
    }
    const int head0 = max(0, *p.free_head);
    if (cluster > 1) cluster_wait();
    __syncthreads();
    long long run = 0;  // blocks needed by the forks so far
    int taken = 0;      // ... and handed out, by this thread's forks
    for (int c0 = 0; c0 < p.n; c0 += kPagesThreads) {
      const int c = c0 + tid;
      int par = 0, kid = 0, L = 0, full = 0, need = 0;
      bool ok = false;
      if (c < p.n) {
        par = p.parents[c];
        kid = p.children[c];
        ok = par >= 0 && par < p.B && kid >= 0 && kid < p.B && !has_row(m.again, kid) && !has_row(m.parent, kid) &&
             p.blocks_held[kid] <= 0;
        if (ok) {
          L = max(0, p.context_lens[par]);
          if (p.lens) L = min(L, max(0, p.lens[c]));
          full = L >> p.bs_log2;
          need = (L & ((1 << p.bs_log2) - 1)) ? 1 : 0;
          ok = full + need <= min(p.blocks_held[par], p.MB);
          if (!ok) need = 0;
        }
      }
      long long total;
      const long long upto = head0 + run + block_scan(need, s_warp, &total);
      run += total;
      if (c < p.n) {
        if (ok && need && upto > p.num_free) ok = false;
        int src = -1, dst = -1;
        if (ok && need) {
          ++taken;
          src = p.block_table[(size_t)par * p.MB + full];
          dst = p.free_ids[upto - 1];
          p.block_table[(size_t)kid * p.MB + full] = dst;
          if (src < 0 || src >= p.NB || dst < 0 || dst >= p.NB) {
            pages_flag(p, kPagesStatusBadBlock);
            src = dst = -1;
          }
        }
        if (ok) {
          p.context_lens_out[kid] = L;
          p.blocks_held_out[kid] = full + need;
        } else {
          pages_flag(p, kPagesStatusRefused);
        }
        p.copy_src[c] = src;
        p.copy_dst[c] = dst;
        p.granted[c] = ok ? 1 : 0;
        p.ws_a[c] = ok ? full : -1;
      }
    }
    long long all;
    block_scan(taken, s_warp, &all);
    if (tid == 0) *p.free_head_out = head0 + (int)all;
  } else {
    cluster_wait();
  }
  pages_sync(cluster);
  const int segs = (p.MB + kPagesSegment - 1) / kPagesSegment, warps = cluster * kPagesWarps;
  const long long units = (long long)p.n * segs;
  bool bad = false;
  for (long long u = rank * kPagesWarps + (tid >> 5); u < units; u += warps) {
    const int c = (int)(u / segs), j0 = (int)(u - (long long)c * segs) * kPagesSegment;
    const int full = p.ws_a[c];
    if (j0 >= full) continue;
    const int32_t* src = p.block_table + (size_t)p.parents[c] * p.MB;
    int32_t* dst = p.block_table + (size_t)p.children[c] * p.MB;
    int id[kPagesSegment / 32];
#pragma unroll
    for (int k = 0; k < kPagesSegment / 32; ++k) {
      const int j = j0 + 32 * k + lane;
      id[k] = j < full ? src[j] : 0;
    }
#pragma unroll
    for (int k = 0; k < kPagesSegment / 32; ++k) {
      const int j = j0 + 32 * k + lane;
      if (j >= full) continue;
      dst[j] = id[k];
      if (id[k] >= 0 && id[k] < p.NB)
        atomicAdd(&p.shares_out[id[k]], 1);
      else
        bad = true;
    }
  }
  if (bad) pages_flag(p, kPagesStatusBadBlock);
}

// ------------------------------------------------------------------------------------ release
// An entry that is given back has the key (index in the list) * MB + (index in the table).  Phases, a cluster barrier
// between each two:
//   1  copies of the state, and per row which entries go                     (CTA 0)
//   2  every entry takes one from its block's count: a count below 0 means that the block is free
//   3  every entry of such a block puts key - 2^31 there by a minimum: the count now says which entry stands first
//   4  every warp, which has a contiguous share of the entries, counts those that stand first
//   5  prefix sums of the warps' counts give every freed block its place in the free list, in the order of the keys; its
//      count becomes 0 (no key's value, so entries that look later see that they do not stand first)
// The order of the atomics changes nothing, and the keys (below 2^30) cannot meet the counts of phase 2 (above -2^30).
__global__ void __launch_bounds__(kPagesThreads, 1) release_pages_kernel(const PagesParams p, const int cluster) {
  extern __shared__ uint32_t s_maps[];
  __shared__ int s_count[kPagesWarps], s_total[kPagesMaxCluster];
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int rank = cluster > 1 ? (int)cluster_rank() : 0;
  grid_dep_wait();
  grid_dep_launch();
  pages_copy_state(p, rank * kPagesThreads + tid, cluster * kPagesThreads);
  const int head0 = min(max(0, *p.free_head), p.num_free);
  if (rank == 0) {
    const RowMaps m = row_maps(s_maps, p.B, false);
    for (int c = tid; c < p.n; c += kPagesThreads) mark_row(m, p.parents[c], p.B);
    __syncthreads();
    for (int c = tid; c < p.n; c += kPagesThreads) {
      const int row = p.parents[c];
      int from = 0, to = 0;
      if (row >= 0 && row < p.B && !has_row(m.again, row)) {
        const int keep = p.lens ? max(0, p.lens[c]) : 0;
        to = min(max(0, p.blocks_held[row]), p.MB);
        from = min(to, (int)(((long long)keep + (1 << p.bs_log2) - 1) >> p.bs_log2));
      } else {
        pages_flag(p, kPagesStatusRefused);
      }
      p.ws_a[c] = from;
      p.ws_b[c] = to;
    }
  }
  pages_sync(cluster);
  if (rank == 0) {  // (behind the copies)
    const RowMaps m = {s_maps, s_maps + (p.B + 31) / 32, nullptr, 0};
    for (int c = tid; c < p.n; c += kPagesThreads) {
      const int row = p.parents[c];
      if (row < 0 || row >= p.B || has_row(m.again, row)) continue;
      p.context_lens_out[row] = min(max(0, p.context_lens[row]), p.lens ? max(0, p.lens[c]) : 0);
      p.blocks_held_out[row] = p.ws_a[c];
    }
  }
  const int segs = (p.MB + kPagesSegment - 1) / kPagesSegment, warps = cluster * kPagesWarps;
  const long long units = (long long)p.n * segs;
  const long long u0 = units * (rank * kPagesWarps + wid) / warps, u1 = units * (rank * kPagesWarps + wid + 1) / warps;
  // visits the warp's entries, 32 table entries at a time: f(block id or -1, key, lane has an entry)
  auto visit = [&](auto f) {
    for (long long u = u0; u < u1; ++u) {
      const int c = (int)(u / segs), j0 = (int)(u - (long long)c * segs) * kPagesSegment;
      const int from = p.ws_a[c], to = p.ws_b[c];
      if (j0 >= to || j0 + kPagesSegment <= from) continue;
      const int32_t* src = p.block_table + (size_t)p.parents[c] * p.MB;
      int id[kPagesSegment / 32];
#pragma unroll
      for (int k = 0; k < kPagesSegment / 32; ++k) {
        const int j = j0 + 32 * k + lane;
        id[k] = j >= from && j < to ? src[j] : -1;
      }
      f(id, (int)((long long)c * p.MB + j0 + lane), c, j0);
    }
  };
  bool bad = false;
  visit([&](const int (&id)[kPagesSegment / 32], int, int c, int j0) {
#pragma unroll
    for (int k = 0; k < kPagesSegment / 32; ++k) {
      if (id[k] >= 0 && id[k] < p.NB) {
        atomicSub(&p.shares_out[id[k]], 1);
      } else {
        const int j = j0 + 32 * k + lane;
        bad |= j >= p.ws_a[c] && j < p.ws_b[c];
      }
    }
  });
  if (bad) pages_flag(p, kPagesStatusBadBlock);
  pages_sync(cluster);
  visit([&](const int (&id)[kPagesSegment / 32], int key, int, int) {
    int left[kPagesSegment / 32];
#pragma unroll
    for (int k = 0; k < kPagesSegment / 32; ++k) left[k] = id[k] >= 0 && id[k] < p.NB ? __ldcg(&p.shares_out[id[k]]) : 0;
#pragma unroll
    for (int k = 0; k < kPagesSegment / 32; ++k)
      if (left[k] < 0) atomicMin(&p.shares_out[id[k]], key + 32 * k + INT32_MIN);
  });
  pages_sync(cluster);
  int mine = 0;  // of the warp
  visit([&](const int (&id)[kPagesSegment / 32], int key, int, int) {
    int left[kPagesSegment / 32];
#pragma unroll
    for (int k = 0; k < kPagesSegment / 32; ++k) left[k] = id[k] >= 0 && id[k] < p.NB ? __ldcg(&p.shares_out[id[k]]) : 0;
#pragma unroll
    for (int k = 0; k < kPagesSegment / 32; ++k) mine += __popc(__ballot_sync(0xffffffffu, left[k] == key + 32 * k + INT32_MIN));
  });
  if (lane == 0) s_count[wid] = mine;
  __syncthreads();
  if (wid == 0) {
    int v = s_count[lane];
    const int own = v;
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += u;
    }
    s_count[lane] = v - own;  // freed by the warps before
    const int sum = __shfl_sync(0xffffffffu, v, 31);
    if (cluster > 1) {
      if (lane < cluster) st_cluster(map_cluster(smem_u32(&s_total[rank]), lane), sum);
    } else if (lane == 0) {
      s_total[0] = sum;
    }
  }
  pages_sync(cluster);
  int before = 0, all = 0;
  for (int r = 0; r < cluster; ++r) {
    if (r < rank) before += s_total[r];
    all += s_total[r];
  }
  const int put = min(all, head0), head1 = head0 - put;  // (ids for which the list has no room are dropped)
  int at = before + s_count[wid];
  visit([&](const int (&id)[kPagesSegment / 32], int key, int, int) {
    int left[kPagesSegment / 32];
#pragma unroll
    for (int k = 0; k < kPagesSegment / 32; ++k) left[k] = id[k] >= 0 && id[k] < p.NB ? __ldcg(&p.shares_out[id[k]]) : 0;
#pragma unroll
    for (int k = 0; k < kPagesSegment / 32; ++k) {
      const bool first = left[k] == key + 32 * k + INT32_MIN;
      const uint32_t m = __ballot_sync(0xffffffffu, first);
      const int place = at + __popc(m & ((1u << lane) - 1));
      if (first) {
        if (place < put) p.free_ids[head1 + place] = id[k];
        p.shares_out[id[k]] = 0;
      }
      at += __popc(m);
    }
  });
  if (rank == 0 && tid == 0) {
    *p.free_head_out = head1;
    if (put < all) pages_flag(p, kPagesStatusRefused);
  }
}

}  // namespace ooco
