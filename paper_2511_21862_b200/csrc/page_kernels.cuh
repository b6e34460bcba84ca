// Kernels that share and give back pages of the cache between sequences: block tables, holder counts, the free list.
// Whole-number bookkeeping in a few phases: one CTA decides per fork or row what is to be done and sums up the table entries that
// this concerns; then all warps share the entries evenly, 16 of them in the registers of a lane at a time.  Few entries are bound
// by latency (dependent trips to memory): one launch of one CTA, or of a thread-block cluster whose barriers order the phases.
// Many: a launch per phase, on all SMs (176000 entries of 512 rows given back: 33 us, 62 in a cluster of 16 CTAs; 512 forks of
// prefixes of 32 rows: 14 and 24; a few forks or rows: 7 to 10).  Of the five launches of that release the decision and the two that
// send atomics (250000 sectors of reductions at L2 each) take 9 to 10 us alone, the two that only look at counts, sum up and place 13
// and 16: every launch finds its entries' owners, loads the entries and looks at their counts anew, one after another (2 to 3 million
// warp instructions at 30 % of the issue slots).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "cta_util.cuh"
#include "ptx.cuh"

namespace ooco {

constexpr int kPagesStatusBadBlock = 4, kPagesStatusRefused = 128;
constexpr int kPagesThreads = 1024, kPagesWarps = kPagesThreads / 32, kPagesMaxCluster = 16;
constexpr int kPagesRound = 16;         // table entries that a lane has in its registers
constexpr int kPagesListInSmem = 4096;  // forks or rows whose entries are looked up in shared memory

struct PagesParams {
  const int32_t *parents;          // fork: the parents; release: the rows
  const int32_t *children;         // fork only
  const int32_t *lens;             // fork: shared_lens, release: keep_lens; may be NULL
  const int32_t *context_lens, *blocks_held, *free_head, *shares;
  int32_t *block_table, *free_ids;
  int32_t *context_lens_out, *blocks_held_out, *free_head_out, *shares_out;  // equal to the inputs where in place
  int32_t *copy_src, *copy_dst, *granted, *status;
  int32_t *ws_from, *ws_off;       // [n] first table entry concerned; [n + 1] entries concerned before each
  int32_t *ws_total;               // [CTAs] blocks freed by each
  int32_t *ws_head;                // [1] free_head as it was (it may be updated in place while late CTAs still need it)
  int32_t n, B, NB, MB, bs_log2, num_free;
  int32_t phase;                   // -1: all phases in this launch, by a cluster of CTAs; else this one, by a grid
};
// The calling CTA among those that share the work.
struct Part {
  int rank, count;
  bool all;  // all phases in this launch
};
__device__ __forceinline__ Part pages_part(const PagesParams& p) {
  const bool all = p.phase < 0;
  return {all && gridDim.x > 1 ? (int)cluster_rank() : (int)blockIdx.x, (int)gridDim.x, all};
}

__device__ __forceinline__ void pages_flag(const PagesParams& p, int bit) {
  if (p.status) atomicOr(p.status, bit);
}
// Between two phases.
__device__ __forceinline__ void pages_sync(const Part& t) {
  if (t.all && t.count > 1) {
    cluster_arrive();
    cluster_wait();
  } else if (t.all) {
    __syncthreads();
  }
}

// The outputs that are not in place start as copies of the inputs: the counts by all CTAs, the lengths by CTA 0.
__device__ __forceinline__ void pages_copy_shares(const PagesParams& p, int tid, int threads) {
  if (p.shares_out == p.shares) return;
  const bool wide = !(((uintptr_t)p.shares | (uintptr_t)p.shares_out) & 15);
  const int n4 = wide ? p.NB / 4 : 0;
  for (int i = tid; i < n4; i += threads) reinterpret_cast<int4*>(p.shares_out)[i] = reinterpret_cast<const int4*>(p.shares)[i];
  for (int i = 4 * n4 + tid; i < p.NB; i += threads) p.shares_out[i] = p.shares[i];
}
__device__ __forceinline__ void pages_copy_lens(const PagesParams& p) {
  if (p.context_lens_out != p.context_lens)
    for (int i = threadIdx.x; i < p.B; i += kPagesThreads) p.context_lens_out[i] = p.context_lens[i];
  if (p.blocks_held_out != p.blocks_held)
    for (int i = threadIdx.x; i < p.B; i += kPagesThreads) p.blocks_held_out[i] = p.blocks_held[i];
}

// Bit maps over the rows in shared memory: rows named (once), named again, and (fork) named as parents.
struct RowMaps {
  uint32_t *once, *again, *parent;
};
__device__ __forceinline__ RowMaps row_maps(uint32_t* smem, int B, bool with_parents) {
  const int words = (B + 31) / 32;
  for (int i = threadIdx.x; i < words * (with_parents ? 3 : 2); i += kPagesThreads) smem[i] = 0u;
  __syncthreads();
  return {smem, smem + words, smem + 2 * words};
}
__device__ __forceinline__ void mark_row(const RowMaps& m, int row, int B) {
  if (row < 0 || row >= B) return;
  const uint32_t bit = 1u << (row & 31);
  if (atomicOr(&m.once[row >> 5], bit) & bit) atomicOr(&m.again[row >> 5], bit);
}
__device__ __forceinline__ bool has_row(const uint32_t* map, int row) { return (map[row >> 5] >> (row & 31)) & 1u; }

// The table entries concerned, numbered in the order of the list and, within a row, of the table.
struct Entries {
  const int32_t *off, *from, *row;  // per fork or row of the list: entries before it, its first table entry, its table row
  int n, total;
  int first;  // of this lane, which has every 32nd of `per_warp` neighbouring numbers of its warp
  int last;   // end of the warp's
};
__device__ __forceinline__ Entries load_entries(const PagesParams& p, int32_t* smem, const Part& t) {
  Entries e = {p.ws_off, p.ws_from, p.parents, p.n};
  if (p.n <= kPagesListInSmem) {
    int32_t *off = smem, *from = off + p.n + 1, *row = from + p.n;
    for (int c = threadIdx.x; c <= p.n; c += kPagesThreads) {
      off[c] = p.ws_off[c];
      if (c < p.n) {
        from[c] = p.ws_from[c];
        row[c] = p.parents[c];
      }
    }
    e.off = off;
    e.from = from;
    e.row = row;
    __syncthreads();
  }
  e.total = e.off[p.n];
  const int warp = t.rank * kPagesWarps + (threadIdx.x >> 5), warps = t.count * kPagesWarps;
  const int per_warp = (e.total + 32 * warps - 1) / (32 * warps) * 32;
  const long long begin = (long long)warp * per_warp;
  e.first = (int)min(begin, (long long)e.total) + (threadIdx.x & 31);
  e.last = (int)min(begin + per_warp, (long long)e.total);
  return e;
}
// Whose entry number g is; `c` = the owner of an earlier one, or 0.
__device__ __forceinline__ int entry_owner(const Entries& e, int g, int c) {
#pragma unroll 1
  for (int k = 0; k < 3; ++k) {
    if (g < e.off[c + 1]) return c;
    ++c;
  }
  int lo = c, hi = e.n;  // largest c with off[c] <= g
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (e.off[mid] <= g) lo = mid; else hi = mid;
  }
  return lo;
}

// ------------------------------------------------------------------------------------ fork
// CTA 0 decides who is granted (a prefix sum of the needed blocks over the forks) and writes what there is one of per fork,
// while the other CTAs copy the counts; then all copy table entries and count holders.  Counts are whole numbers: the order of
// the atomics does not matter.
__global__ void __launch_bounds__(kPagesThreads, 1) fork_pages_kernel(const PagesParams p) {
  extern __shared__ uint32_t s_pages[];  // CTA 0: row maps; then the list of entries
  __shared__ long long s_warp[32];
  const int tid = threadIdx.x;
  const Part t = pages_part(p);
  grid_dep_wait();
  grid_dep_launch();
  if (t.all || p.phase == 1) pages_copy_shares(p, t.rank * kPagesThreads + tid, t.count * kPagesThreads);
  if (t.rank == 0 && (t.all || p.phase == 1)) {
    pages_copy_lens(p);
    const RowMaps m = row_maps(s_pages, p.B, true);
    for (int c = tid; c < p.n; c += kPagesThreads) {
      mark_row(m, p.children[c], p.B);
      const int par = p.parents[c];
      if (par >= 0 && par < p.B) atomicOr(&m.parent[par >> 5], 1u << (par & 31));
    }
    const int head0 = max(0, *p.free_head);
    __syncthreads();
    long long needed = 0, entries = 0;  // by the forks so far
    int taken = 0;                      // blocks handed out, by this thread's forks
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
      const long long upto = head0 + needed + block_scan(need, s_warp, &total);
      needed += total;
      if (ok && need && upto > p.num_free) ok = false;
      const long long before = entries + block_scan(ok ? full : 0, s_warp, &total) - (ok ? full : 0);
      entries += total;
      if (c >= p.n) continue;
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
      p.ws_from[c] = 0;
      p.ws_off[c] = (int)before;
    }
    long long all;
    block_scan(taken, s_warp, &all);
    if (tid == 0) {
      *p.free_head_out = head0 + (int)all;
      p.ws_off[p.n] = (int)entries;
    }
  }
  if (p.phase == 1) return;
  pages_sync(t);
  const Entries e = load_entries(p, reinterpret_cast<int32_t*>(s_pages), t);
  bool bad = false;
  int owner = 0;
  for (int g0 = e.first; g0 < e.last; g0 += 32 * kPagesRound) {
    int id[kPagesRound];
    int32_t* dst[kPagesRound];
#pragma unroll
    for (int k = 0; k < kPagesRound; ++k) {
      const int g = g0 + 32 * k;
      dst[k] = nullptr;
      if (g >= e.last) continue;
      owner = entry_owner(e, g, owner);
      const int c = owner, j = g - e.off[c];
      id[k] = p.block_table[(size_t)e.row[c] * p.MB + j];
      dst[k] = p.block_table + (size_t)p.children[c] * p.MB + j;
    }
#pragma unroll
    for (int k = 0; k < kPagesRound; ++k) {
      if (!dst[k]) continue;
      *dst[k] = id[k];
      if (id[k] >= 0 && id[k] < p.NB)
        atomicAdd(&p.shares_out[id[k]], 1);
      else
        bad = true;
    }
  }
  if (bad) pages_flag(p, kPagesStatusBadBlock);
}

// ------------------------------------------------------------------------------------ release
// Phases, a cluster barrier between each two:
//   1  copies of the state, and per row which entries go                     (CTA 0)
//   2  every entry takes one from its block's count: a count below 0 means that the block is free
//   3  every entry of such a block puts its number - 2^31 there by a minimum: the count now says which entry stands first
//   4  every warp, which has neighbouring entries, counts those that stand first
//   5  prefix sums of the warps' counts give every freed block its place in the free list, in the order of the entries; its
//      count becomes 0 (no entry's number, so entries that look later see that they do not stand first)
// The order of the atomics changes nothing, and the numbers (below 2^30) cannot meet the counts of phase 2 (above -2^30).
__global__ void __launch_bounds__(kPagesThreads, 1) release_pages_kernel(const PagesParams p) {
  extern __shared__ uint32_t s_pages[];  // CTA 0: row maps; then the list of entries
  __shared__ long long s_warp[32];
  __shared__ int s_count[kPagesWarps], s_total[kPagesMaxCluster];
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const Part t = pages_part(p);
  grid_dep_wait();
  grid_dep_launch();
  if (t.all || p.phase == 1) pages_copy_shares(p, t.rank * kPagesThreads + tid, t.count * kPagesThreads);
  if (t.rank == 0 && (t.all || p.phase == 1)) {
    pages_copy_lens(p);
    const RowMaps m = row_maps(s_pages, p.B, false);
    for (int c = tid; c < p.n; c += kPagesThreads) mark_row(m, p.parents[c], p.B);
    __syncthreads();
    long long entries = 0;
    for (int c0 = 0; c0 < p.n; c0 += kPagesThreads) {
      const int c = c0 + tid;
      int from = 0, to = 0;
      if (c < p.n) {
        const int row = p.parents[c];
        if (row >= 0 && row < p.B && !has_row(m.again, row)) {
          const int keep = p.lens ? max(0, p.lens[c]) : 0;
          to = min(max(0, p.blocks_held[row]), p.MB);
          from = min(to, (int)(((long long)keep + (1 << p.bs_log2) - 1) >> p.bs_log2));
          p.context_lens_out[row] = min(max(0, p.context_lens[row]), keep);
          p.blocks_held_out[row] = from;
        } else {
          pages_flag(p, kPagesStatusRefused);
        }
      }
      long long total;
      const long long before = entries + block_scan(to - from, s_warp, &total) - (to - from);
      entries += total;
      if (c < p.n) {
        p.ws_from[c] = from;
        p.ws_off[c] = (int)before;
      }
    }
    if (tid == 0) {
      p.ws_off[p.n] = (int)entries;
      *p.ws_head = min(max(0, *p.free_head), p.num_free);
    }
  }
  if (p.phase == 1) return;
  pages_sync(t);
  const Entries e = load_entries(p, reinterpret_cast<int32_t*>(s_pages), t);
  const bool once = e.last - e.first <= 32 * kPagesRound;  // (of the warp's first lane, which has the most: else ids are loaded anew)
  const bool one_round = __shfl_sync(0xffffffffu, once ? 1 : 0, 0);
  int id[kPagesRound];  // blocks of a round's entries; -1: none, or outside the pool
  bool bad = false;
  int owner = 0;
  auto load = [&](int g0) {
#pragma unroll
    for (int k = 0; k < kPagesRound; ++k) {
      const int g = g0 + 32 * k;
      id[k] = -1;
      if (g >= e.last) continue;
      owner = entry_owner(e, g, owner);
      const int c = owner;
      const int v = p.block_table[(size_t)e.row[c] * p.MB + e.from[c] + g - e.off[c]];
      if (v >= 0 && v < p.NB) id[k] = v; else bad = true;
    }
  };
  // f(number of the round's first entry of the lane), with the round's ids; whole warps
  auto rounds = [&](bool fresh, auto f) {
    owner = 0;
    for (int g0 = e.first; g0 - lane < e.last; g0 += 32 * kPagesRound) {
      if (fresh || !one_round) load(g0);
      f(g0);
    }
  };
  int left[kPagesRound];
  auto look = [&] {
#pragma unroll
    for (int k = 0; k < kPagesRound; ++k) left[k] = id[k] >= 0 ? __ldcg(&p.shares_out[id[k]]) : 0;
  };
  if (t.all || p.phase == 2) {
    rounds(true, [&](int) {
#pragma unroll
      for (int k = 0; k < kPagesRound; ++k)
        if (id[k] >= 0) atomicSub(&p.shares_out[id[k]], 1);
    });
    if (bad) pages_flag(p, kPagesStatusBadBlock);
  }
  pages_sync(t);
  if (t.all || p.phase == 3) {
    rounds(!t.all, [&](int g0) {
      look();
#pragma unroll
      for (int k = 0; k < kPagesRound; ++k)
        if (left[k] < 0) atomicMin(&p.shares_out[id[k]], g0 + 32 * k + INT32_MIN);
    });
  }
  if (p.phase == 2 || p.phase == 3) return;
  pages_sync(t);
  int mine = 0;  // of the warp
  rounds(!t.all, [&](int g0) {
    look();
#pragma unroll
    for (int k = 0; k < kPagesRound; ++k) mine += __popc(__ballot_sync(0xffffffffu, left[k] == g0 + 32 * k + INT32_MIN));
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
    if (t.all && t.count > 1) {
      if (lane < t.count) st_cluster(map_cluster(smem_u32(&s_total[t.rank]), lane), sum);
    } else if (t.all && lane == 0) {
      s_total[0] = sum;
    } else if (p.phase == 4 && lane == 0) {
      p.ws_total[t.rank] = sum;
    }
  }
  if (p.phase == 4) return;
  int before = 0, all = 0;
  if (t.all) {
    pages_sync(t);
    for (int r = 0; r < t.count; ++r) {
      if (r < t.rank) before += s_total[r];
      all += s_total[r];
    }
  } else {
    long long total;
    const long long v = tid < t.count ? p.ws_total[tid] : 0;  // (at most as many CTAs as threads)
    block_scan(v, s_warp, &total);
    all = (int)total;
    block_scan(tid < t.rank ? v : 0, s_warp, &total);
    before = (int)total;
  }
  const int head0 = *p.ws_head;
  const int put = min(all, head0), head1 = head0 - put;  // (ids for which the list has no room are dropped)
  int at = before + s_count[wid];
  rounds(false, [&](int g0) {
    if (!one_round) look();  // (else what was seen before: only an entry itself puts its block's count to 0)
#pragma unroll
    for (int k = 0; k < kPagesRound; ++k) {
      const bool first = left[k] == g0 + 32 * k + INT32_MIN;
      const uint32_t m = __ballot_sync(0xffffffffu, first);
      const int place = at + __popc(m & ((1u << lane) - 1));
      if (first) {
        if (place < put) p.free_ids[head1 + place] = id[k];
        p.shares_out[id[k]] = 0;
      }
      at += __popc(m);
    }
  });
  if (t.rank == 0 && tid == 0) {
    *p.free_head_out = head1;
    if (put < all) pages_flag(p, kPagesStatusRefused);
  }
}

}  // namespace ooco
