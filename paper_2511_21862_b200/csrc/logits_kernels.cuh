// From logits to probabilities: penalties for repeated tokens, biases, grammar masks, temperature, softmax.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "cta_util.cuh"
#include "ptx.cuh"

namespace ooco {

constexpr int kLogitsThreads = 256, kLogitsWarps = kLogitsThreads / 32, kLogitsMaxCluster = 16, kLogitsMaxBias = 1024;
constexpr int kLogitsList = 1024;   // tokens of a share, with a text that names them, that are listed
constexpr int kLogitsBlock = 256;   // neighbouring tokens that one CTA of a row has
constexpr int kLogitsAhead = 10;    // groups of a thread whose loads are in flight together

struct LogitsParams {
  const void* logits;
  const float *temperature, *repetition, *frequency, *presence, *bias_values;
  const int32_t *history, *history_lens, *prompt_lens, *tokens, *parents, *tree_sizes, *bias_tokens;
  const uint32_t* mask;
  float *out, *probs;
  int64_t l_seq, l_node, o_seq, o_node, p_seq, p_node, m_seq, m_node;
  int32_t B, N, V, L, M;   // L = history width, M = bias entries
  int32_t penalties;       // any of the three is given
  int32_t share;           // tokens of a CTA, a multiple of kLogitsBlock
  int32_t cluster_log2;    // CTAs of a row
};

__device__ __forceinline__ float logit(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float logit(const float* p) { return *p; }

struct Penalties {
  float rep, freq, pres;
};
// Every operation is rounded to fp32, none contracted, so that equal logits stay equal and near ones keep their order.
__device__ __forceinline__ float penalised(float x, uint32_t made, const Penalties& w) {
  x = x > 0.f ? __fdiv_rn(x, w.rep) : __fmul_rn(x, w.rep);
  if (made) x = __fsub_rn(__fsub_rn(x, __fmul_rn(w.freq, (float)made)), w.pres);
  return x;
}

// A reference r, and the sum of exp((x - r) / T) (or, where the temperature asks for the largest logit, its lowest index).
struct Softmax {
  float top, sum;
};

__device__ __forceinline__ void prefetch_l2(const void* ptr) { asm volatile("prefetch.global.L2 [%0];" ::"l"(ptr)); }

constexpr uint32_t kMinusInf2 = 0xff80ff80u;  // two bf16 values of -inf
// The larger of two pairs of bf16 values, the other one where one is a NaN.
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// The signs of the four bytes that kSelect's digits name (8 + byte), each over a byte.
template <int kSelect>
__device__ __forceinline__ uint32_t spread_signs(uint32_t a) {
  uint32_t d;
  asm("prmt.b32 %0, %1, %1, %2;" : "=r"(d) : "r"(a), "n"(kSelect));
  return d;
}
__device__ __forceinline__ uint32_t select(uint32_t a, uint32_t b, uint32_t bits) { return (a & bits) | (b & ~bits); }

// A thread's neighbouring tokens.
template <int W>
struct Group {
  float x[W];
  __device__ float& operator[](int j) { return x[j]; }
  __device__ const float& operator[](int j) const { return x[j]; }
};

// What a token's text says: a bit for the prompt above the number of generated occurrences.  Half a word where the history is
// short enough (two tokens share a word of shared memory, and their fields cannot run into one another), else a word.
template <bool kHalf>
struct Counter {
  static constexpr uint32_t kPrompt = kHalf ? 0x8000u : 0x80000000u;
  __device__ static uint32_t read(const uint32_t* s, int at) {
    return kHalf ? (s[at >> 1] >> (16 * (at & 1))) & 0xffffu : s[at];
  }
  __device__ static uint32_t add(uint32_t* s, int at, uint32_t v) {  // returns what was there
    return kHalf ? (atomicAdd(&s[at >> 1], v << (16 * (at & 1))) >> (16 * (at & 1))) & 0xffffu : atomicAdd(&s[at], v);
  }
  __device__ static void take(uint32_t* s, int at) { kHalf ? atomicSub(&s[at >> 1], 1u << (16 * (at & 1))) : atomicSub(&s[at], 1u); }
  __device__ static uint32_t mark(uint32_t* s, int at) {
    return kHalf ? (atomicOr(&s[at >> 1], kPrompt << (16 * (at & 1))) >> (16 * (at & 1))) & 0xffffu : atomicOr(&s[at], kPrompt);
  }
};

// A cluster of CTAs works on an equal part of the rows, node by node of a sequence.  Blocks of 256 neighbouring tokens go to its CTAs in
// turn, so that the low token numbers, which tokenisers give to frequent pieces, do not all fall to one.  The text is read and
// counted once for all the nodes: every CTA reads the whole history (from L2 but for the first) and counts what falls into its
// share, which is cheaper than sending counts through the cluster; tokens that it meets are listed, so that the arithmetic of the
// penalties runs with full warps.  Then, for each node: the masked logits to shared memory, one word a token; penalties and
// biases on the tokens concerned; the largest; weights and their sum; one exchange in the cluster; probabilities.  So logits are
// read once and probabilities written once.  Many rows are bound by instructions, by the chain of a node's steps and, with clusters
// of 16, by the SMs that hold none (256 rows of 152064 in trees of 16: 116 us, 2.0 TB/s; fp32 logits 149, shaped logits out as well
// 141), few rows by the chain of loads, reductions and the exchange (4 rows of 128256: 12 us).
// The largest value is found on the way: over the masked logits as they come and over the values that penalties change.  Only where
// the second cannot stand for the true one (biases, a largest logit that fell far, a greedy row) are the values gone through again.
// Sums are fp32: 2^-24 relative a step, over the up to 100 values of a thread, a tree of 8 levels, and a tree over the CTAs.
// kWide: rows of logits and outputs begin on boundaries of four values, so a thread has groups of four neighbours, which every
// access to shared and global memory moves without conflicts or partial sectors; else single tokens, side by side across the lanes
// (256 rows of 152064 and 152065: 116 and 305 us; of 50256 and 50257: 59 and 106).
// Biases: a token's first entry looks for its others, for every row again: 16 entries cost nothing, 256 16 us and 1024 155 us a row
// of a cluster.
template <typename T, bool kWide, bool kHalf>
__global__ void __launch_bounds__(kLogitsThreads, 3) shape_logits_kernel(const LogitsParams p) {
  using C = Counter<kHalf>;
  constexpr int W = kWide ? 4 : 1;
  using G = Group<W>;
  extern __shared__ uint4 s_dyn[];  // values [share]; biases: tokens, places; with penalties: counters [share], ancestors of the nodes
  float* s_val = reinterpret_cast<float*>(s_dyn);
  int* s_bias_token = reinterpret_cast<int*>(s_val + p.share);
  int* s_bias_at = s_bias_token + ((p.M + 3) & ~3);
  uint32_t* s_count = reinterpret_cast<uint32_t*>(s_bias_at + ((p.M + 3) & ~3));
  uint32_t* s_above = s_count + (kHalf ? p.share / 2 : p.share);  // [N][words]
  __shared__ float s_warp[4][kLogitsWarps], s_factor;
  __shared__ Softmax s_rank[2][kLogitsMaxCluster];
  __shared__ int s_token[kTreeMaxNodes], s_parent[kTreeMaxNodes], s_listed;
  __shared__ uint16_t s_list[kLogitsList];
  const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
  const int cluster = 1 << p.cluster_log2;
  const uint32_t rank = cluster > 1 ? cluster_rank() : 0;
  grid_dep_wait();
  grid_dep_launch();
  const bool exchange = cluster > 1 && p.probs;
  if (exchange) cluster_arrive();  // (waited for before the first write to another CTA's memory)
  bool started = false;  // every CTA of the cluster has started
  int turn = 0;
  // the token at place i of the share, and the place of a token, or -1
  auto token = [&](uint32_t i) {
    return (int)((((i / kLogitsBlock) << p.cluster_log2) + rank) * kLogitsBlock + i % kLogitsBlock);
  };
  auto place = [&](uint32_t tok) {
    const uint32_t block = tok / kLogitsBlock;
    return tok < (uint32_t)p.V && (block & (cluster - 1)) == rank
               ? (int)((block >> p.cluster_log2) * kLogitsBlock + tok % kLogitsBlock) : -1;
  };
  // the cluster's rows: an equal part of all, sequence by sequence
  const int clusters = gridDim.x >> p.cluster_log2, me = blockIdx.x >> p.cluster_log2;
  const int64_t rows = (int64_t)p.B * p.N;
  const int row1 = (int)(rows * (me + 1) / clusters);
  for (int row = (int)(rows * me / clusters); row < row1;) {
    const int b = row / p.N, node0 = row - b * p.N, count = min(p.N - node0, row1 - row);
    row += count;
    const int nodes = p.tree_sizes ? min(p.N, p.tree_sizes[b]) : p.N, node1 = min(nodes, node0 + count);
    if (node0 >= node1) continue;  // (the whole cluster)
    const T* src0 = reinterpret_cast<const T*>(p.logits) + (int64_t)b * p.l_seq;
    const uint32_t* mask0 = p.mask ? p.mask + (int64_t)b * p.m_seq : nullptr;
    auto prefetch = [&](int node) {
      constexpr int kLine = 128 / (int)sizeof(T);
      const T* src = src0 + (int64_t)node * p.l_node;
      for (int i = tid * kLine; i < p.share; i += kLogitsThreads * kLine)
        if (token(i) < p.V) prefetch_l2(src + token(i));
      if (mask0)
        for (int i = tid * kLogitsBlock; i < p.share; i += kLogitsThreads * kLogitsBlock)
          if (token(i) < p.V) prefetch_l2(mask0 + (int64_t)node * p.m_node + (token(i) >> 5));
    };
    // ---- once: the text, the biases
    const float t = p.temperature ? p.temperature[b] : 1.f;
    const bool soft = t > 0.f;
    if (tid == 0) {
      s_listed = 0;
      if (soft) s_factor = (float)(1.4426950408889634 / (double)t);  // (one rounding)
    }
    Penalties w = {1.f, 0.f, 0.f};
    const bool drafts = p.penalties && p.tokens && p.N > 1;
    const int words = (p.N + 31) / 32;
    auto list = [&](int at) {  // a token whose counter was 0
      const int i = atomicAdd(&s_listed, 1);
      if (i < kLogitsList) s_list[i] = (uint16_t)at;
    };
    if (p.M > 0)
      for (int j = tid; j < p.M; j += kLogitsThreads) s_bias_token[j] = p.bias_tokens[(int64_t)b * p.M + j];
    if (p.penalties) {
      const int len = min(max(0, p.history_lens[b]), p.L), prompt = p.prompt_lens ? min(max(0, p.prompt_lens[b]), len) : 0;
      if (p.repetition) w.rep = p.repetition[b] > 0.f ? p.repetition[b] : 1.f;
      if (p.frequency) w.freq = p.frequency[b];
      if (p.presence) w.pres = p.presence[b];
      prefetch(node0);
      if (node0 + 1 < node1) prefetch(node0 + 1);
      for (int i = tid; i < (kHalf ? p.share / 8 : p.share / 4); i += kLogitsThreads)
        reinterpret_cast<uint4*>(s_count)[i] = make_uint4(0u, 0u, 0u, 0u);
      if (drafts)
        for (int i = tid; i < p.N; i += kLogitsThreads) {
          const int up = p.parents ? p.parents[(int64_t)b * p.N + i] : i - 1;
          s_parent[i] = up < i ? up : -1;
          s_token[i] = p.tokens[(int64_t)b * p.N + i];
        }
      __syncthreads();
      if (drafts && wid == kLogitsWarps - 1)  // the nodes of every branch but the root, parents first
        for (int i = 0; i < node1; ++i) {
          const int up = s_parent[i];
          if (lane < words) {
            const uint32_t own = i > 0 && (i >> 5) == lane ? 1u << (i & 31) : 0u;
            s_above[i * words + lane] = (up >= 0 ? s_above[up * words + lane] : 0u) | own;
          }
          __syncwarp();
        }
      auto named = [&](int tok, bool generated) {
        const int at = place(tok);
        if (at >= 0 && !(generated ? C::add(s_count, at, 1u) : C::mark(s_count, at))) list(at);
      };
      const int32_t* text = p.history + (int64_t)b * p.L;
      const int whole = ((uintptr_t)text & 15) ? 0 : len / 4;
      for (int i0 = tid; i0 < whole; i0 += 4 * kLogitsThreads) {  // four loads in flight
        int4 u[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int i = i0 + k * kLogitsThreads;
          u[k] = i < whole ? reinterpret_cast<const int4*>(text)[i] : make_int4(-1, -1, -1, -1);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int i = 4 * (i0 + k * kLogitsThreads);
          named(u[k].x, i >= prompt);
          named(u[k].y, i + 1 >= prompt);
          named(u[k].z, i + 2 >= prompt);
          named(u[k].w, i + 3 >= prompt);
        }
      }
      for (int i = 4 * whole + tid; i < len; i += kLogitsThreads) named(text[i], i >= prompt);
    }
    __syncthreads();
    for (int j = tid; j < p.M; j += kLogitsThreads) {  // a token's first entry stands for all of them
      int at = place(s_bias_token[j]);
      for (int k = 0; k < j && at >= 0; ++k)
        if (s_bias_token[k] == s_bias_token[j]) at = -1;
      s_bias_at[j] = at;
    }
    const int listed0 = s_listed;  // (of the text; the drafts of a node come behind)
    const float factor = soft ? s_factor : 0.f;
    __syncthreads();  // (before a draft is listed)
    // ---- a thread's groups of W tokens: places and tokens move on by fixed steps, since a step is whole blocks
    constexpr int kStep = kLogitsThreads * W;
    const int i_first = tid * W, v_first = token(i_first), v_step = kStep << p.cluster_log2;
    // f(place, token) for the groups in the vocabulary (a row's last one may end behind it: kEnd)
    const int blocks_in = max(0, (p.V / kLogitsBlock - (int)rank + cluster - 1) >> p.cluster_log2);  // blocks wholly inside
    const int steps_in = blocks_in * kLogitsBlock / kStep;                                          // ... and steps
    auto groups = [&](auto f) {
      int i = i_first, v = v_first;
#pragma unroll 4
      for (int k = 0; k < steps_in; ++k, i += kStep, v += v_step) f(i, v, std::false_type{});
      for (; i < p.share; i += kStep, v += v_step)
        if (v < p.V) f(i, v, std::true_type{});
    };
    auto store = [&](float* dst, int v, const G& x, auto end) {
      if constexpr (kWide) {
        if (!decltype(end)::value || v + W <= p.V) {
          *reinterpret_cast<float4*>(dst + v) = make_float4(x[0], x[1], x[2], x[3]);
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j)
            if (v + j < p.V) dst[v + j] = x[j];
        }
      } else {
        dst[v] = x[0];
      }
    };
    auto get = [&](int i, G& x) {
      if constexpr (kWide) {
        const float4 u = *reinterpret_cast<const float4*>(s_val + i);
        x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
      } else {
        x[0] = s_val[i];
      }
    };
    auto put = [&](int i, const G& x) {
      if constexpr (kWide)
        *reinterpret_cast<float4*>(s_val + i) = make_float4(x[0], x[1], x[2], x[3]);
      else
        s_val[i] = x[0];
    };
    // reductions over the CTA, by a barrier between the two halves
    auto post = [&](float v, float* s, auto op) {
#pragma unroll
      for (int o = 16; o; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
      if (lane == 0) s[wid] = v;
    };
    auto fetch = [&](const float* s, auto op) {
      float v = s[lane & (kLogitsWarps - 1)];
#pragma unroll
      for (int o = kLogitsWarps / 2; o; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
      return v;
    };
    auto reduce = [&](float v, float* s, auto op) {
      post(v, s, op);
      __syncthreads();
      return fetch(s, op);
    };
    auto larger = [](float a, float c) { return fmaxf(a, c); };
    // The weight of a logit beside a reference; equal infinite logits have a weight of 1 each, whatever the temperature.  Where they are
    // finite, exponents are differences to the rounded product of reference and factor, whose error all weights then share.
    auto weight = [&](float v, float ref) {
      if (v == ref) return 1.f;
      if (v == -INFINITY || ref == INFINITY) return 0.f;
      const float a = __fmul_rn(v, factor), c = __fmul_rn(ref, factor);
      return ex2(fabsf(a) < INFINITY && fabsf(c) < INFINITY ? __fsub_rn(a, c) : (v - ref) * factor);
    };

    // a group's logits as they are loaded, and as values (the maximum with -inf turns a NaN into it)
    using Raw = std::conditional_t<kWide, std::conditional_t<sizeof(T) == 2, uint2, float4>, T>;
    auto values = [&](const Raw& r, G& x) {
      if constexpr (!kWide) {
        x[0] = logit(&r);
      } else if constexpr (sizeof(T) == 2) {
        x[0] = bf16_lo(r.x), x[1] = bf16_hi(r.x), x[2] = bf16_lo(r.y), x[3] = bf16_hi(r.y);
      } else {
        x[0] = r.x, x[1] = r.y, x[2] = r.z, x[3] = r.w;
      }
    };
    // groups that lie wholly inside the share and the vocabulary, as far as their loads fly together
    const int n_ahead = min(kLogitsAhead, min((p.share - i_first + kStep - 1) / kStep, v_first + W <= p.V ? (p.V - W - v_first) / v_step + 1 : 0));
    const uint32_t mask_shift = v_first & 31;  // (steps are whole words)

    for (int node = node0; node < node1; ++node) {
      // ---- masked logits to shared memory.  They come from L2, where they were sent for two nodes ago.  (Registers loaded a node ahead
      // would serve better, but what a warp waits for later, it then waits for together with them: 161 us for 133.)
      Raw ahead[kLogitsAhead];
      uint32_t ahead_mask[kLogitsAhead];
      {
        const T* src = src0 + (int64_t)node * p.l_node + v_first;
        const uint32_t* mask = mask0 ? mask0 + (int64_t)node * p.m_node + (v_first >> 5) : nullptr;
#pragma unroll
        for (int k = 0; k < kLogitsAhead; ++k) {
          if (k < n_ahead) {
            ahead[k] = *reinterpret_cast<const Raw*>(src + k * v_step);
            ahead_mask[k] = mask ? mask[k * (v_step >> 5)] : ~0u;
          }
        }
      }
      float top = -INFINITY;
      auto finish = [&](int i, G& x, uint32_t allowed) {
#pragma unroll
        for (int j = 0; j < W; ++j) {
          x[j] = (allowed >> j) & 1u ? fmaxf(x[j], -INFINITY) : -INFINITY;
          top = fmaxf(top, x[j]);
        }
        put(i, x);
      };
      uint32_t top2 = kMinusInf2;
#pragma unroll
      for (int k = 0; k < kLogitsAhead; ++k) {
        if (k < n_ahead) {
          const uint32_t allowed = ahead_mask[k] >> mask_shift;
          G x;
          if constexpr (kWide && sizeof(T) == 2) {  // two logits at a time, as they are stored
            // four bits to the signs of four bytes (no two of the product's terms meet), each sign to 16 bits
            const uint32_t signs = (allowed & 15u) * 0x10204080u;
            Raw v = ahead[k];
            v.x = max_bf16x2(kMinusInf2, select(v.x, kMinusInf2, spread_signs<0x9988>(signs)));
            v.y = max_bf16x2(kMinusInf2, select(v.y, kMinusInf2, spread_signs<0xbbaa>(signs)));
            top2 = max_bf16x2(top2, max_bf16x2(v.x, v.y));
            values(v, x);
            put(i_first + k * kStep, x);
          } else {
            values(ahead[k], x);
            finish(i_first + k * kStep, x, allowed);
          }
        }
      }
      if constexpr (kWide && sizeof(T) == 2) top = fmaxf(bf16_lo(top2), bf16_hi(top2));
      {  // what is left: further steps, the group across the end of the vocabulary
        const T* src = src0 + (int64_t)node * p.l_node;
        const uint32_t* mask = mask0 ? mask0 + (int64_t)node * p.m_node : nullptr;
        for (int i = i_first + n_ahead * kStep, v = v_first + n_ahead * v_step; i < p.share && v < p.V; i += kStep, v += v_step) {
          G x;
          if (v + W <= p.V) {
            values(*reinterpret_cast<const Raw*>(src + v), x);
          } else {
#pragma unroll
            for (int j = 0; j < W; ++j) x[j] = v + j < p.V ? logit(src + v + j) : -INFINITY;
          }
          finish(i, x, mask ? mask[v >> 5] >> (v & 31) : ~0u);
        }
      }
      if (node + 2 < node1) prefetch(node + 2);
      // ---- penalties and biases
      if (drafts && tid > 0 && tid <= node && ((s_above[node * words + (tid >> 5)] >> (tid & 31)) & 1u)) {
        const int at = place(s_token[tid]);
        if (at >= 0 && !C::add(s_count, at, 1u)) list(at);
      }
      post(top, s_warp[0], larger);
      __syncthreads();
      bool exact = p.M == 0;  // top does for a reference
      if (!p.penalties) {
        top = fetch(s_warp[0], larger);
      } else {
        float changed = -INFINITY;
        const int listed = s_listed;
        const bool all = listed > kLogitsList;  // a share with more tokens than the list holds is walked through
        for (int i = tid; i < (all ? p.share : listed); i += kLogitsThreads) {
          const int at = all ? i : s_list[i];
          const uint32_t word = C::read(s_count, at);
          if (!word || (all && token(at) >= p.V)) continue;
          const float x = s_val[at];
          if (x == -INFINITY) continue;
          const float y = fmaxf(penalised(x, word & (C::kPrompt - 1), w), -INFINITY);
          s_val[at] = y;
          changed = fmaxf(changed, y);
        }
        changed = reduce(changed, s_warp[1], larger);
        top = fmaxf(fetch(s_warp[0], larger), changed);
        // What was the largest may have fallen.  The largest now is then at least the largest of the values changed; if that is near
        // what was, it does for a reference: no weight is above 2^16, and those that fall below the smallest numbers do not matter.
        if (listed > 0) {
          exact = exact && soft && (top - changed) * factor < 16.f;
          if (exact) top = changed;
        }
        if (tid == 0) s_listed = listed0;
        if (drafts && tid > 0 && tid <= node && ((s_above[node * words + (tid >> 5)] >> (tid & 31)) & 1u)) {
          const int at = place(s_token[tid]);
          if (at >= 0) C::take(s_count, at);  // back to what the text says
        }
      }
      if (p.M > 0) {
        for (int j = tid; j < p.M; j += kLogitsThreads) {
          const int at = s_bias_at[j];
          if (at < 0 || s_val[at] == -INFINITY) continue;
          float x = s_val[at];
          for (int k = j; k < p.M; ++k)
            if (s_bias_token[k] == s_bias_token[j]) x = __fadd_rn(x, p.bias_values[(int64_t)b * p.M + k]);
          s_val[at] = fmaxf(x, -INFINITY);
        }
        __syncthreads();
      }
      float* out = p.out ? p.out + (int64_t)b * p.o_seq + (int64_t)node * p.o_node : nullptr;
      if (!p.probs) {
        groups([&](int i, int v, auto end) {
          G x;
          get(i, x);
          store(out, v, x, end);
        });
        __syncthreads();
        continue;
      }
      // ---- softmax: a CTA has a reference of its own, at most its largest logit, so one exchange between the CTAs does
      if (!exact) {  // its largest logit
        top = -INFINITY;
        groups([&](int i, int, auto) {
          G x;
          get(i, x);
#pragma unroll
          for (int j = 0; j < W; ++j) top = fmaxf(top, x[j]);
        });
        top = reduce(top, s_warp[3], larger);
      }
      float sum;
      if (soft) {
        sum = 0.f;
        const float c = __fmul_rn(top, factor);
        const bool plain = fabsf(top) < INFINITY && factor > 0.f && factor < INFINITY && fabsf(c) < INFINITY;
        if (out)
          groups([&](int i, int v, auto end) {
            G x;
            get(i, x);
            store(out, v, x, end);
          });
        if (plain) {
          float2 sums = make_float2(0.f, 0.f);
          groups([&](int i, int, auto) {
            G x;
            get(i, x);
            if constexpr (kWide) {
#pragma unroll
              for (int j = 0; j < W; j += 2) {
                const float2 e = ffma2(make_float2(x[j], x[j + 1]), make_float2(factor, factor), make_float2(-c, -c));
                x[j] = ex2(e.x), x[j + 1] = ex2(e.y);
                sums = fadd2(sums, make_float2(x[j], x[j + 1]));
              }
            } else {
              x[0] = ex2(__fmaf_rn(x[0], factor, -c));
              sums.x += x[0];
            }
            put(i, x);
          });
          sum = sums.x + sums.y;
        } else {
          groups([&](int i, int, auto) {
            G x;
            get(i, x);
#pragma unroll
            for (int j = 0; j < W; ++j) {
              x[j] = top == -INFINITY ? 0.f : weight(x[j], top);
              sum += x[j];
            }
            put(i, x);
          });
        }
        sum = reduce(sum, s_warp[2], [](float a, float c) { return a + c; });
      } else {
        sum = INFINITY;  // the lowest index (below 2^24: exact) of the CTA's largest logit
        groups([&](int i, int v, auto end) {
          G x;
          get(i, x);
          if (out) store(out, v, x, end);
#pragma unroll
          for (int j = 0; j < W; ++j)
            if (x[j] == top && v + j < p.V) sum = fminf(sum, (float)(v + j));
        });
        sum = reduce(sum, s_warp[2], [](float a, float c) { return fminf(a, c); });
      }
      Softmax all = {top, sum};
      if (exchange) {
        Softmax* ranks = s_rank[turn ^= 1];  // (one of two: a CTA may still read the row before's)
        if (!started) cluster_wait();
        started = true;
        if (wid == 0 && lane < cluster) {
          const uint32_t at = map_cluster(smem_u32(&ranks[rank]), lane);
          st_cluster(at, top);
          st_cluster(at + 4, sum);
        }
        cluster_arrive();
        cluster_wait();
        Softmax o = {-INFINITY, soft ? 0.f : INFINITY};
        if (lane < cluster) o = ranks[lane];
        all.top = o.top;
#pragma unroll
        for (int k = kLogitsMaxCluster / 2; k; k >>= 1) all.top = fmaxf(all.top, __shfl_xor_sync(0xffffffffu, all.top, k));
        all.top = __shfl_sync(0xffffffffu, all.top, 0);
        all.sum = soft ? o.sum * weight(o.top, all.top) : (o.top == all.top ? o.sum : INFINITY);
#pragma unroll
        for (int k = kLogitsMaxCluster / 2; k; k >>= 1) {
          const float other = __shfl_xor_sync(0xffffffffu, all.sum, k);
          all.sum = soft ? all.sum + other : fminf(all.sum, other);
        }
        all.sum = __shfl_sync(0xffffffffu, all.sum, 0);
      }
      float* probs = p.probs + (int64_t)b * p.p_seq + (int64_t)node * p.p_node;
      if (soft) {
        const float scale = all.top == -INFINITY ? 0.f : weight(top, all.top) * __fdiv_rn(1.f, all.sum);
        groups([&](int i, int v, auto end) {
          G x;
          get(i, x);
          if constexpr (kWide) {
#pragma unroll
            for (int j = 0; j < W; j += 2) {
              const float2 y = fmul2(make_float2(x[j], x[j + 1]), make_float2(scale, scale));
              x[j] = y.x, x[j + 1] = y.y;
            }
          } else {
            x[0] *= scale;
          }
          store(probs, v, x, end);
        });
      } else {
        groups([&](int, int v, auto end) {
          G x;
#pragma unroll
          for (int j = 0; j < W; ++j) x[j] = all.top != -INFINITY && (float)(v + j) == all.sum ? 1.f : 0.f;
          store(probs, v, x, end);
        });
      }
      // (a thread's groups are its own: the next node's logits may overwrite them.  The counters are back to the text's behind the
      // barriers of the reductions)
    }
  }
  if (exchange && !started) cluster_wait();
}

}  // namespace ooco
