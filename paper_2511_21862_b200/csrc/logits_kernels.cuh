// From logits to probabilities: penalties for repeated tokens, biases, grammar masks, temperature, softmax.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "cta_util.cuh"
#include "ptx.cuh"

namespace ooco {

constexpr int kLogitsThreads = 512, kLogitsMaxCluster = 16, kLogitsMaxBias = 1024;
constexpr uint32_t kSeenBit = 0x80000000u;  // of a counter: the token stands in the prompt

struct LogitsParams {
  const void* logits;
  const float *temperature, *repetition, *frequency, *presence, *bias_values;
  const int32_t *history, *history_lens, *prompt_lens, *tokens, *parents, *tree_sizes, *bias_tokens;
  const uint32_t* mask;
  float *out, *probs;
  int64_t l_seq, l_node, o_seq, o_node, p_seq, p_node, m_seq, m_node;
  int32_t B, N, V, L, M;   // L = history width, M = bias entries
  int32_t share;           // values per CTA, a multiple of 256
  int32_t penalties;       // any of the three is given
};

__device__ __forceinline__ void add_cluster(uint32_t addr, uint32_t v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void or_cluster(uint32_t addr, uint32_t v) {
  asm volatile("red.relaxed.cluster.shared::cluster.or.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ float logit(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float logit(const float* p) { return *p; }
__device__ __forceinline__ float no_nan(float x) { return x == x ? x : -INFINITY; }

struct Penalties {
  float rep, freq, pres;
};
// Every operation is rounded to fp32, none contracted, so that equal logits stay equal and near ones keep their order.
__device__ __forceinline__ float penalised(float x, uint32_t count, const Penalties& w) {
  x = x > 0.f ? __fdiv_rn(x, w.rep) : __fmul_rn(x, w.rep);
  const uint32_t n = count & ~kSeenBit;
  if (n) x = __fsub_rn(__fsub_rn(x, __fmul_rn(w.freq, (float)n)), w.pres);
  return x;
}

// Reduction over the CTA, then over the cluster through distributed shared memory; every thread gets the result.  The order of
// a sum depends on the launch shape alone.
template <typename Op>
__device__ __forceinline__ float cluster_reduce(float v, Op op, float* s_warp, float* s_rank, int rank, int cluster) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  for (int o = 16; o; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  if (lane == 0) s_warp[wid] = v;
  __syncthreads();
  if (wid == 0) {
    v = s_warp[lane % (kLogitsThreads / 32)];
    for (int o = kLogitsThreads / 64; o; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
    if (cluster > 1) {
      if (lane < cluster) st_cluster(map_cluster(smem_u32(s_rank + rank), lane), v);
    } else if (lane == 0) {
      s_rank[0] = v;
    }
  }
  if (cluster > 1) {
    cluster_arrive();
    cluster_wait();
  } else {
    __syncthreads();
  }
  v = s_rank[0];
  for (int r = 1; r < cluster; ++r) v = op(v, s_rank[r]);
  return v;
}

// A cluster of CTAs per row.  Each CTA holds its share of the vocabulary in shared memory as one word per token: first the
// token's count (the history is read once, split over the CTAs, which count in one another's shared memory), then the shaped
// logit, then its weight.  So logits are read once and probabilities written once, which is what bounds the kernel: HBM for
// many rows, the chain of passes and cluster barriers for few.  Sums are fp32: 2^-24 relative a term and step of a tree of
// about 16 levels and the 40 to 130 values of a thread.
template <typename T>
__global__ void __launch_bounds__(kLogitsThreads, 2) shape_logits_kernel(const LogitsParams p, const int cluster) {
  extern __shared__ uint32_t s_word[];  // [share]
  __shared__ float s_warp[2][kLogitsThreads / 32], s_rank[2][kLogitsMaxCluster];
  __shared__ int s_parent[kTreeMaxNodes], s_bias_token[kLogitsMaxBias];
  const int tid = threadIdx.x;
  const int rank = cluster > 1 ? (int)cluster_rank() : 0;
  const int row = blockIdx.x / cluster, b = row / p.N, node = row - b * p.N;
  grid_dep_wait();
  grid_dep_launch();
  if (p.tree_sizes && node >= p.tree_sizes[b]) return;  // (the whole cluster)
  const int lo = min(p.V, rank * p.share), hi = min(p.V, lo + p.share), n = hi - lo;
  const T* src = reinterpret_cast<const T*>(p.logits) + (int64_t)b * p.l_seq + (int64_t)node * p.l_node + lo;
  const uint32_t* mask = p.mask ? p.mask + (int64_t)b * p.m_seq + (int64_t)node * p.m_node + (lo >> 5) : nullptr;
  float* s_val = reinterpret_cast<float*>(s_word);
  Penalties w = {1.f, 0.f, 0.f};
  if (p.penalties) {
    if (p.repetition) w.rep = p.repetition[b] > 0.f ? p.repetition[b] : 1.f;
    if (p.frequency) w.freq = p.frequency[b];
    if (p.presence) w.pres = p.presence[b];
    for (int i = tid; i < p.share / 4; i += kLogitsThreads) reinterpret_cast<uint4*>(s_word)[i] = make_uint4(0u, 0u, 0u, 0u);
    const int len = min(max(0, p.history_lens[b]), p.L), prompt = p.prompt_lens ? min(max(0, p.prompt_lens[b]), len) : 0;
    const bool drafts = p.tokens && node > 0;
    if (rank == 0 && drafts)
      for (int i = tid; i <= node; i += kLogitsThreads) s_parent[i] = p.parents ? p.parents[(int64_t)b * p.N + i] : i - 1;
    if (cluster > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
    const uint32_t base = smem_u32(s_word);
    auto count = [&](int tok, bool generated) {
      if (tok < 0 || tok >= p.V) return;
      const int owner = tok / p.share;
      const uint32_t at = base + 4u * (uint32_t)(tok - owner * p.share);
      if (cluster > 1) {
        const uint32_t far = map_cluster(at, owner);
        if (generated) add_cluster(far, 1u); else or_cluster(far, kSeenBit);
      } else {
        if (generated) atomicAdd(&s_word[tok], 1u); else atomicOr(&s_word[tok], kSeenBit);
      }
    };
    const int32_t* text = p.history + (int64_t)b * p.L;
    for (int i = rank * kLogitsThreads + tid; i < len; i += cluster * kLogitsThreads) count(text[i], i >= prompt);
    if (rank == 0 && drafts && tid == 0)
      for (int k = node; k > 0;) {
        count(p.tokens[(int64_t)b * p.N + k], true);
        const int up = s_parent[k];
        k = up < k ? up : -1;
      }
    if (cluster > 1) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
  } else if (cluster > 1 && p.probs) {
    cluster_arrive();  // (waited for before the first write to another CTA's memory)
  }
  // ---- the shaped logits but for the biases
  constexpr int W = 8;
  const bool wide = !((uintptr_t)src & 15);
  const int groups = wide ? n / W : 0;
  for (int g = tid; g < groups; g += kLogitsThreads) {
    float x[W];
    if (sizeof(T) == 2) {
      unpack8(reinterpret_cast<const uint4*>(src)[g], x);
    } else {
      const float4 lo4 = reinterpret_cast<const float4*>(src)[2 * g], hi4 = reinterpret_cast<const float4*>(src)[2 * g + 1];
      x[0] = lo4.x, x[1] = lo4.y, x[2] = lo4.z, x[3] = lo4.w, x[4] = hi4.x, x[5] = hi4.y, x[6] = hi4.z, x[7] = hi4.w;
    }
    const uint32_t allowed = mask ? mask[g >> 2] >> (8 * (g & 3)) : 0xffu;
    if (p.penalties) {
      const uint4 c0 = reinterpret_cast<const uint4*>(s_word)[2 * g], c1 = reinterpret_cast<const uint4*>(s_word)[2 * g + 1];
      const uint32_t c[W] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w};
#pragma unroll
      for (int k = 0; k < W; ++k)
        if (c[k]) x[k] = penalised(x[k], c[k], w);
    }
#pragma unroll
    for (int k = 0; k < W; ++k) x[k] = (allowed >> k) & 1u ? no_nan(x[k]) : -INFINITY;
    reinterpret_cast<float4*>(s_val)[2 * g] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(s_val)[2 * g + 1] = make_float4(x[4], x[5], x[6], x[7]);
  }
  for (int i = groups * W + tid; i < n; i += kLogitsThreads) {
    float x = logit(src + i);
    if (p.penalties && s_word[i]) x = penalised(x, s_word[i], w);
    s_val[i] = !mask || ((mask[i >> 5] >> (i & 31)) & 1u) ? no_nan(x) : -INFINITY;
  }
  __syncthreads();
  if (p.M > 0) {  // a token may be listed more than once: the thread of its first entry adds them all, in their order
    for (int j = tid; j < p.M; j += kLogitsThreads) s_bias_token[j] = p.bias_tokens[(int64_t)b * p.M + j];
    __syncthreads();
    for (int j = tid; j < p.M; j += kLogitsThreads) {
      const int tok = s_bias_token[j];
      if (tok < lo || tok >= hi) continue;
      bool first = true;
      for (int k = 0; k < j; ++k) first &= s_bias_token[k] != tok;
      if (!first || s_val[tok - lo] == -INFINITY) continue;
      float x = s_val[tok - lo];
      for (int k = j; k < p.M; ++k)
        if (s_bias_token[k] == tok) x = __fadd_rn(x, p.bias_values[(int64_t)b * p.M + k]);
      s_val[tok - lo] = no_nan(x);
    }
    __syncthreads();
  }
  float* out = p.out ? p.out + (int64_t)b * p.o_seq + (int64_t)node * p.o_node + lo : nullptr;
  if (out)
    for (int i = tid; i < n; i += kLogitsThreads) out[i] = s_val[i];
  if (!p.probs) return;  // (the whole grid)
  float* probs = p.probs + (int64_t)b * p.p_seq + (int64_t)node * p.p_node + lo;
  if (cluster > 1 && !p.penalties) cluster_wait();
  // ---- softmax
  float top = -INFINITY;
  for (int i = tid; i < n; i += kLogitsThreads) top = fmaxf(top, s_val[i]);
  top = cluster_reduce(top, [](float a, float c) { return fmaxf(a, c); }, s_warp[0], s_rank[0], rank, cluster);
  const float t = p.temperature ? p.temperature[b] : 1.f;
  if (top == -INFINITY) {
    for (int i = tid; i < n; i += kLogitsThreads) probs[i] = 0.f;
  } else if (t > 0.f) {
    const float inv = __fdiv_rn(1.f, t);
    float sum = 0.f;
    for (int i = tid; i < n; i += kLogitsThreads) {
      const float x = s_val[i];
      const float e = x == top ? 1.f : (x == -INFINITY ? 0.f : expf((x - top) * inv));
      s_val[i] = e;
      sum += e;
    }
    sum = cluster_reduce(sum, [](float a, float c) { return a + c; }, s_warp[1], s_rank[1], rank, cluster);
    const float scale = __fdiv_rn(1.f, sum);
    for (int i = tid; i < n; i += kLogitsThreads) probs[i] = s_val[i] * scale;
  } else {  // the lowest index of the largest logit
    float at = INFINITY;  // (indices are below 2^24: exact)
    for (int i = tid; i < n; i += kLogitsThreads)
      if (s_val[i] == top) at = fminf(at, (float)(lo + i));
    at = cluster_reduce(at, [](float a, float c) { return fminf(a, c); }, s_warp[1], s_rank[1], rank, cluster);
    for (int i = tid; i < n; i += kLogitsThreads) probs[i] = (float)(lo + i) == at ? 1.f : 0.f;
  }
  // (every write to another CTA's memory lies before a barrier that this CTA has passed)
}

}  // namespace ooco
