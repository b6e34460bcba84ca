// Device helpers shared by kernels of several files: scans over a CTA, distributed shared memory, pieces of 16-bit rows.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "ptx.cuh"

namespace ooco {

constexpr int kTreeMaxNodes = 256;
constexpr int kScanThreads = 1024;

// Inclusive scan of one value per thread over a block of kScanThreads threads; *total = the sum.
__device__ __forceinline__ long long block_scan(long long v, long long* s_warp, long long* total) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  __syncthreads();  // earlier readers of s_warp are done
  if (lane == 31) s_warp[wid] = v;
  __syncthreads();
  if (wid == 0) {
    long long w = s_warp[lane];
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += u;
    }
    s_warp[lane] = w;
  }
  __syncthreads();
  *total = s_warp[31];
  return v + (wid ? s_warp[wid - 1] : 0);
}

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
// Address of `addr` (this CTA's shared memory) in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t map_cluster(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, int v) {
  asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

struct RopeParams {
  const uint16_t *q, *k, *v;  // bf16 rows
  uint16_t* q_out;
  uint8_t *k_cache, *v_cache;
  const int32_t *positions, *slots;
  const float* inv_freq;
  int64_t q_stride, k_stride, v_stride, q_out_stride;  // elements
  int64_t bstr, hstr, tstr;                            // elements of the cache
  int32_t T, Hq, Hkv, half, bs_log2, tile;             // half = rot_dim / 2; tile = tokens per CTA and step
  int64_t num_slots;
  float magnitude, k_scale, v_scale;
};

constexpr int kRopeThreads = 256, kRopeMaxTile = 4, kRopeBatch = 2;

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Eight fp32 values as a 16-byte (bf16) or 8-byte (E4M3 of value / scale) piece of a row.
__device__ __forceinline__ uint4 pack8_bf16(const float (&x)[8]) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ uint2 pack8_e4m3(const float (&x)[8], float scale) {
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float2 v = make_float2(__fdiv_rn(x[i], scale), __fdiv_rn(x[i + 1], scale));
    w[i >> 2] |= (uint32_t)__nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3) << (8 * (i & 3));
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void unpack8(const uint4 w, float (&x)[8]) {
  const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = bf16_lo(in[i]);
    x[2 * i + 1] = bf16_hi(in[i]);
  }
}

}  // namespace ooco
