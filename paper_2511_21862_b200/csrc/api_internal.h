// Host helpers shared by the translation units of the C ABI (defined in ooco_api.cu).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <utility>

#include "../../include/ooco.h"
#include "../../include/ooco_batch.h"

namespace ooco {

struct DeviceInfo {
  int sm_count = 0;
  int smem_optin = 0;
};
DeviceInfo device_info(int dev);        // attributes of device `dev`, looked up once
int current_device(int* dev);           // OOCO_OK or OOCO_E_CUDA
int fail_cuda(const char* where, long code);  // remembers where a CUDA-side failure happened; returns OOCO_E_CUDA
int validate_shape(const ooco_shape_t* s);
bool pdl_enabled();                     // tuning knob 8

// Tensor maps of a pool: bf16, boxes of tile_rows tokens (five_d: both 64-dim halves in one box); 8-bit codes.
int encode_kv_map(CUtensorMap* tm, const ooco_shape_t* s, const void* base, int tile_rows, bool five_d);
int encode_kv8_map(CUtensorMap* tm, const ooco_shape_t* s, const void* base, int tile_rows);
// ooco_rope_kv_append and its variants (norm NULL: without norms).
int rope_append(const ooco_shape_t* s, const ooco_rope_t* r, const ooco_head_norm_t* norm, int32_t T, const void* q,
                int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* positions,
                const int32_t* slot_map, void* q_out, int64_t q_out_stride, void* k_cache, void* v_cache, bool kv8,
                float k_scale, float v_scale, void* cuda_stream);

struct Range {
  const void* p;
  size_t bytes;
};
inline bool overlap(const Range& a, const Range& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

// Whether any of T rows of `la` bytes, `sa` apart from `a` on, shares memory with any of T rows of `lb` bytes, `sb` apart from
// `b` on (rows of one spacing may lie in one another's gaps, as the parts of a projection do).
inline bool rows_overlap(const void* a, int64_t sa, int64_t la, const void* b, int64_t sb, int64_t lb, int64_t T) {
  if (!overlap({a, (size_t)((T - 1) * sa + la)}, {b, (size_t)((T - 1) * sb + lb)})) return false;
  if (T == 1 || sa != sb) return true;
  const int64_t d = (int64_t)((uintptr_t)b - (uintptr_t)a) % sa, gap = d < 0 ? d + sa : d;  // b's row begins this far into a's period
  return gap < la || gap + lb > sa;
}

inline int log2_of(int x) {  // x: a power of two
  int k = 0;
  while ((1 << k) < x) ++k;
  return k;
}
inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int finish(cudaError_t e, const char* where) {
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? OOCO_OK : fail_cuda(where, (long)e);
}

// Launch with the programmatic-stream-serialization attribute (the kernel itself waits for its
// predecessor with griddepcontrol.wait) when `pdl`, else an ordinary launch; `cluster` > 1: thread-block
// clusters of that many CTAs along x.
template <typename... KArgs, typename... Args>
cudaError_t launch_clustered(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool pdl,
                             unsigned cluster, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (pdl) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = cluster;
    attr[n].val.clusterDim.y = 1;
    attr[n++].val.clusterDim.z = 1;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<Args>(args)...);
}
template <typename... KArgs, typename... Args>
cudaError_t launch_ex(void (*kern)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, bool pdl,
                      Args&&... args) {
  return launch_clustered(kern, grid, block, smem, st, pdl, 1u, std::forward<Args>(args)...);
}

}  // namespace ooco
