// Host helpers shared by the translation units of the C ABI (defined in ooco_api.cu).
#pragma once
#include <cuda_runtime.h>

#include <utility>

#include "../../include/ooco.h"

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
