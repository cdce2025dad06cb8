// Host-side helpers shared by the library's translation units.  Not part of the C ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace osdp {

// OSDP_OK for cudaSuccess; otherwise remembers the error for osdp_last_cuda_error() and returns OSDP_ERR_CUDA.
int report_cuda(cudaError_t e);
// Number of SMs of the current device (cached per device).
int sm_count(int *sms);

// A 3-D tensor map (strides in bytes); swizzle: 128-byte, else none.
int encode_map3d(CUtensorMap *map, CUtensorMapDataType dt, const void *base, const cuuint64_t (&dims)[3], const cuuint64_t (&strides)[2],
                 const cuuint32_t (&box)[3], bool swizzle);

inline int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool aligned_to(const void *p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Launch that takes part in programmatic dependent launch: the kernel may be scheduled while the previous kernel
// on the stream drains and calls griddepcontrol.wait before it touches global memory.  cluster_x > 1: the grid is
// made of clusters of that many blocks.
template <typename... KArgs, typename... Args>
int launch_overlapped(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, int cluster_x, cudaStream_t stream,
                      const Args &...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster_x;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster_x > 1 ? 2 : 1;
  return report_cuda(cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...));
}

}  // namespace osdp
