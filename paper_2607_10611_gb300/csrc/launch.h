// launch.h -- launches whose CTAs may set up while earlier kernels of the stream
// end (internal to the CUDA library).  The kernels execute griddepcontrol.wait
// before they touch global memory.
#pragma once

#include <cuda_runtime.h>

namespace mpadam {

// cluster: CTAs per cluster, 0 where the kernel fixes it or has none.  args: the kernel's one parameter.
template <typename Args>
cudaError_t launch_dependent(const void* kernel, unsigned grid, unsigned threads, int cluster, int smem, const Args* args,
                             cudaStream_t stream) {
  cudaLaunchAttribute attr[2] = {};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = cluster ? 2 : 1;
  void* params[] = {const_cast<Args*>(args)};
  return cudaLaunchKernelExC(&cfg, kernel, params);
}

}  // namespace mpadam
