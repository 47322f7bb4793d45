// Test-only build of the 8-bit products in which all epilogue warps of a chosen block give up after two microseconds, with copies
// and products in flight.  Everybody else's waits are the library's.
#include "step_kernel.cuh"
#include "tcgen05.cuh"

namespace mpadam {

__device__ int32_t g_leaves = -1;  // the block

__device__ __forceinline__ bool leaves() {
  if ((int)blockIdx.x != g_leaves || threadIdx.x < 4 * 32) return false;
  const long long begun = clock64();
  while (clock64() - begun < 4000) {}  // (the producer has looked whether anyone has given up)
  return true;
}
__device__ __forceinline__ bool probe_warp_wait(uint32_t bar, uint32_t parity) { return !leaves() && warp_wait(bar, parity); }
__device__ __forceinline__ bool probe_warp_wait_cluster(uint32_t bar, uint32_t parity) {
  return !leaves() && warp_wait_cluster(bar, parity);
}

}  // namespace mpadam

#define warp_wait probe_warp_wait
#define warp_wait_cluster probe_warp_wait_cluster
#include "fp8_matmul.cu"

extern "C" int give_up(int32_t block, int32_t, int32_t, uint32_t) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(mpadam::g_leaves, &block, sizeof(block));
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  return (int)e;
}
