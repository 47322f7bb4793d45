// Test-only build of a source's kernels (PROBE_SOURCE) in which a chosen wait says that it gave up, although what it waited
// for has come: linked with the library's other objects in place of that source's.
#include "step_kernel.cuh"

#ifndef PROBE_SOURCE
#define PROBE_SOURCE "fp8_matmul.cu"
#endif

namespace mpadam {

// The block, warp and lane (-1: all of the warp's) whose waits of this parity give up; block -1: none.
struct GiveUp {
  int32_t block, warp, lane;
  uint32_t parity;
};
__device__ GiveUp g_give_up = {-1, 0, 0, 0};

__device__ __forceinline__ bool gives_up(uint32_t parity) {
  const GiveUp g = g_give_up;
  return (int)blockIdx.x == g.block && (int)(threadIdx.x >> 5) == g.warp && (g.lane < 0 || (int)(threadIdx.x & 31) == g.lane) &&
         parity == g.parity;
}
__device__ __forceinline__ bool probe_wait(uint32_t bar, uint32_t parity) { return mbar_wait(bar, parity) && !gives_up(parity); }
// (each attempt waits until the phase is there, and then says that it is not: the caller's limit is soon reached)
__device__ __forceinline__ bool probe_try(uint32_t bar, uint32_t parity) {
  return gives_up(parity) ? mbar_wait(bar, parity) && false : mbar_try_wait(bar, parity);
}

}  // namespace mpadam

#define mbar_wait probe_wait
#define mbar_try_wait probe_try
#include PROBE_SOURCE

extern "C" int give_up(int32_t block, int32_t warp, int32_t lane, uint32_t parity) {
  const mpadam::GiveUp g = {block, warp, lane, parity};
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(mpadam::g_give_up, &g, sizeof(g));
  return (int)e;
}
