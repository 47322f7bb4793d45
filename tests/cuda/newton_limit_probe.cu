// Test-only build of the Newton-Schulz products in which a chosen warp's waits run out: from its given look at what it waits
// for on, their limit is 0.  What ends the pair (products done, copies landed) waits as in the library.
#include "step_kernel.cuh"
#include "tcgen05.cuh"

namespace mpadam {

// The block and warp whose waits run out after `looks` looks of its lanes in all; block -1: none.
struct RunOut {
  int32_t block, warp;
  uint32_t looks;
};
__device__ RunOut g_run_out = {-1, 0, 0};
__device__ uint32_t g_looks = 0;

__device__ __forceinline__ uint32_t probe_limit() {
  const RunOut r = g_run_out;
  if ((int)blockIdx.x != r.block || (int)(threadIdx.x >> 5) != r.warp) return kSpinLimit;
  return atomicAdd(&g_looks, 1u) >= r.looks ? 0u : kSpinLimit;
}

}  // namespace mpadam

#define kSpinLimit probe_limit()
#include "muon_products.cu"

extern "C" int run_out(int32_t block, int32_t warp, uint32_t looks) {
  const mpadam::RunOut r = {block, warp, looks};
  const uint32_t none = 0;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(mpadam::g_run_out, &r, sizeof(r));
  if (e == cudaSuccess) e = cudaMemcpyToSymbol(mpadam::g_looks, &none, sizeof(none));
  if (e == cudaSuccess) e = cudaDeviceSynchronize();
  return (int)e;
}
