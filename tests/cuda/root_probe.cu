// Test-only probe: root2 (the AdamW step's square root) against the correctly
// rounded one on every binary32 value whose bits are first .. first + count - 1,
// and the hardware reciprocal's largest relative error over the same values
// (where they and their reciprocals are normal).
#include <cstdint>
#include <cuda_runtime.h>

#include "adamw_math.cuh"

__global__ void probe(uint32_t first, uint32_t count, unsigned long long* wrong, float* worst) {
  float w = 0.0f;
  for (uint64_t i = blockIdx.x * (uint64_t)blockDim.x + threadIdx.x; i < count; i += (uint64_t)gridDim.x * blockDim.x) {
    const float x = __uint_as_float(first + (uint32_t)i);
    float r0, r1;
    mpadam::unpk(mpadam::root2(mpadam::pk(x, x)), r0, r1);
    const float want = __fsqrt_rn(x);
    if (__float_as_uint(r0) != __float_as_uint(want) || __float_as_uint(r1) != __float_as_uint(want)) atomicAdd(wrong, 1ull);
    if (x >= 0x1p-125f && x <= 0x1p125f) {
      const double r = mpadam::rcp_approx_ftz(x);
      w = fmaxf(w, (float)fabs(r * (double)x - 1.0));
    }
  }
  atomicMax(reinterpret_cast<int*>(worst), __float_as_int(w));
}

extern "C" int root_probe(uint32_t first, uint32_t count, unsigned long long* wrong, float* worst) {
  probe<<<2048, 256>>>(first, count, wrong, worst);
  return (int)cudaDeviceSynchronize();
}
