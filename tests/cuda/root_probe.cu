// Test-only probes of the AdamW step's arithmetic.  root_probe: root2 against the
// correctly rounded square root on every binary32 value whose bits are first ..
// first + count - 1.  reciprocal_probe: the same for reciprocal2.
// quotient_probe: quotient2 against the correctly rounded quotient of a[i] and
// d[i].  Each counts what differs.
#include <cstdint>
#include <cuda_runtime.h>

#include "adamw_math.cuh"

__global__ void roots(uint32_t first, uint32_t count, unsigned long long* wrong) {
  for (uint64_t i = blockIdx.x * (uint64_t)blockDim.x + threadIdx.x; i < count; i += (uint64_t)gridDim.x * blockDim.x) {
    const float x = __uint_as_float(first + (uint32_t)i);
    float r0, r1;
    mpadam::unpk(mpadam::root2(mpadam::pk(x, x)), r0, r1);
    const float want = __fsqrt_rn(x);
    if (__float_as_uint(r0) != __float_as_uint(want) || __float_as_uint(r1) != __float_as_uint(want)) atomicAdd(wrong, 1ull);
  }
}
__global__ void reciprocals(uint32_t first, uint32_t count, unsigned long long* wrong) {
  for (uint64_t i = blockIdx.x * (uint64_t)blockDim.x + threadIdx.x; i < count; i += (uint64_t)gridDim.x * blockDim.x) {
    const float x = __uint_as_float(first + (uint32_t)i);
    float r0, r1;
    mpadam::unpk(mpadam::reciprocal2(mpadam::pk(-x, -x)), r0, r1);
    const float want = __frcp_rn(x);
    if (__float_as_uint(r0) != __float_as_uint(want) || __float_as_uint(r1) != __float_as_uint(want)) atomicAdd(wrong, 1ull);
  }
}
__global__ void quotients(const float* a, const float* d, int64_t n, unsigned long long* wrong) {
  for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) {
    float q0, q1;
    mpadam::unpk(mpadam::quotient2(mpadam::pk(a[i], -a[i]), mpadam::pk(-d[i], -d[i])), q0, q1);
    const float want = __fdiv_rn(a[i], d[i]);
    if (__float_as_uint(q0) != __float_as_uint(want) || __float_as_uint(-q1) != __float_as_uint(want)) atomicAdd(wrong, 1ull);
  }
}

extern "C" int root_probe(uint32_t first, uint32_t count, unsigned long long* wrong) {
  roots<<<2048, 256>>>(first, count, wrong);
  return (int)cudaDeviceSynchronize();
}
extern "C" int reciprocal_probe(uint32_t first, uint32_t count, unsigned long long* wrong) {
  reciprocals<<<2048, 256>>>(first, count, wrong);
  return (int)cudaDeviceSynchronize();
}
extern "C" int quotient_probe(const float* a, const float* d, int64_t n, unsigned long long* wrong) {
  quotients<<<2048, 256>>>(a, d, n, wrong);
  return (int)cudaDeviceSynchronize();
}
