// Test-only probes of the AdamW step's stochastic roundings by the hardware's
// conversions, against the definition in integers, for every value that they are
// used for: random bits that are all 0, all 1, just enough to round up, one too
// few, and arbitrary ones, in either place of the pair.  Each counts what differs.
#include <cstdint>
#include <cuda_runtime.h>

#include "adamw_math.cuh"

namespace {

__device__ uint32_t mix(uint32_t x) {
  x = (x ^ x >> 16) * 0x7FEB352Du;
  x = (x ^ x >> 15) * 0x846CA68Bu;
  return x ^ x >> 16;
}

// |y| <= 448 given by its bits: its value in units of 2^-29 below 2^-6 (rounded there, ties to even), else its bits;
// r is added below the grid's last bit, and the code is read off.
__device__ uint32_t code_of(uint32_t bits, uint32_t r) {
  const uint32_t sign = bits >> 31 << 7, a = bits & 0x7FFFFFFFu, e = a >> 23;
  if (e >= 121) return sign | ((((a + (r << 4)) >> 20) - (120u << 3)) & 0xFFu);  // 2^-6 has the exponent field 121, E4M3's 1
  uint32_t n = 0;  // y in units of 2^-29
  if (e >= 97) {  // from 2^-30 on
    const uint32_t mant = (a & 0x7FFFFFu) | 0x800000u, cut = 121 - e;  // y = mant 2^(e - 150) = mant 2^-29 / 2^cut
    const uint32_t rest = mant & ((1u << cut) - 1), half = 1u << (cut - 1);
    n = mant >> cut;
    n += rest > half || (rest == half && (n & 1));
  }
  return sign | ((n + (r << 4)) >> 20);  // codes are multiples of 2^-9
}

__global__ void codes(unsigned long long* wrong) {
  for (uint64_t i = blockIdx.x * (uint64_t)blockDim.x + threadIdx.x; i <= 0x43E00000u; i += (uint64_t)gridDim.x * blockDim.x) {
    for (int t = 0; t < 6; ++t) {
      const uint32_t h = mix((uint32_t)i * 8 + t), enough = 0x10000u - ((uint32_t)i >> 4 & 0xFFFFu);
      const uint32_t r = (t == 0 ? 0 : t == 1 ? 0xFFFFu : t == 2 ? enough : t == 3 ? enough - 1 : h) & 0xFFFFu, r2 = h >> 16;
      const uint32_t y = (uint32_t)i | (h & 0x80000000u), z = mix(h + 1) % 0x43E00001u;
      const float fy = mpadam::settle(__uint_as_float(y)), fz = mpadam::settle(__uint_as_float(z));
      const uint32_t wy = code_of(y, r), wz = code_of(z, r2);
      if (mpadam::rs_codes(fy, fz, r | r2 << 16) != (wy | wz << 16)) atomicAdd(wrong, 1ull);
      if (mpadam::rs_codes(fz, fy, r2 | r << 16) != (wz | wy << 16)) atomicAdd(wrong, 1ull);
    }
  }
}

__global__ void pairs(unsigned long long* wrong) {
  for (uint64_t i = blockIdx.x * (uint64_t)blockDim.x + threadIdx.x; i < 1ull << 32; i += (uint64_t)gridDim.x * blockDim.x) {
    const uint32_t x = (uint32_t)i;
    if ((x & 0x7F800000u) == 0x7F800000u) continue;
    for (int t = 0; t < 5; ++t) {
      const uint32_t h = mix(x * 8 + t), enough = 0x10000u - (x & 0xFFFFu);
      const uint32_t r = (t == 0 ? 0 : t == 1 ? 0xFFFFu : t == 2 ? enough : t == 3 ? enough - 1 : h) & 0xFFFFu, r2 = h >> 16;
      const uint32_t z = mix(h + 3) & 0xBFFFFFFFu;  // finite
      const uint32_t wx = (x + r) >> 16, wz = (z + r2) >> 16;
      if (mpadam::rs_bf16x2(__uint_as_float(x), __uint_as_float(z), r | r2 << 16) != (wx | wz << 16)) atomicAdd(wrong, 1ull);
      if (mpadam::rs_bf16x2(__uint_as_float(z), __uint_as_float(x), r2 | r << 16) != (wz | wx << 16)) atomicAdd(wrong, 1ull);
    }
  }
}

}  // namespace

extern "C" int codes_probe(unsigned long long* wrong) {
  codes<<<2048, 256>>>(wrong);
  return (int)cudaDeviceSynchronize();
}
extern "C" int pairs_probe(unsigned long long* wrong) {
  pairs<<<2048, 256>>>(wrong);
  return (int)cudaDeviceSynchronize();
}
