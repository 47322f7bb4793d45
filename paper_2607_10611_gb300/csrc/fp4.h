// fp4.h -- launch arguments of products with NVFP4 weights (internal to the CUDA
// library; the C ABI is mpadam_nvfp4_linear in include/mpadam.h).
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace mpadam {

struct Fp4Args {
  const void* x;          // [tokens, cols], binary32 or BF16, row stride ldx
  const uint8_t* codes;   // E2M1, two per byte, of [rows, cols] as one flat array
  const uint8_t* scales;  // E4M3, one per 16 consecutive codes
  void* y;                // [tokens, rows], as x, row stride ldy
  int64_t tokens, rows, cols, ldx, ldy;
  float global_scale;
  int32_t x_f32;
  int32_t vec_x;          // rows of x start on 16-byte boundaries (set by the launch, as the next)
  int32_t split;          // blocks of a cluster that share k
  float up, out0, out1;   // of the scales, and of the sums
};

cudaError_t launch_fp4_linear(const Fp4Args& a, cudaStream_t stream);

}  // namespace mpadam
