// layer_norm.h -- launch arguments of layer normalisation (internal to the CUDA
// library; the C ABI is mpadam_layer_norm_* in include/mpadam.h).
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace mpadam {

struct NormForwardArgs {
  const void* x;  // [rows, cols], binary32 or BF16, row stride ldx
  const void* w;  // cols each, or nullptr
  const void* b;
  void* y;        // as x, row stride ldy
  float* mean;    // rows each, or nullptr
  float* rstd;
  int64_t rows, cols, ldx, ldy;
  float eps, inv_cols, all_cols;  // 1 / cols and cols
  int32_t x_f32, w_f32;
};

struct NormBackwardArgs {
  const void* x;
  const void* dy;
  const void* w;       // or nullptr
  const float* mean;
  const float* rstd;
  void* dx;            // or nullptr
  float* partial;      // [parts, 2, cols]: sums of dy n and of dy over each part's rows, or nullptr
  int64_t rows, cols, ldx, lddy, lddx;
  float inv_cols;
  int32_t x_f32, w_f32;
  int32_t parts;
};

struct NormSumArgs {
  const float* partial;
  void* dw;            // cols each, or nullptr
  void* db;
  int64_t cols;
  int32_t parts, w_f32;
};

// Parts that the rows' sums are made in: a rule on the sizes alone, so that the same sizes give the same bits.
int norm_parts(int64_t rows, int64_t cols);
cudaError_t launch_norm_forward(const NormForwardArgs& a, cudaStream_t stream);
cudaError_t launch_norm_backward(const NormBackwardArgs& a, cudaStream_t stream);
cudaError_t launch_norm_sums(const NormSumArgs& a, cudaStream_t stream);

}  // namespace mpadam
