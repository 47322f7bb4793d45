// fp8.h -- E4M3 matrices with a power-of-two scale per block of 128: their
// storage, and the launch arguments of the kernels that write and multiply
// them (internal to the CUDA library; the C ABI is mpadam_e4m3_* in
// include/mpadam.h).
#pragma once

#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

namespace mpadam {

constexpr int kScaleBlock = 128;  // values along a row that share a scale
constexpr int kScaleTile = 512;   // bytes of scales of 128 rows x 4 blocks

// Scales are stored in the order in which the tensor cores take them: tiles of
// 128 rows x 4 blocks, [row tile][group of 4 blocks][32][4][4], the four blocks
// of row 32 j + i at [i][j].  A tile is 512 contiguous bytes, copied to tensor
// memory as it lies.
__host__ __device__ inline int64_t scale_offset(int64_t row, int64_t block, int64_t groups) {
  return ((row >> 7) * groups + (block >> 2)) * kScaleTile + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

struct QuantArgs {
  const void* x;       // [rows, cols], binary32 or BF16, row stride ld
  int64_t rows, cols, ld;
  uint8_t* q;          // [rows, cols] codes, row stride ldq, or nullptr
  uint8_t* s;          // their scales
  uint8_t* qt;         // [cols, rows] codes of the transpose, row stride ldqt, or nullptr
  uint8_t* st;
  int64_t ldq, ldqt;
  int32_t f32, square;
  int32_t vec;         // rows of x start on 16-byte boundaries (set by the launch)
};

cudaError_t launch_quantize(const QuantArgs& a, cudaStream_t stream);

struct MatmulArgs {
  CUtensorMap a, b;            // codes [m, k] and [n, k]
  CUtensorMap sa_map, sb_map;  // their scales, [row tiles, groups of 4 blocks, 128 words] (CTA pairs only)
  const uint8_t* sa;           // scales of a and b
  const uint8_t* sb;
  void* d;                     // [m, n], row stride ldd
  int64_t ldd;
  int32_t m, n, k;
  int32_t f32, accumulate;
  int32_t split;
  int32_t b_early;             // b was complete before the kernel that this launch follows, which writes a (not for pairs)
  int32_t* err;                // device error word
};

// How a product of this shape is cut up, and its launch.
struct MatmulPlan {
  int tile;    // rows of a per tile
  int split;   // CTAs that share a tile's k
  bool pair;   // tiles of 256 x `tile` by pairs of CTAs, which need the scales' maps
  int box() const { return pair ? tile / 2 : tile; }  // rows of a's boxes
};
MatmulPlan matmul_plan(int64_t m, int64_t n, int64_t k);
cudaError_t launch_matmul(MatmulArgs& a, const MatmulPlan& plan, cudaStream_t stream);
// Address of the device error word that matmul kernels set.
cudaError_t matmul_error_word(int32_t** p);

}  // namespace mpadam
