// fp8_quant.cu -- a matrix into E4M3 with a power-of-two scale per block of
// 128 (fp8.h): q = E4M3(x 2^-k), k the smallest integer with A <= 448 2^k, A the
// block's largest finite |x|.  Blocks run along a row (1 x 128), or are squares
// of 128 x 128, whose codes and scales are the same seen from the transpose.
// One pass gives the codes as they lie, the transpose's, or both.
#include "fp8.h"
#include "step_kernel.cuh"

namespace mpadam {

namespace {

constexpr int kQuantThreads = 256;
constexpr int kQuantWarps = kQuantThreads / 32;
constexpr int kTile = 128;     // a CTA takes a tile of 128 x 128
constexpr int kPitch = 129;    // words of a tile's row in shared memory: columns fall on different banks

// The bits of |x| where x is finite, else 0.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}
// The smallest k >= -127 with a <= 448 2^k, a given by its bits; 0 for a = 0.
// 448 = 1.75 2^8, so k = floor(log2 a) - 8, and one more where a's mantissa is
// above 1.75: adding 0x1FFFFF carries into the exponent exactly then.
__device__ __forceinline__ int block_exponent(uint32_t a) {
  return a == 0 ? 0 : max(-127, (int)((a + 0x1FFFFFu) >> 23) - 135);
}
// 2^-k for a block exponent k (-127 <= k <= 120).
__device__ __forceinline__ float inverse_scale(int k) { return __uint_as_float((uint32_t)(127 - k) << 23); }

// Two values as E4M3, nearest-even, saturating; `lo` in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t h;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(hi), "f"(lo));
  return h;
}

template <bool F32>
__device__ __forceinline__ float load(const void* x, int64_t at) {
  if (F32) return __ldg(static_cast<const float*>(x) + at);
  return __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t*>(x) + at) << 16);
}

// Codes of 128 values v[i] at i = 4 lane .. 4 lane + 3, stored where inside.
__device__ __forceinline__ void store_codes(uint8_t* q, int64_t left, int lane, const float (&v)[4], float inv) {
  const uint32_t c = e4m3x2(__fmul_rn(v[0], inv), __fmul_rn(v[1], inv)) |
                     e4m3x2(__fmul_rn(v[2], inv), __fmul_rn(v[3], inv)) << 16;
  const int i = 4 * lane;
  if (i + 4 <= left) {
    *reinterpret_cast<uint32_t*>(q + i) = c;
  } else {
    for (int j = 0; j < 4; ++j)
      if (i + j < left) q[i + j] = (uint8_t)(c >> (8 * j));
  }
}

// Row `row`'s scale of block `block`; the tile of the last block fills its group of four with 1.
__device__ __forceinline__ void store_scale(uint8_t* s, int64_t row, int64_t block, int64_t blocks, int k) {
  const int64_t groups = (blocks + 3) / 4;
  s[scale_offset(row, block, groups)] = (uint8_t)(k + 127);
  if (block == blocks - 1)
    for (int64_t b = blocks; b < 4 * groups; ++b) s[scale_offset(row, b, groups)] = 127;
}

template <bool F32>
__global__ void __launch_bounds__(kQuantThreads) quantize_kernel(const __grid_constant__ QuantArgs p) {
  extern __shared__ float tile[];  // [kTile][kPitch]
  __shared__ uint32_t square_max[kQuantWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t blocks_c = (p.cols + kTile - 1) / kTile, blocks_r = (p.rows + kTile - 1) / kTile;
  const int64_t tr = blockIdx.x / blocks_c, tc = blockIdx.x % blocks_c;
  const int64_t r0 = tr * kTile, c0 = tc * kTile;
  const int64_t left_r = p.rows - r0, left_c = p.cols - c0;

  uint32_t seen = 0;
  for (int r = warp; r < kTile; r += kQuantWarps) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = lane + 32 * j;
      const float v = r < left_r && c < left_c ? load<F32>(p.x, (r0 + r) * p.ld + c0 + c) : 0.0f;
      tile[r * kPitch + c] = v;
      seen = max(seen, finite_bits(v));
    }
  }
  if (p.square) {
    seen = __reduce_max_sync(~0u, seen);
    if (lane == 0) square_max[warp] = seen;
  }
  __syncthreads();
  int k = 0;
  if (p.square) {
    seen = 0;
    for (int w = 0; w < kQuantWarps; ++w) seen = max(seen, square_max[w]);
    k = block_exponent(seen);
  }
  if (p.q) {
    for (int r = warp; r < kTile; r += kQuantWarps) {
      float v[4];
      uint32_t a = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = tile[r * kPitch + 4 * lane + j];
        a = max(a, finite_bits(v[j]));
      }
      if (!p.square) k = block_exponent(__reduce_max_sync(~0u, a));
      const bool row = r < left_r;
      if (row) store_codes(p.q + (r0 + r) * p.ldq + c0, left_c, lane, v, inverse_scale(k));
      if (lane == 0) store_scale(p.s, r0 + r, tc, blocks_c, row ? k : 0);
    }
  }
  if (p.qt) {
    for (int c = warp; c < kTile; c += kQuantWarps) {
      float v[4];
      uint32_t a = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = tile[(4 * lane + j) * kPitch + c];
        a = max(a, finite_bits(v[j]));
      }
      if (!p.square) k = block_exponent(__reduce_max_sync(~0u, a));
      const bool col = c < left_c;
      if (col) store_codes(p.qt + (c0 + c) * p.ldqt + r0, left_r, lane, v, inverse_scale(k));
      if (lane == 0) store_scale(p.st, c0 + c, tr, blocks_r, col ? k : 0);
    }
  }
}

template <bool F32>
cudaError_t launch(const QuantArgs& a, cudaStream_t stream) {
  constexpr int kSmem = kTile * kPitch * 4;
  cudaError_t e = cudaFuncSetAttribute(quantize_kernel<F32>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e != cudaSuccess) return e;
  const int64_t tiles = ((a.cols + kTile - 1) / kTile) * ((a.rows + kTile - 1) / kTile);
  quantize_kernel<F32><<<(unsigned)tiles, kQuantThreads, kSmem, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_quantize(const QuantArgs& a, cudaStream_t stream) {
  return a.f32 ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace mpadam
