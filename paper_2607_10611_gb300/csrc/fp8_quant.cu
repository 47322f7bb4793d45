// fp8_quant.cu -- a matrix into E4M3 with a power-of-two scale per block of
// 128 (fp8.h): q = E4M3(x 2^-k), k the smallest integer with A <= 448 2^k, A the
// block's largest finite |x|.  Blocks run along a row (1 x 128), or are squares
// of 128 x 128, whose codes and scales are the same seen from the transpose.
// One pass gives the codes as they lie, the transpose's, or both.
#include "fp8.h"
#include "launch.h"
#include "step_kernel.cuh"

namespace mpadam {

namespace {

// A CTA takes a tile of 128 x 128 and a thread a patch of 8 x 8, in registers
// from the load to the last store: nothing is staged.  A warp is 4 patches wide
// and 8 high, so that every access, to either output, is of whole 32-byte
// sectors: 64 bytes of a row of x in BF16, 32 of a row of codes, 64 of a row of
// the transpose's.  Memory bounds it: 8192 x 4096 in BF16 with its transpose takes
// 22.5 us (134.7 MB, 6.0 TB/s, 0.89 of the copy's rate, 2 us of them the launch),
// GPT-2's embedding in binary32, in squares, 39.7 (232 MB, 5.8 TB/s).  Whole tiles
// have no look at their edges (with one at every access, 17 instructions a value:
// 25.2 and 43.6 us).  Four CTAs an SM in BF16 (three: 23.6 us, five spill: 25.6),
// two in binary32 (three spill: 47.0).  Through shared memory, with both outputs
// gathered from it, they took 131 and 107.
constexpr int kQuantThreads = 256;
constexpr int kTile = 128;

// The smallest k >= -127 with a <= 448 2^k, a given by its bits; 0 for a = 0.
// 448 = 1.75 2^8, so k = floor(log2 a) - 8, and one more where a's mantissa is
// above 1.75: adding 0x1FFFFF carries into the exponent exactly then.
__device__ __forceinline__ int block_exponent(uint32_t a) {
  return a == 0 ? 0 : max(-127, (int)((a + 0x1FFFFFu) >> 23) - 135);
}
// 2^-k for a block exponent k (-127 <= k <= 120).
__device__ __forceinline__ float inverse_scale(int k) { return __uint_as_float((uint32_t)(127 - k) << 23); }

// Two values times inv as E4M3, nearest-even, saturating; `lo` in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi, float inv) {
  uint16_t h;
  unpk(mul2_rn(pk(lo, hi), pk(inv, inv)), lo, hi);
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(hi), "f"(lo));
  return h;
}

// A patch: 8 rows of 8 values, BF16 ones packed in pairs.
template <bool F32>
struct Patch;

template <>
struct Patch<true> {
  float x[8][8];
  static constexpr uint32_t kInf = 0x7F800000u;
  __device__ __forceinline__ void load_row(const void* p, int64_t at, int64_t left, bool vec, int r) {
    const float* q = static_cast<const float*>(p) + at;
    if (vec && left >= 8) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(q)), b = __ldg(reinterpret_cast<const float4*>(q) + 1);
      x[r][0] = a.x, x[r][1] = a.y, x[r][2] = a.z, x[r][3] = a.w;
      x[r][4] = b.x, x[r][5] = b.y, x[r][6] = b.z, x[r][7] = b.w;
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) x[r][c] = c < left ? q[c] : 0.0f;
    }
  }
  __device__ __forceinline__ void load_whole(const uint8_t* p, int r) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    x[r][0] = a.x, x[r][1] = a.y, x[r][2] = a.z, x[r][3] = a.w;
    x[r][4] = b.x, x[r][5] = b.y, x[r][6] = b.z, x[r][7] = b.w;
  }
  __device__ __forceinline__ void clear_row(int r) {
#pragma unroll
    for (int c = 0; c < 8; ++c) x[r][c] = 0.0f;
  }
  __device__ __forceinline__ float get(int r, int c) const { return x[r][c]; }
  // Largest |value| of each row and column over the warp's lanes that share it, as bits; FINITE: of the finite ones.
  template <bool FINITE>
  __device__ __forceinline__ void maxima(uint32_t (&rows)[8], uint32_t (&cols)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) rows[i] = cols[i] = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        uint32_t a = __float_as_uint(x[r][c]) & 0x7FFFFFFFu;
        if (FINITE && a >= kInf) a = 0;
        rows[r] = max(rows[r], a);
        cols[c] = max(cols[c], a);
      }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) rows[i] = max(rows[i], __shfl_xor_sync(~0u, rows[i], d));
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) cols[i] = max(cols[i], __shfl_xor_sync(~0u, cols[i], d));
    }
  }
  static __device__ __forceinline__ uint32_t wide(uint32_t a) { return a; }
};

template <>
struct Patch<false> {
  uint32_t x[8][4];
  static constexpr uint32_t kInf = 0x7F80u;
  __device__ __forceinline__ void load_row(const void* p, int64_t at, int64_t left, bool vec, int r) {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    if (vec && left >= 8) {
      const uint4 a = __ldg(reinterpret_cast<const uint4*>(q));
      x[r][0] = a.x, x[r][1] = a.y, x[r][2] = a.z, x[r][3] = a.w;
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        x[r][c] = (2 * c < left ? (uint32_t)q[2 * c] : 0u) | (2 * c + 1 < left ? (uint32_t)q[2 * c + 1] << 16 : 0u);
    }
  }
  __device__ __forceinline__ void load_whole(const uint8_t* p, int r) {
    const uint4 a = __ldg(reinterpret_cast<const uint4*>(p));
    x[r][0] = a.x, x[r][1] = a.y, x[r][2] = a.z, x[r][3] = a.w;
  }
  __device__ __forceinline__ void clear_row(int r) { x[r][0] = x[r][1] = x[r][2] = x[r][3] = 0; }
  __device__ __forceinline__ float get(int r, int c) const { return c & 1 ? bf16_hi(x[r][c / 2]) : bf16_lo(x[r][c / 2]); }
  // In 16-bit halves, two rows or columns to a word.
  template <bool FINITE>
  __device__ __forceinline__ void maxima(uint32_t (&rows)[8], uint32_t (&cols)[8]) const {
    uint32_t rp[4], cp[4] = {0, 0, 0, 0};
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      uint32_t m = 0;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t a = x[r][c] & 0x7FFF7FFFu;
        if (FINITE) a &= ~__vcmpgeu2(a, 0x7F807F80u);
        m = __vmaxu2(m, a);
        cp[c] = __vmaxu2(cp[c], a);
      }
      m = __vmaxu2(m, m >> 16);  // in the low half
      rp[r / 2] = r & 1 ? __byte_perm(rp[r / 2], m, 0x5410) : m;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) rp[i] = __vmaxu2(rp[i], __shfl_xor_sync(~0u, rp[i], d));
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) cp[i] = __vmaxu2(cp[i], __shfl_xor_sync(~0u, cp[i], d));
      rows[2 * i] = rp[i] & 0xFFFFu, rows[2 * i + 1] = rp[i] >> 16;
      cols[2 * i] = cp[i] & 0xFFFFu, cols[2 * i + 1] = cp[i] >> 16;
    }
  }
  static __device__ __forceinline__ uint32_t wide(uint32_t a) { return a << 16; }
};

// 8 codes, `left` of them inside.
__device__ __forceinline__ void store_codes(uint8_t* q, int64_t left, uint2 c) {
  if (left >= 8) {
    *reinterpret_cast<uint2*>(q) = c;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) q[j] = (uint8_t)((j < 4 ? c.x : c.y) >> (8 * (j & 3)));
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
__global__ void __launch_bounds__(kQuantThreads, F32 ? 2 : 4) quantize_kernel(const __grid_constant__ QuantArgs p) {
  __shared__ uint32_t row_max[4][kTile], col_max[2][kTile];
  __shared__ alignas(16) float row_inv[kTile], col_inv[kTile];
  // A product that follows may set itself up from here on; it waits for this kernel's end before it reads.
  asm volatile("griddepcontrol.wait;\ngriddepcontrol.launch_dependents;" ::: "memory");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int wc = warp & 3, wr = warp >> 2;
  const int pc = wc * 32 + (lane & 3) * 8, pr = wr * 64 + (lane >> 2) * 8;  // the patch's place in the tile
  const uint32_t blocks_c = (uint32_t)((p.cols + kTile - 1) / kTile), blocks_r = (uint32_t)((p.rows + kTile - 1) / kTile);
  const uint32_t tr = blockIdx.x / blocks_c, tc = blockIdx.x - tr * blocks_c;
  const int64_t r0 = (int64_t)tr * kTile + pr, c0 = (int64_t)tc * kTile + pc;
  const int64_t left_r = p.rows - r0, left_c = p.cols - c0;
  // A tile that is whole and can be read in vectors, as most are, needs no look at every access.
  const bool whole = p.vec && (int64_t)(tr + 1) * kTile <= p.rows && (int64_t)(tc + 1) * kTile <= p.cols;

  Patch<F32> x;
  if (whole) {
    const uint8_t* at = static_cast<const uint8_t*>(p.x) + (r0 * p.ld + c0) * (F32 ? 4 : 2);
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      x.load_whole(at, r);
      at += p.ld * (F32 ? 4 : 2);
    }
  } else {
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      if (r < left_r && left_c > 0) x.load_row(p.x, (r0 + r) * p.ld + c0, left_c, p.vec, r);
      else x.clear_row(r);
    }
  }
  // Maxima of all |values|; where one is not finite, once more over the finite ones.
  uint32_t rows[8], cols[8];
  x.template maxima<false>(rows, cols);
  auto publish = [&] {
    if ((lane & 3) == 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) row_max[wc][pr + i] = rows[i];
    }
    if (lane < 4) {
#pragma unroll
      for (int i = 0; i < 8; ++i) col_max[wr][pc + i] = cols[i];
    }
  };
  publish();
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, rows[i]);
  if (__syncthreads_or(most >= Patch<F32>::kInf)) {
    x.template maxima<true>(rows, cols);
    publish();
    __syncthreads();
  }
  // Half of the threads finish a row each, the others a column.
  {
    const int i = threadIdx.x & 127;
    const bool is_row = threadIdx.x < 128;
    uint32_t a;
    if (p.square) {
      a = max(max(row_max[0][i], row_max[1][i]), max(row_max[2][i], row_max[3][i]));
      a = __reduce_max_sync(~0u, a);
      __syncthreads();
      if (lane == 0) row_max[0][warp] = a;
      __syncthreads();
      a = max(max(row_max[0][0], row_max[0][1]), max(row_max[0][2], row_max[0][3]));
    } else {
      a = is_row ? max(max(row_max[0][i], row_max[1][i]), max(row_max[2][i], row_max[3][i])) : max(col_max[0][i], col_max[1][i]);
    }
    const int k = block_exponent(Patch<F32>::wide(a));
    if (is_row) {
      row_inv[i] = inverse_scale(k);
      if (p.q) store_scale(p.s, tr * kTile + i, tc, blocks_c, tr * kTile + i < p.rows ? k : 0);
    } else {
      col_inv[i] = inverse_scale(k);
      if (p.qt) store_scale(p.st, tc * kTile + i, tr, blocks_r, tc * kTile + i < p.cols ? k : 0);
    }
  }
  __syncthreads();
  // Codes of a row (`i`) or column of the patch.
  auto row_codes = [&](int i, float inv) {
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = e4m3x2(x.get(i, 2 * j), x.get(i, 2 * j + 1), inv);
    return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
  };
  auto col_codes = [&](int i, float inv) {
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = e4m3x2(x.get(2 * j, i), x.get(2 * j + 1, i), inv);
    return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
  };
  if (whole) {
    if (p.q) {
      uint8_t* at = p.q + r0 * p.ldq + c0;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        *reinterpret_cast<uint2*>(at) = row_codes(r, row_inv[pr + r]);
        at += p.ldq;
      }
    }
    if (p.qt) {
      uint8_t* at = p.qt + c0 * p.ldqt + r0;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        *reinterpret_cast<uint2*>(at) = col_codes(c, col_inv[pc + c]);
        at += p.ldqt;
      }
    }
    return;
  }
  if (p.q && left_c > 0) {
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (r < left_r) store_codes(p.q + (r0 + r) * p.ldq + c0, left_c, row_codes(r, row_inv[pr + r]));
  }
  if (p.qt && left_r > 0) {
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (c < left_c) store_codes(p.qt + (c0 + c) * p.ldqt + r0, left_r, col_codes(c, col_inv[pc + c]));
  }
}

template <bool F32>
cudaError_t launch(QuantArgs a, cudaStream_t stream) {
  const int64_t size = F32 ? 4 : 2;
  a.vec = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && (a.ld * size % 16 == 0 || a.rows == 1);
  const int64_t tiles = ((a.cols + kTile - 1) / kTile) * ((a.rows + kTile - 1) / kTile);
  return launch_dependent((const void*)quantize_kernel<F32>, (unsigned)tiles, kQuantThreads, 0, 0, &a, stream);
}

}  // namespace

cudaError_t launch_quantize(const QuantArgs& a, cudaStream_t stream) {
  return a.f32 ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace mpadam
