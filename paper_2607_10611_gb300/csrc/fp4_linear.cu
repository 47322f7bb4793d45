// fp4_linear.cu -- few tokens times a weight in NVFP4, as M+Adam's step leaves it:
//   y[t, n] = G sum over k of x[t, k] q[n, k] s[n, k / 16]
// with E2M1 codes q, E4M3 scales s per 16 consecutive weights and a binary32
// scale G.  Sums are in binary32, one rounding follows.  Weights are q s 2^e, with
// 2^e the power of two in G (within limits, see launch_fp4_linear): a sum is then
// about as large as its result, and leaves binary32's range where that does.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "fp4.h"
#include "launch.h"
#include "step_kernel.cuh"
#include "tcgen05.cuh"

namespace mpadam {

namespace {

constexpr int kSms = 152;    // GB300
constexpr int kWarps = 8;
constexpr int kFp4Threads = 32 * kWarps;
constexpr int kChunk = 128;  // values of k that a warp takes at once: 32 a lane, 16 bytes of codes, two scales

__device__ __forceinline__ void let_later_kernels_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ float get(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float get(const uint16_t* p, int64_t i) { return __uint_as_float((uint32_t)p[i] << 16); }
__device__ __forceinline__ void put(float* p, int64_t i, float x) { p[i] = x; }
__device__ __forceinline__ void put(uint16_t* p, int64_t i, float x) { p[i] = (uint16_t)bf16x2_rn(x, 0.0f); }

// Two E4M3 scales as binary32.
__device__ __forceinline__ float2 scale_values(uint16_t codes) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(codes));
  float2 s;
  asm("{\n .reg .f16 lo, hi;\n mov.b32 {lo, hi}, %2;\n cvt.f32.f16 %0, lo;\n cvt.f32.f16 %1, hi;\n}" : "=f"(s.x), "=f"(s.y) : "r"(h));
  return s;
}

// Two codes of `word`, of the nibbles I and I + 4, times 2^-126 as BF16 each: a
// code's sign, exponent and mantissa in the places of BF16's sign and of the last
// two exponent bits and first mantissa bit.  E2M1's subnormal becomes BF16's.
template <int I>
__device__ __forceinline__ uint32_t code_pair(uint32_t word) {
  constexpr int kSign = 12 - 4 * I, kRest = 6 - 4 * I;
  const uint32_t sign = kSign > 0 ? word << kSign : word, rest = kRest > 0 ? word << kRest : word >> -kRest;
  return (sign & 0x80008000u) | (rest & 0x01C001C0u);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// y of a sum: times what G is of 2^e, in two factors of which one is a power of two.
__device__ __forceinline__ float result_of(const Fp4Args& p, float sum) { return __fmul_rn(__fmul_rn(sum, p.out0), p.out1); }

// Two scales times `up`, 2^(126 + e), twice each: a weight is then q s 2^e, which BF16 holds exactly.
struct Scales {
  uint32_t s[2];
  __device__ __forceinline__ Scales(uint16_t codes, float up) {
    const float2 v = scale_values(codes);
    const float lo = __fmul_rn(v.x, up), hi = __fmul_rn(v.y, up);
    s[0] = bf16x2_rn(lo, lo), s[1] = bf16x2_rn(hi, hi);
  }
};
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
// Eight codes of one row and eight of the row 8 below, as the first operands of two products.
__device__ __forceinline__ void weights(uint32_t w0, uint32_t w1, uint32_t s0, uint32_t s1, uint32_t (&a0)[4], uint32_t (&a1)[4]) {
  a0[0] = mul_bf16x2(code_pair<0>(w0), s0), a0[1] = mul_bf16x2(code_pair<0>(w1), s1);
  a0[2] = mul_bf16x2(code_pair<1>(w0), s0), a0[3] = mul_bf16x2(code_pair<1>(w1), s1);
  a1[0] = mul_bf16x2(code_pair<2>(w0), s0), a1[1] = mul_bf16x2(code_pair<2>(w1), s1);
  a1[2] = mul_bf16x2(code_pair<3>(w0), s0), a1[3] = mul_bf16x2(code_pair<3>(w1), s1);
}
// d += a b for a 16 x 16 and b 16 x 8 in BF16.
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Eight values of x as they are staged: the pairs (0, 4), (1, 5), (2, 6), (3, 7)
// that meet code_pair<0> to <3>, in BF16; binary32 in three parts that add up to it.
template <typename X>
struct Staged;
template <>
struct Staged<uint16_t> {
  static constexpr int kParts = 1;
  uint4 r;
  __device__ __forceinline__ void fetch(const uint16_t* p, int64_t left, bool vec) {
    if (vec && left >= 8) {
      r = *reinterpret_cast<const uint4*>(p);
    } else {
      uint32_t u[4] = {};
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) u[i / 2] |= (uint32_t)p[i] << 16 * (i & 1);
      r = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
  __device__ __forceinline__ void clear() { r = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ uint4 part(int) const {
    return make_uint4(__byte_perm(r.x, r.z, 0x5410), __byte_perm(r.x, r.z, 0x7632), __byte_perm(r.y, r.w, 0x5410),
                      __byte_perm(r.y, r.w, 0x7632));
  }
};
template <>
struct Staged<float> {
  static constexpr int kParts = 3;
  float x[8];
  __device__ __forceinline__ void fetch(const float* p, int64_t left, bool vec) {
    if (vec && left >= 8) {
      const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = i < left ? p[i] : 0.0f;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.0f;
  }
  // Part 0: the upper 16 bits; 1 and 2: those of what is left, which ends there, exactly.  An infinity or a NaN has part 0 alone.
  static __device__ __forceinline__ uint32_t bits(float v, int part) {
    uint32_t u = __float_as_uint(v);
    if ((u & 0x7F800000u) == 0x7F800000u) return part ? 0u : (u & 0x007FFFFFu) ? 0x7FC00000u : u;
    for (int i = 0; i < part; ++i) u = __float_as_uint(__fsub_rn(__uint_as_float(u), __uint_as_float(u & 0xFFFF0000u)));
    return u & 0xFFFF0000u;
  }
  __device__ __forceinline__ uint4 part(int i) const {
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = bits(x[j], i) >> 16 | bits(x[j + 4], i);
    return make_uint4(o[0], o[1], o[2], o[3]);
  }
};

__device__ __forceinline__ float lds_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// What a block takes at once.
__host__ __device__ constexpr int fp4_panel(int rows) { return kWarps / rows * 2 * kChunk; }
template <typename X>
constexpr int fp4_smem(int tiles, int rows) {
  return std::max(2 * Staged<X>::kParts * 8 * tiles * (2 * fp4_panel(rows) + 64), (kWarps + rows) * 8 * tiles * 16 * 4);
}

// A block takes 16 ROWS rows of the weight and 8 TILES tokens; its warps are ROWS
// groups of 16 rows times kWarps / ROWS shares of k, chunks in turn, joined in
// order through shared memory at the end.  Where that makes too few blocks, a cluster of them takes a run of k's panels each, and
// their sums are joined in order through the cluster's shared memory.  Weights go
// from memory to registers, a panel of k ahead; x goes through shared memory, where
// a lane's 32 values of a chunk lie as four times 16 bytes, those of the four lanes
// of a row next to one another.  Within a chunk the order of k is the lanes': lane l
// of four takes values 32 l to 32 l + 31, four to each product of 16.
template <typename X, int TILES, int ROWS, int BLOCKS>
__global__ void __launch_bounds__(kFp4Threads, BLOCKS) fp4_kernel(const __grid_constant__ Fp4Args p) {
  constexpr int kShares = kWarps / ROWS, kParts = Staged<X>::kParts;
  constexpr int kOwn = 2;                             // chunks of a warp in a panel
  constexpr int kPanelChunks = kShares * kOwn, kPanel = kPanelChunks * kChunk;
  static_assert(kPanel == fp4_panel(ROWS), "a panel");
  constexpr int kTokens = 8 * TILES;
  constexpr int kStride = kPanel * 2 + 64;            // bytes of a token in a panel; the 64 keep neighbours off each other's banks
  constexpr int kPartBytes = kTokens * kStride, kBufferBytes = kParts * kPartBytes;
  constexpr int kPieces = kTokens * kPanel / 8 / kFp4Threads;  // of 8 values, a thread's share of a panel
  static_assert(kTokens * kPanel % (8 * kFp4Threads) == 0, "whole shares");
  extern __shared__ uint4 smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>(smem_raw);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, l = lane & 3;
  const int group = warp / kShares, share = warp % kShares;
  const int rank = (int)(blockIdx.x % p.split);
  const int64_t block_row = (int64_t)(blockIdx.x / p.split) * (16 * ROWS), row0 = block_row + group * 16;
  const int64_t token0 = (int64_t)blockIdx.y * kTokens;
  const int tokens = (int)(p.tokens - token0 < kTokens ? p.tokens - token0 : kTokens);
  const int64_t rows[2] = {min(row0 + g, p.rows - 1), min(row0 + g + 8, p.rows - 1)};
  wait_for_earlier_kernels();
  let_later_kernels_begin();

  struct Codes {
    uint4 q[2];
    uint16_t s[2];
  };
  Codes next[kOwn];
  Staged<X> x[kPieces];
  auto fetch = [&](int64_t panel) {
#pragma unroll
    for (int c = 0; c < kOwn; ++c) {
      const int64_t k = panel * kPanel + (c * kShares + share) * kChunk + l * 32;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t at = rows[h] * p.cols + k;
        next[c].q[h] = k < p.cols ? __ldcs(reinterpret_cast<const uint4*>(p.codes + at / 2)) : make_uint4(0, 0, 0, 0);
        next[c].s[h] = k < p.cols ? __ldcs(reinterpret_cast<const uint16_t*>(p.scales + at / 16)) : (uint16_t)0;
      }
    }
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int piece = i * kFp4Threads + threadIdx.x, token = piece / (kPanel / 8);
      const int64_t k = panel * kPanel + (int64_t)(piece % (kPanel / 8)) * 8;
      if (token < tokens && k < p.cols)
        x[i].fetch(static_cast<const X*>(p.x) + (token0 + token) * p.ldx + k, p.cols - k, p.vec_x);
      else
        x[i].clear();
    }
  };
  float acc[TILES][4] = {};
  const int64_t panels = (p.cols + kPanel - 1) / kPanel, first = panels * rank / p.split, last = panels * (rank + 1) / p.split;
  fetch(first);
  for (int64_t panel = first; panel < last; ++panel) {
    uint8_t* buffer = smem + (panel - first & 1) * kBufferBytes;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int piece = i * kFp4Threads + threadIdx.x, token = piece / (kPanel / 8), in = piece % (kPanel / 8);
      const int chunk = in / 16, owner = in / 4 % 4, quarter = in % 4;  // of 128, 32 and 8 values
      if (token >= tokens && panel - first >= 2) continue;  // zeros, which lie there already
      uint8_t* to = buffer + token * kStride + chunk * (2 * kChunk) + quarter * 64 + owner * 16;
#pragma unroll
      for (int part = 0; part < kParts; ++part) *reinterpret_cast<uint4*>(to + part * kPartBytes) = x[i].part(part);
    }
    Codes now[kOwn];
#pragma unroll
    for (int c = 0; c < kOwn; ++c) now[c] = next[c];
    __syncthreads();
    if (panel + 1 < last) fetch(panel + 1);
#pragma unroll
    for (int c = 0; c < kOwn; ++c) {
      const Scales scale[2] = {Scales(now[c].s[0], p.up), Scales(now[c].s[1], p.up)};
      const uint8_t* from = buffer + g * kStride + (c * kShares + share) * (2 * kChunk) + l * 16;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t a0[4], a1[4];
        weights(word_of(now[c].q[0], q), word_of(now[c].q[1], q), scale[0].s[q / 2], scale[1].s[q / 2], a0, a1);
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
#pragma unroll
          for (int part = kParts - 1; part >= 0; --part) {
            const uint4 b = *reinterpret_cast<const uint4*>(from + part * kPartBytes + t * 8 * kStride + q * 64);
            mma(acc[t], a0, b.x, b.y);
            mma(acc[t], a1, b.z, b.w);
          }
        }
      }
    }
  }
  // The shares of k, in order.  A lane's four sums are rows g, g and g + 8, g + 8 of tokens 2 l and 2 l + 1.
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);  // [warps][tokens][16]
#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      sums[(warp * kTokens + t * 8 + 2 * l + (i & 1)) * 16 + g + 8 * (i >> 1)] = acc[t][i];
  __syncthreads();
  auto shares_of = [&](int i) {
    const int token = i / (16 * ROWS), r = i % (16 * ROWS);
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < kShares; ++k) s = __fadd_rn(s, sums[((r / 16 * kShares + k) * kTokens + token) * 16 + r % 16]);
    return s;
  };
  auto finish = [&](int i, float s) {
    const int64_t row = block_row + i % (16 * ROWS);
    if (row < p.rows) put(static_cast<X*>(p.y), (token0 + i / (16 * ROWS)) * p.ldy + row, result_of(p, s));
  };
  const int results = tokens * 16 * ROWS;
  if (p.split == 1) {
    for (int i = threadIdx.x; i < results; i += kFp4Threads) finish(i, shares_of(i));
    return;
  }
  float* mine = sums + kWarps * kTokens * 16;
  for (int i = threadIdx.x; i < results; i += kFp4Threads) mine[i] = shares_of(i);
  cluster_sync();
  const uint32_t at = smem_addr(mine);
  for (int i = rank * kFp4Threads + threadIdx.x; i < results; i += p.split * kFp4Threads) {
    float s = 0.0f;
    for (int k = 0; k < p.split; ++k) s = __fadd_rn(s, lds_cluster_f32(peer_addr(at + 4 * i, k)));
    finish(i, s);
  }
  cluster_sync();  // nobody leaves while its sums are read
}

// At most 8 tokens in BF16: nothing is staged and no warp waits for another before
// the end.  A block takes 16 rows, its warps (and those of its cluster) chunks of k
// in turn, kFewAhead of them on their way; x comes straight from L1.  One token
// through 11008 x 4096 takes 14.3 us out of memory, 11.0 where the weight lies in L2.
// For a third of that no block has begun or all have ended; the rest is a wave of
// blocks whose warps wait for their first codes (31 % of their time), then share the
// issue slots (used in 58 % of the cycles) for the codes' expansion.
constexpr int kFewWarps = 4, kFewAhead = 4, kFewBlocks = 5;
__global__ void __launch_bounds__(32 * kFewWarps, kFewBlocks) fp4_few_kernel(const __grid_constant__ Fp4Args p) {
  constexpr int kTokens = 8;
  __shared__ float sums[kFewWarps][kTokens * 16], mine[kTokens * 16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, l = lane & 3;
  const int rank = (int)(blockIdx.x % p.split);
  const int64_t block_row = (int64_t)(blockIdx.x / p.split) * 16, token0 = (int64_t)blockIdx.y * kTokens;
  const int tokens = (int)min(p.tokens - token0, (int64_t)kTokens);
  const int64_t chunks = (p.cols + kChunk - 1) / kChunk, stride = p.split * kFewWarps;
  int64_t chunk = rank * kFewWarps + warp;
  const uint8_t *codes[2], *scales[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t row = min(block_row + g + 8 * h, p.rows - 1);
    codes[h] = p.codes + row * (p.cols / 2) + chunk * (kChunk / 2) + l * 16;
    scales[h] = p.scales + row * (p.cols / 16) + chunk * (kChunk / 16) + l * 2;
  }
  const uint16_t* x = static_cast<const uint16_t*>(p.x) + (token0 + g) * p.ldx + chunk * kChunk + l * 32;
  const bool here = g < tokens;
  wait_for_earlier_kernels();
  let_later_kernels_begin();

  uint4 q[kFewAhead][2];
  uint16_t s[kFewAhead][2];
  int64_t k = chunk * kChunk + l * 32;  // of the next fetch
  auto fetch = [&](int d) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      q[d][h] = k < p.cols ? __ldcs(reinterpret_cast<const uint4*>(codes[h])) : make_uint4(0, 0, 0, 0);
      s[d][h] = k < p.cols ? __ldcs(reinterpret_cast<const uint16_t*>(scales[h])) : (uint16_t)0;
      codes[h] += stride * (kChunk / 2);
      scales[h] += stride * (kChunk / 16);
    }
    k += stride * kChunk;
  };
#pragma unroll
  for (int d = 0; d < kFewAhead; ++d) fetch(d);
  float acc[4] = {};
  while (chunk < chunks) {
#pragma unroll
    for (int d = 0; d < kFewAhead; ++d) {
      if (chunk >= chunks) break;
      uint4 b[4];
      if (here && chunk * kChunk + l * 32 < p.cols) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          Staged<uint16_t> v;
          v.fetch(x + 8 * i, 8, p.vec_x);
          b[i] = v.part(0);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = make_uint4(0, 0, 0, 0);
      }
      const Scales scale[2] = {Scales(s[d][0], p.up), Scales(s[d][1], p.up)};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t a0[4], a1[4];
        weights(word_of(q[d][0], i), word_of(q[d][1], i), scale[0].s[i / 2], scale[1].s[i / 2], a0, a1);
        mma(acc, a0, b[i].x, b[i].y);
        mma(acc, a1, b[i].z, b[i].w);
      }
      fetch(d);
      chunk += stride;
      x += stride * kChunk;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) sums[warp][(2 * l + (i & 1)) * 16 + g + 8 * (i >> 1)] = acc[i];
  __syncthreads();
  const int i = threadIdx.x;  // a result a thread
  static_assert(kTokens * 16 == 32 * kFewWarps, "a result a thread");
  float sum = 0.0f;
#pragma unroll
  for (int w = 0; w < kFewWarps; ++w) sum = __fadd_rn(sum, sums[w][i]);
  bool out = i < tokens * 16 && block_row + i % 16 < p.rows;
  if (p.split > 1) {
    mine[i] = sum;
    cluster_sync();
    out = out && i % p.split == rank;
    if (out) {
      const uint32_t at = smem_addr(&mine[i]);
      sum = 0.0f;
      for (int r = 0; r < p.split; ++r) sum = __fadd_rn(sum, lds_cluster_f32(peer_addr(at, r)));
    }
    cluster_sync();  // nobody leaves while its sums are read
  }
  if (out)
    put(static_cast<uint16_t*>(p.y), (token0 + i / 16) * p.ldy + block_row + i % 16, result_of(p, sum));
}

// Any number of columns and any alignment: a warp takes a row and four tokens.
constexpr int kAnyTokens = 4;
template <typename X>
__global__ void __launch_bounds__(kFp4Threads) fp4_any_kernel(const __grid_constant__ Fp4Args p) {
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5), token0 = (int64_t)blockIdx.y * kAnyTokens;
  wait_for_earlier_kernels();
  let_later_kernels_begin();
  if (row >= p.rows) return;
  const X* x = static_cast<const X*>(p.x);
  float acc[kAnyTokens] = {};
  for (int64_t k = lane; k < p.cols; k += 32) {
    const int64_t at = row * p.cols + k;
    const uint32_t code = p.codes[at >> 1] >> 4 * (at & 1) & 15u;
    const float q = __uint_as_float((code & 8u) << 28 | (code & 7u) << 22);  // times 2^-126
    const float w = __fmul_rn(q, __fmul_rn(scale_values(p.scales[at >> 4]).x, p.up));
#pragma unroll
    for (int t = 0; t < kAnyTokens; ++t)
      if (token0 + t < p.tokens) acc[t] = __fmaf_rn(get(x, (token0 + t) * p.ldx + k), w, acc[t]);
  }
#pragma unroll
  for (int t = 0; t < kAnyTokens; ++t) {
#pragma unroll
    for (int d = 16; d; d >>= 1) acc[t] = __fadd_rn(acc[t], __shfl_xor_sync(~0u, acc[t], d));
    if (lane == 0 && token0 + t < p.tokens)
      put(static_cast<X*>(p.y), (token0 + t) * p.ldy + row, result_of(p, acc[t]));
  }
}

template <typename X, int TILES, int ROWS, int BLOCKS>
cudaError_t launch(Fp4Args a, cudaStream_t stream) {
  constexpr int kSmem = fp4_smem<X>(TILES, ROWS), kTokens = 8 * TILES;
  const void* kernel = (const void*)fp4_kernel<X, TILES, ROWS, BLOCKS>;
  if (kSmem > 48 * 1024) {
    static std::atomic<uint64_t> ready{0};
    const cudaError_t e = allow_smem(kernel, kSmem, ready);
    if (e != cudaSuccess) return e;
  }
  const int64_t blocks = (a.rows + 16 * ROWS - 1) / (16 * ROWS), tiles = (a.tokens + kTokens - 1) / kTokens;
  const int64_t panels = (a.cols + fp4_panel(ROWS) - 1) / fp4_panel(ROWS);
  a.split = 1;
  while (a.split < 8 && 2 * a.split <= panels && 2 * blocks * tiles * a.split <= BLOCKS * kSms) a.split *= 2;
  return launch_dependent(kernel, dim3((unsigned)(blocks * a.split), (unsigned)tiles), kFp4Threads, a.split > 1 ? a.split : 0, kSmem, &a,
                          stream);
}

cudaError_t launch_few(Fp4Args a, cudaStream_t stream) {
  const int64_t blocks = (a.rows + 15) / 16, chunks = (a.cols + kChunk - 1) / kChunk;
  a.split = 1;
  while (a.split < 8 && 2 * a.split * kFewWarps <= chunks && 2 * blocks * a.split <= kFewBlocks * kSms) a.split *= 2;
  return launch_dependent((const void*)fp4_few_kernel, (unsigned)(blocks * a.split), 32 * kFewWarps, a.split > 1 ? a.split : 0, 0, &a, stream);
}

}  // namespace

cudaError_t launch_fp4_linear(const Fp4Args& args, cudaStream_t stream) {
  Fp4Args a = args;
  // e in [-44, -8]: up times the largest scale, 448, stays in range; with e = -44 no sum leaves it (weights are below 2^12, x
  // below 2^128, k below 2^31).  G above 2^-8 makes results larger than their sums, so those need no more room.  The factors: 1
  // and G / 2^e, or, where that might be out of range, 2^-e and G.
  int e = 0;
  std::frexp(a.global_scale, &e);
  e = std::min(std::max(e - 1, -44), -8);
  a.up = std::ldexp(1.0f, 126 + e);
  a.out0 = a.global_scale < 1.0f ? 1.0f : std::ldexp(1.0f, -e);
  a.out1 = a.global_scale < 1.0f ? std::ldexp(a.global_scale, -e) : a.global_scale;
  const int64_t xs = a.x_f32 ? 4 : 2;
  a.vec_x = reinterpret_cast<uintptr_t>(a.x) % 16 == 0 && (a.tokens == 1 || a.ldx * xs % 16 == 0);
  // Rows of codes and scales start on 16- and 2-byte boundaries, and whole groups make up a row.
  const bool packed = a.cols % 32 == 0 && reinterpret_cast<uintptr_t>(a.codes) % 16 == 0 && reinterpret_cast<uintptr_t>(a.scales) % 2 == 0;
  if (!packed) {
    const dim3 grid((unsigned)((a.rows + kWarps - 1) / kWarps), (unsigned)((a.tokens + kAnyTokens - 1) / kAnyTokens));
    return a.x_f32 ? launch_dependent((const void*)fp4_any_kernel<float>, grid, kFp4Threads, 0, 0, &a, stream)
                   : launch_dependent((const void*)fp4_any_kernel<uint16_t>, grid, kFp4Threads, 0, 0, &a, stream);
  }
  if (a.x_f32) return launch<float, 1, 2, 2>(a, stream);
  if (a.tokens <= 8) return launch_few(a, stream);
  if (a.tokens <= 16) return launch<uint16_t, 2, 4, 2>(a, stream);
  if (a.tokens <= 24) return launch<uint16_t, 3, 4, 2>(a, stream);
  return launch<uint16_t, 4, 4, 2>(a, stream);
}

}  // namespace mpadam
