// layer_norm.cu -- layer normalisation of rows, forward and backward:
//   n = (x - mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps),  y = n w + b
//   dn = dy w,  dx = (dn - mean(dn) - n mean(dn n)) rstd
//   dw = sum over rows of dy n,  db = sum over rows of dy
// Everything is in binary32 from the load to the store.  The variance is taken
// around a first mean, whose own roundings are taken off the deviations again
// (Moments below): a mean far from 0 costs the forward pass no bits, and the
// backward pass the rounding of the mean that it is given.
#include <algorithm>

#include "launch.h"
#include "layer_norm.h"
#include "step_kernel.cuh"

namespace mpadam {

namespace {

constexpr int kSms = 152;        // GB300
constexpr int kRowWarps = 8;     // rows of a block where a row is one warp's
constexpr int kMaxThreads = 512; // of a row that a block shares
constexpr int kWideThreads = 512;

__device__ __forceinline__ void wait_for_earlier_kernels() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_later_kernels_begin() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ float get(const float* p, int64_t i) { return p[i]; }
__device__ __forceinline__ float get(const uint16_t* p, int64_t i) { return __uint_as_float((uint32_t)p[i] << 16); }
__device__ __forceinline__ void put(float* p, int64_t i, float x) { p[i] = x; }
__device__ __forceinline__ void put(uint16_t* p, int64_t i, float x) { p[i] = (uint16_t)bf16x2_rn(x, 0.0f); }

// 16 bytes of values, as they lie.
template <typename T>
struct Pack;
template <>
struct Pack<float> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void open(const uint4& r, float* x) {
    x[0] = __uint_as_float(r.x), x[1] = __uint_as_float(r.y), x[2] = __uint_as_float(r.z), x[3] = __uint_as_float(r.w);
  }
  static __device__ __forceinline__ uint4 close(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <>
struct Pack<uint16_t> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void open(const uint4& r, float* x) {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
  }
  static __device__ __forceinline__ uint4 close(const float* x) {
    return make_uint4(bf16x2_rn(x[0], x[1]), bf16x2_rn(x[2], x[3]), bf16x2_rn(x[4], x[5]), bf16x2_rn(x[6], x[7]));
  }
};

// A thread's E values of a row of T values, shared out among `threads`: VEC:
// packs of 16 bytes, the threads' packs next to one another; else single
// values.  raw[] holds them as they lie, so that a row fetched ahead takes few registers.
template <typename T, bool VEC, int E>
struct Slice {
  static constexpr int kN = VEC ? Pack<T>::kN : 1, kSlots = E / kN, kWords = VEC ? 4 * kSlots : kSlots;
  static_assert(E % kN == 0, "whole packs");
  static __device__ __forceinline__ int64_t at(int slot, int t, int threads) { return (int64_t)(slot * threads + t) * kN; }
  static __device__ __forceinline__ void fetch(const T* p, int64_t cols, int t, int threads, uint32_t* raw) {
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const int64_t c = at(s, t, threads);
      if constexpr (VEC) {
        const uint4 v = c < cols ? *reinterpret_cast<const uint4*>(p + c) : make_uint4(0, 0, 0, 0);
        raw[4 * s] = v.x, raw[4 * s + 1] = v.y, raw[4 * s + 2] = v.z, raw[4 * s + 3] = v.w;
      } else {
        raw[s] = c < cols ? __float_as_uint(get(p, c)) : 0u;
      }
    }
  }
  // The same by way of shared memory, where a thread's pieces are its own: it alone waits for them, and reads them.
  // (A single BF16 is too small for an asynchronous copy.)
  static constexpr bool kAsync = VEC || sizeof(T) == 4;
  static constexpr int kPiece = VEC ? 16 : 4;
  static __host__ __device__ constexpr int bytes(int threads) { return kSlots * threads * kPiece; }
  static __device__ __forceinline__ void begin(const T* p, int64_t cols, int t, int threads, uint32_t to) {
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const int64_t c = at(s, t, threads);
      const int size = c < cols ? kPiece : 0;  // nothing read: zeros
      const T* from = c < cols ? p + c : p;
      if constexpr (VEC)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + (s * threads + t) * kPiece), "l"(from), "r"(size) : "memory");
      else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + (s * threads + t) * kPiece), "l"(from), "r"(size) : "memory");
    }
  }
  static __device__ __forceinline__ void read(uint32_t from, int t, int threads, float* x) {
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const uint32_t at = from + (s * threads + t) * kPiece;
      if constexpr (VEC) {
        uint4 v;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
        Pack<T>::open(v, x + s * kN);
      } else {
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x[s]) : "r"(at) : "memory");
      }
    }
  }
  static __device__ __forceinline__ void open(const uint32_t* raw, float* x) {
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      if constexpr (VEC) Pack<T>::open(make_uint4(raw[4 * s], raw[4 * s + 1], raw[4 * s + 2], raw[4 * s + 3]), x + s * kN);
      else x[s] = __uint_as_float(raw[s]);
    }
  }
  static __device__ __forceinline__ void store(T* p, int64_t cols, int t, int threads, const float* x) {
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const int64_t c = at(s, t, threads);
      if (c >= cols) continue;
      if constexpr (VEC) *reinterpret_cast<uint4*>(p + c) = Pack<T>::close(x + s * kN);
      else put(p, c, x[0 + s]);
    }
  }
  // The same columns of a vector of another type (`absent` where there is none): those of slots [FIRST, FIRST + SLOTS).
  template <int FIRST = 0, int SLOTS = kSlots, typename W>
  static __device__ __forceinline__ void vector(const W* p, float absent, int64_t cols, int t, int threads, float* x) {
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int64_t c = at(FIRST + s, t, threads);
      if constexpr (VEC) {
        if (p && c < cols) {
#pragma unroll
          for (int h = 0; h < kN; h += Pack<W>::kN) {
            float v[Pack<W>::kN];
            Pack<W>::open(*reinterpret_cast<const uint4*>(p + c + h), v);
#pragma unroll
            for (int i = 0; i < Pack<W>::kN && h + i < kN; ++i) x[s * kN + h + i] = v[i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < kN; ++i) x[s * kN + i] = absent;
        }
      } else {
        x[s] = p && c < cols ? get(p, c) : absent;
      }
    }
  }
};

__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_for_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Rows on their way at once, of those that a warp or block takes in turn: so many that an SM waits for 64 KB or more, whatever
// the width; one row ahead in registers left 16384 x 4096 in BF16 at 4 TB/s.
template <typename X, int E>
constexpr int kAhead = sizeof(X) == 2 ? (E == 32 ? 3 : 4) : (E == 8 ? 4 : E == 16 ? 3 : 2);

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int d = 16; d; d >>= 1) x = __fadd_rn(x, __shfl_xor_sync(~0u, x, d));
  return x;
}

// Sums over a block's warps, of one value or two, the same in every thread;
// `slots` (2 x 32 of each) alternate between calls, so that one barrier a call is
// enough: a warp that is two calls ahead would have passed the barrier between them.
struct alignas(16) SumSlots {
  float x[32], y[32];
};
struct BlockSum {
  SumSlots* slots;  // [2]
  int turn = 0;
  __device__ __forceinline__ float operator()(float x) {
    x = warp_sum(x);
    float* s = slots[turn].x;
    turn ^= 1;
    const int warps = blockDim.x / 32;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    float sum = 0.0f;
    for (int i = 0; i < warps; ++i) sum = __fadd_rn(sum, s[i]);
    return sum;
  }
  __device__ __forceinline__ float2 operator()(float x, float y) {
    x = warp_sum(x), y = warp_sum(y);
    SumSlots& s = slots[turn];
    turn ^= 1;
    const int warps = blockDim.x / 32;
    if ((threadIdx.x & 31) == 0) s.x[threadIdx.x >> 5] = x, s.y[threadIdx.x >> 5] = y;
    __syncthreads();
    float2 sum = make_float2(0.0f, 0.0f);
    for (int i = 0; i < warps; i += 4) {
      const float4 a = *reinterpret_cast<const float4*>(s.x + i), b = *reinterpret_cast<const float4*>(s.y + i);
      sum.x = __fadd_rn(sum.x, a.x), sum.y = __fadd_rn(sum.y, b.x);
      if (i + 1 < warps) sum.x = __fadd_rn(sum.x, a.y), sum.y = __fadd_rn(sum.y, b.y);
      if (i + 2 < warps) sum.x = __fadd_rn(sum.x, a.z), sum.y = __fadd_rn(sum.y, b.z);
      if (i + 3 < warps) sum.x = __fadd_rn(sum.x, a.w), sum.y = __fadd_rn(sum.y, b.w);
    }
    return sum;
  }
};
struct WarpSum {
  __device__ __forceinline__ float operator()(float x) { return warp_sum(x); }
  __device__ __forceinline__ float2 operator()(float x, float y) { return make_float2(warp_sum(x), warp_sum(y)); }
};
// The sums of a row that is one warp's, or a block's.
template <bool ONE>
__device__ __forceinline__ auto row_sum(SumSlots* slots) {
  if constexpr (ONE) return WarpSum{};
  else return BlockSum{slots};
}

// A row's mean and 1 / sigma by its sum, by those of its deviations d from a first mean and of their squares.  The first mean is
// off by some roundings of its size, and the deviations may be as small: `rest` is what it lacks, shift makes n = d / sigma +
// shift, and the mean square has the square of the rest too much.  Binary32 values' own sum is off, and the deviations' mean is
// the rest (4096 x 8192 45 us for 43 without).  A sum of BF16 values of one size is exact up to 2^15 of them, and values of
// several sizes lie far apart: what the division left is the rest, without another sum over the row (48 us instead of 50 for
// 16384 x 4096).
template <typename X>
struct Moments {
  static constexpr bool kExactSum = sizeof(X) == 2;
  float first, rest, mean, rstd, shift;
  __device__ __forceinline__ Moments(float sum, const NormForwardArgs& p) {
    first = __fmul_rn(sum, p.inv_cols);
    rest = kExactSum ? __fmul_rn(__fmaf_rn(-first, p.all_cols, sum), p.inv_cols) : 0.0f;
  }
  // One deviation, added to a thread's sums.
  static __device__ __forceinline__ void add(float d, float& r, float& s) {
    if (!kExactSum) r = __fadd_rn(r, d);
    s = __fmaf_rn(d, d, s);
  }
  template <typename Sum>
  __device__ __forceinline__ void finish(float r, float s, Sum& sum, const NormForwardArgs& p) {
    if (kExactSum) {
      s = sum(s);
    } else {
      const float2 sums = sum(r, s);
      rest = __fmul_rn(sums.x, p.inv_cols), s = sums.y;
    }
    mean = __fadd_rn(first, rest);
    const float var = __fmaf_rn(-rest, rest, __fmul_rn(s, p.inv_cols));
    rstd = 1.0f / sqrtf(__fadd_rn(var < 0.0f ? 0.0f : var, p.eps));  // (a NaN stays one)
    shift = -__fmul_rn(rest, rstd);
  }
  __device__ __forceinline__ float normal(float d) const { return __fmaf_rn(d, rstd, shift); }
};

// ---------------------------------------------------------------------------
// Forward: a row in the registers of a warp (ONE) or of a block.
// ---------------------------------------------------------------------------
// y of what is left of a row from slot FIRST on: weight and bias a pack at a time, which spares the registers of wide rows (32768
// x 1024 in BF16 30.0 us, 33.1 with all of them at once), but all at once where those have room (32768 x 768 22.7, 24.5) or they
// come one by one.
template <typename X, typename W, bool VEC, int E, int FIRST>
__device__ __forceinline__ void scale_row(const NormForwardArgs& p, int t, int threads, float (&x)[E], const Moments<X>& m) {
  using S = Slice<X, VEC, E>;
  constexpr int kSlots = VEC && E != 24 ? 1 : S::kSlots, kPart = kSlots * S::kN;
  float w[kPart], b[kPart];
  S::template vector<FIRST, kSlots>(static_cast<const W*>(p.w), 1.0f, p.cols, t, threads, w);
  S::template vector<FIRST, kSlots>(static_cast<const W*>(p.b), 0.0f, p.cols, t, threads, b);
#pragma unroll
  for (int i = 0; i < kPart; ++i) x[FIRST * S::kN + i] = __fmaf_rn(m.normal(x[FIRST * S::kN + i]), w[i], b[i]);
  if constexpr (FIRST + kSlots < S::kSlots) scale_row<X, W, VEC, E, FIRST + kSlots>(p, t, threads, x, m);
}

template <typename X, typename W, bool VEC, int E, typename Sum>
__device__ __forceinline__ void forward_row(const NormForwardArgs& p, int64_t row, int t, int threads, float (&x)[E], Sum& sum,
                                            const float* held_w = nullptr, const float* held_b = nullptr) {
  using S = Slice<X, VEC, E>;
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < E; ++i) s = __fadd_rn(s, x[i]);
  Moments<X> m(sum(s), p);
  float r = s = 0.0f;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    x[i] = __fsub_rn(x[i], m.first);
    if (S::at(i / S::kN, t, threads) < p.cols) m.add(x[i], r, s);
  }
  m.finish(r, s, sum, p);
  if (t == 0 && p.mean) p.mean[row] = m.mean, p.rstd[row] = m.rstd;
  if (held_w) {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = m.normal(x[i]);
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = __fmaf_rn(x[i], held_w[i], held_b[i]);
  } else {
    scale_row<X, W, VEC, E, 0>(p, t, threads, x, m);
  }
  S::store(static_cast<X*>(p.y) + row * p.ldy, p.cols, t, threads, x);
}

template <typename X, typename W, bool VEC, int E, bool ONE>
__global__ void __launch_bounds__(ONE ? 32 * kRowWarps : kMaxThreads) forward_kernel(const __grid_constant__ NormForwardArgs p) {
  using S = Slice<X, VEC, E>;
  __shared__ SumSlots slots[2];
  wait_for_earlier_kernels();
  let_later_kernels_begin();
  const int t = ONE ? threadIdx.x & 31 : threadIdx.x, threads = ONE ? 32 : blockDim.x;
  const int64_t row = ONE ? (int64_t)blockIdx.x * (blockDim.x / 32) + (threadIdx.x >> 5) : blockIdx.x;
  if (row >= p.rows) return;
  auto sum = row_sum<ONE>(slots);
  uint32_t raw[S::kWords];
  float x[E];
  S::fetch(static_cast<const X*>(p.x) + row * p.ldx, p.cols, t, threads, raw);
  S::open(raw, x);
  forward_row<X, W, VEC, E>(p, row, t, threads, x, sum);
}

// Blocks an SM, of eight rows each; with more, registers would not do.  A block of a row of its own holds weight and bias,
// and has 32 values a thread in BF16 (152 registers), 16 in binary32 (104, without packs 120): as many rows at a time on an
// SM as have room, since each waits for two sums over its threads.  16384 x 4096 in BF16 takes 48 us so (5.6 TB/s), with 16
// values 57, without weight and bias held 68.
constexpr int kRegisters = 65536;
constexpr int forward_blocks(int each) { return each == 32 ? 3 : 4; }

// Many rows: each warp or block takes rows in turn, kAhead of them on their way.
template <typename X, typename W, bool VEC, int E, bool ONE>
__global__ void __launch_bounds__(ONE || E == 32 ? 256 : kMaxThreads, ONE ? forward_blocks(E) : 1)
    forward_rows_kernel(const __grid_constant__ NormForwardArgs p) {
  using S = Slice<X, VEC, E>;
  constexpr int kDeep = kAhead<X, E>;
  extern __shared__ uint4 ring[];
  __shared__ SumSlots slots[2];
  wait_for_earlier_kernels();
  let_later_kernels_begin();
  const int t = ONE ? threadIdx.x & 31 : threadIdx.x, threads = ONE ? 32 : blockDim.x, warps = blockDim.x / 32;
  const int64_t stride = ONE ? (int64_t)gridDim.x * warps : gridDim.x;
  int64_t row = ONE ? (int64_t)blockIdx.x * warps + (threadIdx.x >> 5) : blockIdx.x, next = row;
  const int stage = S::bytes(threads);
  const uint32_t mine = smem_addr(ring) + (ONE ? (threadIdx.x >> 5) * kDeep * stage : 0);
  auto sum = row_sum<ONE>(slots);
  auto begin = [&](int at) {
    if (next < p.rows) S::begin(static_cast<const X*>(p.x) + next * p.ldx, p.cols, t, threads, mine + at * stage);
    commit_copies();
    next += stride;
  };
#pragma unroll
  for (int i = 0; i < kDeep - 1; ++i) begin(i);
  float w[E], b[E];
  if (!ONE) {
    S::vector(static_cast<const W*>(p.w), 1.0f, p.cols, t, threads, w);
    S::vector(static_cast<const W*>(p.b), 0.0f, p.cols, t, threads, b);
  }
  int at = 0;
  for (; row < p.rows; row += stride) {
    begin(at ? at - 1 : kDeep - 1);
    wait_for_copies<kDeep - 1>();
    float x[E];
    S::read(mine + at * stage, t, threads, x);
    forward_row<X, W, VEC, E>(p, row, t, threads, x, sum, ONE ? nullptr : w, ONE ? nullptr : b);
    if (++at == kDeep) at = 0;
  }
}

// Rows of any width, read three times.
template <typename X, typename W>
__global__ void __launch_bounds__(kWideThreads) forward_wide_kernel(const __grid_constant__ NormForwardArgs p) {
  __shared__ SumSlots slots[2];
  wait_for_earlier_kernels();
  let_later_kernels_begin();
  BlockSum sum{slots};
  const X* x = static_cast<const X*>(p.x) + blockIdx.x * p.ldx;
  X* y = static_cast<X*>(p.y) + blockIdx.x * p.ldy;
  const W *w = static_cast<const W*>(p.w), *b = static_cast<const W*>(p.b);
  float s = 0.0f;
  for (int64_t c = threadIdx.x; c < p.cols; c += kWideThreads) s = __fadd_rn(s, get(x, c));
  Moments<X> m(sum(s), p);
  float r = s = 0.0f;
  for (int64_t c = threadIdx.x; c < p.cols; c += kWideThreads) m.add(__fsub_rn(get(x, c), m.first), r, s);
  m.finish(r, s, sum, p);
  if (threadIdx.x == 0 && p.mean) p.mean[blockIdx.x] = m.mean, p.rstd[blockIdx.x] = m.rstd;
  for (int64_t c = threadIdx.x; c < p.cols; c += kWideThreads)
    put(y, c, __fmaf_rn(m.normal(__fsub_rn(get(x, c), m.first)), w ? get(w, c) : 1.0f, b ? get(b, c) : 0.0f));
}

// ---------------------------------------------------------------------------
// Backward: a row in the registers of a warp (ONE) or of a block, rows in turn;
// each thread keeps the sums over its rows of dy n and dy for its columns.
// kAhead rows are on their way by asynchronous copies, or one in registers.
// 16384 x 4096 in BF16 takes 79 us (5.1 TB/s), 8192 x 4096 in binary32 66 (6.1):
// registers have room for two rows at a time on an SM, which do not cover the
// exchange of a BF16 row's sums.  32 values a thread took 80, and a third row whose
// values were read a second time instead of held 100.
// ---------------------------------------------------------------------------
template <typename X, typename W, bool VEC, int E, bool ONE>
__global__ void __launch_bounds__(E == 16 ? kMaxThreads : 256, ONE ? 2 : E == 8 ? 3 : 1)
    backward_kernel(const __grid_constant__ NormBackwardArgs p) {
  using S = Slice<X, VEC, E>;
  constexpr int kDeep = S::kAsync ? kAhead<X, E> : 1;
  extern __shared__ uint4 dynamic[];  // the rows on their way, then, ONE: [2][cols] sums
  __shared__ float2 slots[2][32];
  wait_for_earlier_kernels();
  let_later_kernels_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x / 32;
  const int t = ONE ? lane : threadIdx.x, threads = ONE ? 32 : blockDim.x;
  const int64_t stride = ONE ? (int64_t)gridDim.x * warps : gridDim.x;
  int64_t row = ONE ? (int64_t)blockIdx.x * warps + warp : blockIdx.x, next = row;
  const X *x = static_cast<const X*>(p.x), *dy = static_cast<const X*>(p.dy);
  const int stage = S::kAsync ? 2 * S::bytes(threads) : 0;
  const uint32_t mine = smem_addr(dynamic) + (ONE ? warp * kDeep * stage : 0);
  float* joined = reinterpret_cast<float*>(dynamic) + (ONE ? warps : 1) * kDeep * stage / 4;
  float w[E], dw[E], db[E];
  S::vector(static_cast<const W*>(p.w), 1.0f, p.cols, t, threads, w);
#pragma unroll
  for (int i = 0; i < E; ++i) dw[i] = db[i] = 0.0f;
  uint32_t raw_x[S::kAsync ? 1 : S::kWords], raw_dy[S::kAsync ? 1 : S::kWords];
  float mean = 0.0f, rstd = 0.0f;  // of the next row
  auto begin = [&](int at) {
    if (next < p.rows) {
      if constexpr (S::kAsync) {
        S::begin(x + next * p.ldx, p.cols, t, threads, mine + at * stage);
        S::begin(dy + next * p.lddy, p.cols, t, threads, mine + at * stage + stage / 2);
      } else {
        S::fetch(x + next * p.ldx, p.cols, t, threads, raw_x);
        S::fetch(dy + next * p.lddy, p.cols, t, threads, raw_dy);
      }
    }
    if constexpr (S::kAsync) commit_copies();
    next += stride;
  };
#pragma unroll
  for (int i = 0; i < kDeep; ++i) begin(i);
  if (row < p.rows) mean = p.mean[row], rstd = p.rstd[row];
  int turn = 0, at = 0;
  for (; row < p.rows; row += stride) {
    float n[E], dn[E];
    if constexpr (S::kAsync) {
      wait_for_copies<kDeep - 1>();
      S::read(mine + at * stage, t, threads, n);
      S::read(mine + at * stage + stage / 2, t, threads, dn);
    } else {
      S::open(raw_x, n);
      S::open(raw_dy, dn);
    }
    const float scale = rstd;
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      // (columns past the last have dy = 0, and n = 0 whatever the mean: they add nothing)
      n[i] = S::at(i / S::kN, t, threads) < p.cols ? __fmul_rn(__fsub_rn(n[i], mean), scale) : 0.0f;
      dw[i] = __fmaf_rn(dn[i], n[i], dw[i]);
      db[i] = __fadd_rn(db[i], dn[i]);
      dn[i] = __fmul_rn(dn[i], w[i]);
      s0 = __fadd_rn(s0, dn[i]);
      s1 = __fmaf_rn(dn[i], n[i], s1);
    }
    begin(at);
    if (++at == kDeep) at = 0;
    if (row + stride < p.rows) mean = p.mean[row + stride], rstd = p.rstd[row + stride];
    if (!p.dx) continue;
    s0 = warp_sum(s0), s1 = warp_sum(s1);
    if (!ONE) {
      if (lane == 0) slots[turn][warp] = make_float2(s0, s1);
      __syncthreads();
      s0 = s1 = 0.0f;
      for (int i = 0; i < warps; ++i) s0 = __fadd_rn(s0, slots[turn][i].x), s1 = __fadd_rn(s1, slots[turn][i].y);
      turn ^= 1;
    }
    s0 = __fmul_rn(s0, p.inv_cols), s1 = __fmul_rn(s1, p.inv_cols);
#pragma unroll
    for (int i = 0; i < E; ++i) dn[i] = __fmul_rn(__fsub_rn(__fsub_rn(dn[i], s0), __fmul_rn(n[i], s1)), scale);
    S::store(static_cast<X*>(p.dx) + row * p.lddx, p.cols, t, threads, dn);
  }
  if (!p.partial) return;
  if (ONE) {  // the warps' sums one after another
    for (int k = 0; k < warps; ++k) {
      if (warp == k) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const int64_t c = S::at(i / S::kN, t, threads) + i % S::kN;
          if (c >= p.cols) continue;
          joined[c] = k ? __fadd_rn(joined[c], dw[i]) : dw[i];
          joined[p.cols + c] = k ? __fadd_rn(joined[p.cols + c], db[i]) : db[i];
        }
      }
      __syncthreads();
    }
    for (int64_t c = threadIdx.x; c < 2 * p.cols; c += blockDim.x) p.partial[blockIdx.x * 2 * p.cols + c] = joined[c];
  } else {
    float* out = p.partial + blockIdx.x * 2 * p.cols;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int64_t c = S::at(i / S::kN, t, threads) + i % S::kN;
      if (c < p.cols) out[c] = dw[i], out[p.cols + c] = db[i];
    }
  }
}

// Rows of any width: dx, read twice.
template <typename X, typename W>
__global__ void __launch_bounds__(kWideThreads) backward_wide_kernel(const __grid_constant__ NormBackwardArgs p) {
  __shared__ SumSlots slots[2];
  wait_for_earlier_kernels();
  let_later_kernels_begin();
  BlockSum sum{slots};
  const int64_t row = blockIdx.x;
  const X *x = static_cast<const X*>(p.x) + row * p.ldx, *dy = static_cast<const X*>(p.dy) + row * p.lddy;
  X* dx = static_cast<X*>(p.dx) + row * p.lddx;
  const W* w = static_cast<const W*>(p.w);
  const float mean = p.mean[row], rstd = p.rstd[row];
  float s0 = 0.0f, s1 = 0.0f;
  for (int64_t c = threadIdx.x; c < p.cols; c += kWideThreads) {
    const float n = __fmul_rn(__fsub_rn(get(x, c), mean), rstd), dn = __fmul_rn(get(dy, c), w ? get(w, c) : 1.0f);
    s0 = __fadd_rn(s0, dn);
    s1 = __fmaf_rn(dn, n, s1);
  }
  const float2 s = sum(s0, s1);
  s0 = __fmul_rn(s.x, p.inv_cols);
  s1 = __fmul_rn(s.y, p.inv_cols);
  for (int64_t c = threadIdx.x; c < p.cols; c += kWideThreads) {
    const float n = __fmul_rn(__fsub_rn(get(x, c), mean), rstd), dn = __fmul_rn(get(dy, c), w ? get(w, c) : 1.0f);
    put(dx, c, __fmul_rn(__fsub_rn(__fsub_rn(dn, s0), __fmul_rn(n, s1)), rstd));
  }
}

// ... and the sums over each part's rows, a column a thread.
template <typename X>
__global__ void __launch_bounds__(kWideThreads) wide_sums_kernel(const __grid_constant__ NormBackwardArgs p) {
  wait_for_earlier_kernels();
  let_later_kernels_begin();
  const X *x = static_cast<const X*>(p.x), *dy = static_cast<const X*>(p.dy);
  const int64_t tiles = (p.cols + kWideThreads - 1) / kWideThreads;
  const int64_t part = blockIdx.x / tiles, c = blockIdx.x % tiles * kWideThreads + threadIdx.x;
  if (c >= p.cols) return;
  float dw = 0.0f, db = 0.0f;
  for (int64_t r = part; r < p.rows; r += p.parts) {
    const float d = get(dy, r * p.lddy + c);
    dw = __fmaf_rn(d, __fmul_rn(__fsub_rn(get(x, r * p.ldx + c), p.mean[r]), p.rstd[r]), dw);
    db = __fadd_rn(db, d);
  }
  p.partial[part * 2 * p.cols + c] = dw;
  p.partial[part * 2 * p.cols + p.cols + c] = db;
}

// The parts' sums: 32 columns a block, 32 rows of threads that take every 32nd
// part each and are joined in order.
template <typename W>
__global__ void __launch_bounds__(1024) sums_kernel(const __grid_constant__ NormSumArgs p) {
  __shared__ float joined[32][33];
  wait_for_earlier_kernels();
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int64_t tiles = (p.cols + 31) / 32;
  const bool second = blockIdx.x >= tiles;
  const int64_t c = (blockIdx.x - (second ? tiles : 0)) * 32 + lane;
  void* out = second ? p.db : p.dw;
  if (!out) return;
  float s = 0.0f;
  if (c < p.cols) {
    const float* from = p.partial + (second ? p.cols : 0) + c;
#pragma unroll 8
    for (int i = group; i < p.parts; i += 32) s = __fadd_rn(s, from[(int64_t)i * 2 * p.cols]);
  }
  joined[group][lane] = s;
  __syncthreads();
  if (group || c >= p.cols) return;
  s = 0.0f;
#pragma unroll
  for (int i = 0; i < 32; ++i) s = __fadd_rn(s, joined[i][lane]);
  put(static_cast<W*>(out), c, s);
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------
constexpr int64_t kOneCols = 32 * 32;           // widest row of a warp
constexpr int64_t kWarpCols = 8 * 32;           // and in the backward pass, which has five arrays of a row
constexpr int64_t kSmallCols = 8 * 256;         // widest row of a block with 8 values a thread there
constexpr int64_t kBlockCols = 16 * kMaxThreads; // and of a block

bool whole_packs(const void* p, int64_t ld, int64_t rows, int64_t size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows == 1 || ld * size % 16 == 0);
}

constexpr int threads_for(int64_t cols, int each) { return (int)((cols + 32 * each - 1) / (32 * each)) * 32; }

// A launch of a kernel instance that needs `smem` bytes, and MOST for the widest row that it is taken for.  The limit belongs to
// the instance, whoever launches it from whatever thread: it is set once, to MOST.  `ready` is the instance's.
template <int MOST, typename Args>
cudaError_t launch_ring(void (*kernel)(Args), std::atomic<uint64_t>& ready, int64_t blocks, int threads, int smem, const Args& a,
                        cudaStream_t stream) {
  if (MOST > 40 * 1024) {  // (what is not asked for is 48 KB, the kernel's own arrays among it)
    const cudaError_t e = allow_smem((const void*)kernel, MOST, ready);
    if (e != cudaSuccess) return e;
  }
  return launch_dependent((const void*)kernel, (unsigned)blocks, threads, 0, smem, &a, stream);
}

// Shared memory of rows on their way, `threads` to a row (ONE: 32, and a block's rows together).
template <typename X, bool VEC, int E, bool ONE>
constexpr int forward_ring(int threads) {
  return (ONE ? kRowWarps : 1) * kAhead<X, E> * Slice<X, VEC, E>::bytes(threads);
}
// The same, and the sums of a row's columns where a row is one warp's.
template <typename X, bool VEC, int E, bool ONE>
constexpr int backward_ring(int threads, int64_t cols) {
  using S = Slice<X, VEC, E>;
  return (S::kAsync ? (ONE ? kRowWarps : 1) * kAhead<X, E> * 2 * S::bytes(threads) : 0) + (ONE ? (int)(2 * cols * sizeof(float)) : 0);
}

template <typename X, typename W, bool VEC, int E, bool ONE>
cudaError_t launch_forward_rows(const NormForwardArgs& a, int64_t blocks, int threads, cudaStream_t stream) {
  static std::atomic<uint64_t> ready{0};
  constexpr int kMost = forward_ring<X, VEC, E, ONE>(ONE ? 32 : threads_for(kBlockCols, E));
  return launch_ring<kMost>(forward_rows_kernel<X, W, VEC, E, ONE>, ready, blocks, threads, forward_ring<X, VEC, E, ONE>(ONE ? 32 : threads),
                            a, stream);
}

template <typename X, typename W, bool VEC, int E, bool ONE>
cudaError_t launch_backward_rows(const NormBackwardArgs& a, int threads, cudaStream_t stream) {
  static std::atomic<uint64_t> ready{0};
  constexpr int64_t kMostCols = ONE ? kWarpCols : E == 8 ? kSmallCols : kBlockCols;
  constexpr int kMost = backward_ring<X, VEC, E, ONE>(ONE ? 32 : threads_for(kMostCols, E), kMostCols);
  return launch_ring<kMost>(backward_kernel<X, W, VEC, E, ONE>, ready, a.parts, threads,
                            backward_ring<X, VEC, E, ONE>(ONE ? 32 : threads, a.cols), a, stream);
}

template <typename X, typename W, bool VEC>
cudaError_t launch_forward(const NormForwardArgs& a, cudaStream_t stream) {
  auto one = [&](auto* kernel) {
    return launch_dependent((const void*)kernel, (unsigned)((a.rows + kRowWarps - 1) / kRowWarps), 32 * kRowWarps, 0, 0, &a, stream);
  };
  auto block = [&](auto* kernel, int each) {
    return launch_dependent((const void*)kernel, (unsigned)a.rows, threads_for(a.cols, each), 0, 0, &a, stream);
  };
  // Few rows: as many threads to a row as there are packs, for its latency.
  if (a.rows <= 2 * kSms && a.cols > 256 && a.cols <= 8 * kMaxThreads) return block(forward_kernel<X, W, VEC, 8, false>, 8);
  if constexpr (Slice<X, VEC, 8>::kAsync) {  // as many rows in turn as make it worth while
    if (a.cols > 256 && a.cols <= kOneCols) {
      const int threads = 32 * kRowWarps, each = a.cols <= 512 ? 16 : a.cols <= 768 ? 24 : 32;
      const int64_t blocks = kSms * forward_blocks(each);
      if (a.rows >= 4 * blocks * kRowWarps) {
        if (each == 16) return launch_forward_rows<X, W, VEC, 16, true>(a, blocks, threads, stream);
        if (each == 24) return launch_forward_rows<X, W, VEC, 24, true>(a, blocks, threads, stream);
        return launch_forward_rows<X, W, VEC, 32, true>(a, blocks, threads, stream);
      }
    } else if (a.cols > kOneCols && a.cols <= kBlockCols) {
      constexpr int kEach = sizeof(X) == 2 ? 32 : 16, kRegs = sizeof(X) == 2 ? 152 : VEC ? 104 : 120;
      const int threads = threads_for(a.cols, kEach);
      const int64_t blocks = kSms * std::max(1, kRegisters / (kRegs * threads));
      if (a.rows >= 4 * blocks) return launch_forward_rows<X, W, VEC, kEach, false>(a, blocks, threads, stream);
    }
  }
  if (a.cols <= 256) return one(forward_kernel<X, W, VEC, 8, true>);
  if (a.cols <= 512) return one(forward_kernel<X, W, VEC, 16, true>);
  if (a.cols <= 768) return one(forward_kernel<X, W, VEC, 24, true>);
  if (a.cols <= kOneCols) return one(forward_kernel<X, W, VEC, 32, true>);
  if (a.cols <= kBlockCols) return block(forward_kernel<X, W, VEC, 16, false>, 16);
  return launch_dependent((const void*)forward_wide_kernel<X, W>, (unsigned)a.rows, kWideThreads, 0, 0, &a, stream);
}

template <typename X, typename W, bool VEC>
cudaError_t launch_backward(const NormBackwardArgs& a, cudaStream_t stream) {
  if (a.cols <= kWarpCols) return launch_backward_rows<X, W, VEC, 8, true>(a, 32 * kRowWarps, stream);
  if (a.cols <= kSmallCols) return launch_backward_rows<X, W, VEC, 8, false>(a, threads_for(a.cols, 8), stream);
  if (a.cols <= kBlockCols) return launch_backward_rows<X, W, VEC, 16, false>(a, threads_for(a.cols, 16), stream);
  if (a.dx) {
    const cudaError_t e = launch_dependent((const void*)backward_wide_kernel<X, W>, (unsigned)a.rows, kWideThreads, 0, 0, &a, stream);
    if (e != cudaSuccess) return e;
  }
  if (!a.partial) return cudaSuccess;
  const int64_t tiles = (a.cols + kWideThreads - 1) / kWideThreads;
  return launch_dependent((const void*)wide_sums_kernel<X>, (unsigned)(tiles * a.parts), kWideThreads, 0, 0, &a, stream);
}

}  // namespace

// Blocks of the backward pass: as many as an SM has room for, of at least 4 rows each (a warp of its own for every row where a
// row is one warp's), so that what they sum up is little beside what they read.
int norm_parts(int64_t rows, int64_t cols) {
  if (cols <= kWarpCols) return (int)std::min<int64_t>((rows + kRowWarps - 1) / kRowWarps, 2 * kSms);
  if (cols <= kSmallCols) return (int)std::min<int64_t>((rows + 3) / 4, kSms * std::min(4, 768 / threads_for(cols, 8)));
  if (cols <= kBlockCols) return (int)std::min<int64_t>(rows, kSms * std::max(1, 512 / threads_for(cols, 16)));
  return (int)std::min<int64_t>(rows, 32);
}

cudaError_t launch_norm_forward(const NormForwardArgs& a, cudaStream_t stream) {
  const int64_t xs = a.x_f32 ? 4 : 2;
  const bool vec = a.cols % (16 / xs) == 0 && whole_packs(a.x, a.ldx, a.rows, xs) && whole_packs(a.y, a.ldy, a.rows, xs) &&
                   whole_packs(a.w, 0, 1, 1) && whole_packs(a.b, 0, 1, 1);
  if (a.x_f32) return vec ? launch_forward<float, float, true>(a, stream) : launch_forward<float, float, false>(a, stream);
  if (a.w_f32) return vec ? launch_forward<uint16_t, float, true>(a, stream) : launch_forward<uint16_t, float, false>(a, stream);
  return vec ? launch_forward<uint16_t, uint16_t, true>(a, stream) : launch_forward<uint16_t, uint16_t, false>(a, stream);
}

cudaError_t launch_norm_backward(const NormBackwardArgs& a, cudaStream_t stream) {
  const int64_t xs = a.x_f32 ? 4 : 2;
  const bool vec = a.cols % (16 / xs) == 0 && whole_packs(a.x, a.ldx, a.rows, xs) && whole_packs(a.dy, a.lddy, a.rows, xs) &&
                   whole_packs(a.dx, a.lddx, a.rows, xs) && whole_packs(a.w, 0, 1, 1);
  if (a.x_f32) return vec ? launch_backward<float, float, true>(a, stream) : launch_backward<float, float, false>(a, stream);
  if (a.w_f32) return vec ? launch_backward<uint16_t, float, true>(a, stream) : launch_backward<uint16_t, float, false>(a, stream);
  return vec ? launch_backward<uint16_t, uint16_t, true>(a, stream) : launch_backward<uint16_t, uint16_t, false>(a, stream);
}

cudaError_t launch_norm_sums(const NormSumArgs& a, cudaStream_t stream) {
  const unsigned grid = (unsigned)(2 * ((a.cols + 31) / 32));
  return a.w_f32 ? launch_dependent((const void*)sums_kernel<float>, grid, 1024, 0, 0, &a, stream)
                 : launch_dependent((const void*)sums_kernel<uint16_t>, grid, 1024, 0, 0, &a, stream);
}

}  // namespace mpadam
