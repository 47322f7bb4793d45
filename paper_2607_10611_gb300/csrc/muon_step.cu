// muon_step.cu -- what a Muon step does around its products (muon_products.cu),
// element by element over a list of matrices:
//   squares: the sum of U's squares, U = b m' + (1-b) g' (Nesterov) or m', with
//            m' = b m + (1-b) g';  for orthogonalisation alone U is the input
//   begin:   m' is stored, and X = U / |U| in two parts (muon.h)
//   finish:  w' = (w - kwd w) - ka O, rounded; or O is written out
// Every operation rounds on its own, in binary32; the squares' sums are in
// binary64 above 32 of them.
#include <algorithm>
#include <type_traits>

#include "launch.h"
#include "muon.h"
#include "step_kernel.cuh"

namespace mpadam {

namespace {

constexpr int kStepThreads = 256;
constexpr int kVectors = kSquaresPass / kStepThreads / 8;
// A tile's vectors of 8 across, the rows that a block takes at once, and how often.
constexpr int kAcross = kTileCols / 8, kDown = kStepThreads / kAcross, kTimes = kTileRows / kDown;
// Turned: the same of its columns.
constexpr int kAcrossT = kTileRows / 8, kDownT = kStepThreads / kAcrossT, kTimesT = kTileCols / kDownT;

__device__ __forceinline__ void wait_for_earlier_kernels() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ float bf16_value(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }
__device__ __forceinline__ uint16_t half_of(float x) {
  uint16_t h;
  asm("cvt.rn.f16.f32 %0, %1;" : "=h"(h) : "f"(x));
  return h;
}
__device__ __forceinline__ float of_half(uint16_t h) {
  float x;
  asm("cvt.f32.f16 %0, %1;" : "=f"(x) : "h"(h));
  return x;
}

// `count` (at most 8) of 8 consecutive elements from element `at`; vec: all 8, on a 16-byte boundary.
template <bool F32>
__device__ __forceinline__ void load8(const void* p, int64_t at, int count, bool vec, float (&x)[8]) {
  if (F32) {
    const float* q = static_cast<const float*>(p) + at;
    if (vec) {
      const float4 a = *reinterpret_cast<const float4*>(q), b = *reinterpret_cast<const float4*>(q + 4);
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = i < count ? q[i] : 0.0f;
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    if (vec) {
      const uint4 v = *reinterpret_cast<const uint4*>(q);
      const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(u[i] << 16), x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = i < count ? bf16_value(q[i]) : 0.0f;
    }
  }
}
template <bool F32>
__device__ __forceinline__ void store8(void* p, int64_t at, int count, bool vec, const float (&x)[8]) {
  if (F32) {
    float* q = static_cast<float*>(p) + at;
    if (vec) {
      *reinterpret_cast<float4*>(q) = make_float4(x[0], x[1], x[2], x[3]);
      *reinterpret_cast<float4*>(q + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < count) q[i] = x[i];
    }
  } else {
    uint16_t* q = static_cast<uint16_t*>(p) + at;
    if (vec) {
      *reinterpret_cast<uint4*>(q) = make_uint4(bf16x2_rn(x[0], x[1]), bf16x2_rn(x[2], x[3]), bf16x2_rn(x[4], x[5]), bf16x2_rn(x[6], x[7]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < count) q[i] = (uint16_t)bf16x2_rn(x[i], 0.0f);
    }
  }
}

__device__ __forceinline__ const void* pointer_of(const GradTable& t, int k) { return t.grads ? t.grads[k] : t.inline_grads[k]; }
__device__ __forceinline__ bool on_16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// A NaN multiplier: the step changes nothing.
__device__ __forceinline__ bool skipped(const MuonArgs& p) { return p.grad_scale && isnan(*p.grad_scale); }

// The momentum and U of 8 elements; `m` comes out as it is stored, before its rounding.
template <bool STEP, bool G32, bool M32>
__device__ __forceinline__ void update8(const MuonArgs& p, const MuonMatrix& q, const void* in, int64_t at, int count, bool vec,
                                        float scale, float (&m)[8], float (&u)[8]) {
  load8<G32>(in, at, count, vec, u);
  if (!STEP) return;
  load8<M32>(q.m, at, count, vec, m);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float g = __fmul_rn(__fmul_rn(u[i], scale), p.rest);
    m[i] = __fadd_rn(__fmul_rn(m[i], p.beta), g);
    u[i] = p.nesterov ? __fadd_rn(__fmul_rn(m[i], p.beta), g) : m[i];
  }
}
// (without a multiplier, 1: g 1 is g)
__device__ __forceinline__ float multiplier(const MuonArgs& p) { return p.grad_scale ? *p.grad_scale : 1.0f; }

__device__ __forceinline__ double block_sum(double x) {
  __shared__ double part[kStepThreads / 32];
#pragma unroll
  for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
  __syncthreads();
  x = 0.0;
#pragma unroll
  for (int i = 0; i < kStepThreads / 32; ++i) x += part[i];
  return x;
}

// 2^e for e in [-126, 127], and in binary64 for e in [-1022, 1023].
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ double pow2d(int e) { return __longlong_as_double((long long)(e + 1023) << 52); }

// A block takes a chunk of a matrix, 32 elements a thread at once.  Those are
// scaled by a power of two so that no square leaves binary32's range: momentum
// that decays without gradients keeps its direction down to its last bits.
template <bool STEP, bool G32, bool M32>
__global__ void __launch_bounds__(kStepThreads, 4) squares_kernel(const __grid_constant__ MuonArgs p) {
  wait_for_earlier_kernels();
  if (skipped(p)) return;
  const float scale = multiplier(p);
  const int k = p.owner[blockIdx.x];
  const MuonMatrix& q = p.matrices[k];
  const void* in = pointer_of(p.in, q.index);
  const int64_t numel = (int64_t)q.rows * q.cols, first = (blockIdx.x - q.chunk0) * (int64_t)q.chunk;
  const int64_t end = min(numel, first + q.chunk);
  const bool vec = on_16(in) && (!STEP || q.aligned);
  double sum = 0.0;
  auto pass = [&](int64_t base, auto whole_pass) {
    constexpr bool all = decltype(whole_pass)::value;  // of vectors
    float u[kVectors][8];
#pragma unroll
    for (int v = 0; v < kVectors; ++v) {
      const int64_t at = base + (v * kStepThreads + threadIdx.x) * 8;
      const int count = all ? 8 : (int)max((int64_t)0, min((int64_t)8, end - at));
      float m[8];
      if (all || count) {
        update8<STEP, G32, M32>(p, q, in, at, count, all || (vec && count == 8), scale, m, u[v]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[v][i] = 0.0f;
      }
    }
    float most = 0.0f;
#pragma unroll
    for (int v = 0; v < kVectors; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(u[v][i]));
    const int e = max(-100, min(126, (int)(__float_as_uint(most) >> 23) - 127));
    const float down = pow2f(-e);
    float s[4] = {};
#pragma unroll
    for (int v = 0; v < kVectors; ++v)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = __fmul_rn(u[v][i], down);
        s[i & 3] = __fmaf_rn(x, x, s[i & 3]);
      }
    sum += (double)__fadd_rn(__fadd_rn(s[0], s[1]), __fadd_rn(s[2], s[3])) * pow2d(2 * e);
  };
  for (int64_t base = first; base < end; base += kSquaresPass) {
    if (vec && end - base >= kSquaresPass) pass(base, std::true_type());
    else pass(base, std::false_type());
  }
  // The last of a matrix's blocks sums up, in the chunks' order, and leaves the count as it was.
  __shared__ bool last;
  sum = block_sum(sum);
  if (threadIdx.x == 0) {
    p.partial[blockIdx.x] = sum;
    __threadfence();
    last = atomicAdd(&p.norms[k].done, 1u) == (uint32_t)q.chunks - 1;
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  sum = 0.0;
  for (int i = threadIdx.x; i < q.chunks; i += kStepThreads) sum += __ldcg(p.partial + q.chunk0 + i);
  sum = block_sum(sum);
  if (threadIdx.x == 0) {
    const double norm = sqrt(sum);
    MuonNorm n{0.0f, 0.0f, 0.0f, 0u};
    if (!(norm <= 1e300)) {
      n = {1.0f, 1.0f, __uint_as_float(0x7FC00000u), 0u};  // no direction
    } else if (norm > 0.0) {  // |e| < 200: U has less than 2^41 elements
      const int e = (int)(__double_as_longlong(norm) >> 52) - 1023, half = e / 2;
      n = {pow2f(-half), pow2f(-(e - half)), (float)((double)kHeld / (norm * pow2d(-e))), 0u};
    }
    p.norms[k] = n;
  }
}

// A block takes a tile of 64 x 128 of the caller's matrix; a thread 8 neighbours
// of a row, four times.  A tall matrix's tile is turned in shared memory.
template <bool STEP, bool G32, bool M32>
__global__ void __launch_bounds__(kStepThreads, 4) begin_kernel(const __grid_constant__ MuonArgs p) {
  __shared__ uint32_t turned[kTileRows][kTileCols + 1];
  wait_for_earlier_kernels();
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < p.counters; i += kStepThreads) p.progress[i] = 0;
  if (skipped(p)) return;
  const float scale = multiplier(p);
  const MuonMatrix& q = p.matrices[p.owner[blockIdx.x]];
  const void* in = pointer_of(p.in, q.index);
  const int tile = blockIdx.x - q.tile0, i0 = tile / q.tiles_across * kTileRows, j0 = tile % q.tiles_across * kTileCols;
  const bool vec = q.cols % 8 == 0 && on_16(in) && (!STEP || q.aligned);
  const MuonNorm norm = p.norms[p.owner[blockIdx.x]];
  const int r = threadIdx.x / kAcross, c = threadIdx.x % kAcross * 8, rt = threadIdx.x / kAcrossT, ct = threadIdx.x % kAcrossT * 8;
  auto take = [&](auto whole_tile) {
    constexpr bool all = decltype(whole_tile)::value;  // of vectors
    float m[kTimes][8], u[kTimes][8];
#pragma unroll
    for (int h = 0; h < kTimes; ++h) {
      const int i = i0 + r + kDown * h, j = j0 + c, count = all ? 8 : i < q.rows ? max(0, min(8, q.cols - j)) : 0;
      if (all || count) update8<STEP, G32, M32>(p, q, in, (int64_t)i * q.cols + j, count, all || (vec && count == 8), scale, m[h], u[h]);
    }
#pragma unroll
    for (int h = 0; h < kTimes; ++h) {
      const int i = i0 + r + kDown * h, j = j0 + c, count = all ? 8 : i < q.rows ? max(0, min(8, q.cols - j)) : 0;
      uint32_t held[8] = {};
      if (all || count) {
        const int64_t at = (int64_t)i * q.cols + j;
        const bool whole = all || (vec && count == 8);
        if (STEP) store8<M32>(q.m, at, count, whole, m[h]);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float x = __fmul_rn(__fmul_rn(__fmul_rn(u[h][k], norm.down0), norm.down1), norm.rest);
          const uint16_t hi = half_of(x);
          held[k] = hi | (uint32_t)half_of(__fsub_rn(x, of_half(hi))) << 16;
        }
        if (!q.tall) {  // (rows' padding has room for whole vectors)
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) hi[k] = __byte_perm(held[2 * k], held[2 * k + 1], 0x5410), lo[k] = __byte_perm(held[2 * k], held[2 * k + 1], 0x7632);
          const int64_t to = (int64_t)i * q.ld + j;
          *reinterpret_cast<uint4*>(q.hi[0] + to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4*>(q.lo + to) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
      }
      if (q.tall) {
#pragma unroll
        for (int k = 0; k < 8; ++k) turned[r + kDown * h][c + k] = held[k];
      }
    }
  };
  if (vec && i0 + kTileRows <= q.rows && j0 + kTileCols <= q.cols) take(std::true_type());
  else take(std::false_type());
  if (!q.tall) return;
  __syncthreads();
#pragma unroll
  for (int h = 0; h < kTimesT; ++h) {
    const int j = j0 + rt + kDownT * h, i = i0 + ct;  // X's row and its first column
    if (j >= q.cols || i >= q.rows) continue;
    uint32_t x[8], hi[4], lo[4];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = turned[ct + k][rt + kDownT * h];
#pragma unroll
    for (int k = 0; k < 4; ++k) hi[k] = __byte_perm(x[2 * k], x[2 * k + 1], 0x5410), lo[k] = __byte_perm(x[2 * k], x[2 * k + 1], 0x7632);
    const int64_t to = (int64_t)j * q.ld + i;
    *reinterpret_cast<uint4*>(q.hi[0] + to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
    *reinterpret_cast<uint4*>(q.lo + to) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  }
}

// The 16 random bits of the elements e to e + 7 of the list, e a multiple of 8.
__device__ __forceinline__ void random_block(const MuonArgs& p, int64_t e, uint32_t* bits) {
  const uint64_t b = (uint64_t)e / 8;
  const uint4 r = philox4x32_10((uint32_t)b, (uint32_t)(b >> 32), (uint32_t)p.step, (uint32_t)((uint64_t)p.step >> 32), p.rk0, p.rk1);
  const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) bits[i] = i & 1 ? u[i / 2] >> 16 : u[i / 2] & 0xFFFFu;
}
// The same of any e: from the two blocks that they lie in.
__device__ __forceinline__ void random_lanes(const MuonArgs& p, int64_t e, uint32_t (&bits)[8]) {
  uint32_t two[16];
  random_block(p, e & ~(int64_t)7, two);
  random_block(p, (e & ~(int64_t)7) + 8, two + 8);
  // shifted down by e mod 8, in steps of 4, 2 and 1, so that the array stays in registers
#pragma unroll
  for (int d = 4; d; d >>= 1)
    if (e & d) {
#pragma unroll
      for (int i = 0; i + d < 16; ++i) two[i] = two[i + d];
    }
#pragma unroll
  for (int i = 0; i < 8; ++i) bits[i] = two[i];
}

template <bool STEP, bool W32, bool SR>
__global__ void __launch_bounds__(kStepThreads, 5) finish_kernel(const __grid_constant__ MuonArgs p) {
  __shared__ uint16_t turned[kTileRows][kTileCols + 2];
  wait_for_earlier_kernels();
  if (skipped(p) || *p.err) return;  // (a product that gave up: what there is, is no result)
  const MuonMatrix& q = p.matrices[p.owner[blockIdx.x]];
  const int tile = blockIdx.x - q.tile0, i0 = tile / q.tiles_across * kTileRows, j0 = tile % q.tiles_across * kTileCols;
  const int r = threadIdx.x / kAcross, c = threadIdx.x % kAcross * 8, rt = threadIdx.x / kAcrossT, ct = threadIdx.x % kAcrossT * 8;
  const uint16_t* x = q.hi[p.last];
  if (q.tall) {
#pragma unroll
    for (int h = 0; h < kTimesT; ++h) {
      const int j = j0 + rt + kDownT * h, i = i0 + ct;
      if (j >= q.cols || i >= q.rows) continue;
      const uint4 v = *reinterpret_cast<const uint4*>(x + (int64_t)j * q.ld + i);
      const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int k = 0; k < 8; ++k) turned[ct + k][rt + kDownT * h] = (uint16_t)(u[k / 2] >> 16 * (k & 1));
    }
    __syncthreads();
  }
  void* out = STEP ? nullptr : const_cast<void*>(pointer_of(p.out, q.index));
  const bool vec = q.cols % 8 == 0 && (STEP ? q.aligned != 0 : on_16(out));
  const float ka = __fmul_rn(p.lr, q.factor);
  auto take = [&](auto whole_tile) {
    constexpr bool all = decltype(whole_tile)::value;  // of vectors
    float weights[kTimes][8];
    if (STEP) {
#pragma unroll
      for (int h = 0; h < kTimes; ++h) {
        const int i = i0 + r + kDown * h, j = j0 + c, count = all ? 8 : i < q.rows ? max(0, min(8, q.cols - j)) : 0;
        if (all || count) load8<W32>(q.w, (int64_t)i * q.cols + j, count, all || (vec && count == 8), weights[h]);
      }
    }
#pragma unroll
    for (int h = 0; h < kTimes; ++h) {
      const int i = i0 + r + kDown * h, j = j0 + c, count = all ? 8 : i < q.rows ? max(0, min(8, q.cols - j)) : 0;
      if (!all && !count) continue;
      const int64_t at = (int64_t)i * q.cols + j;
      const bool whole = all || (vec && count == 8);
      float o[8];
      if (q.tall) {
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = of_half(turned[r + kDown * h][c + k]);
      } else {
        const uint4 v = *reinterpret_cast<const uint4*>(x + (int64_t)i * q.ld + j);
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 8; ++k) o[k] = of_half((uint16_t)(u[k / 2] >> 16 * (k & 1)));
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) o[k] = __fmul_rn(o[k], kFromHeld);
      if (!STEP) {
        store8<W32>(out, at, count, whole, o);
        continue;
      }
      float (&w)[8] = weights[h];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float kept = p.decay != 0.0f ? __fsub_rn(w[k], __fmul_rn(w[k], p.decay)) : w[k];
        w[k] = __fsub_rn(kept, __fmul_rn(o[k], ka));
      }
      if (SR) {
        uint32_t bits[8];
        if (all) random_block(p, q.goff + at, bits);  // (rows start at multiples of 8)
        else random_lanes(p, q.goff + at, bits);
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = bf16_value((uint16_t)(bf16_sr_sum(w[k], ~bits[k] & 0xFFFFu) >> 16));
      }
      store8<W32>(q.w, at, count, whole, w);
      if (W32 && q.compute) store8<false>(q.compute, at, count, whole, w);
    }
  };
  if (vec && i0 + kTileRows <= q.rows && j0 + kTileCols <= q.cols) take(std::true_type());
  else take(std::false_type());
}

template <bool STEP, bool G32, bool M32>
cudaError_t squares(const MuonArgs& a, cudaStream_t stream) {
  return launch_dependent((const void*)squares_kernel<STEP, G32, M32>, (unsigned)a.count, kStepThreads, 0, 0, &a, stream);
}
template <bool STEP, bool G32, bool M32>
cudaError_t begin(const MuonArgs& a, cudaStream_t stream) {
  return launch_dependent((const void*)begin_kernel<STEP, G32, M32>, (unsigned)a.count, kStepThreads, 0, 0, &a, stream);
}
template <bool STEP, bool W32, bool SR>
cudaError_t finish(const MuonArgs& a, cudaStream_t stream) {
  return launch_dependent((const void*)finish_kernel<STEP, W32, SR>, (unsigned)a.count, kStepThreads, 0, 0, &a, stream);
}

}  // namespace

cudaError_t launch_squares(const MuonArgs& a, const MuonKind& k, cudaStream_t stream) {
  if (!k.step) return k.in_f32 ? squares<false, true, true>(a, stream) : squares<false, false, true>(a, stream);
  if (k.in_f32) return k.m_f32 ? squares<true, true, true>(a, stream) : squares<true, true, false>(a, stream);
  return k.m_f32 ? squares<true, false, true>(a, stream) : squares<true, false, false>(a, stream);
}

cudaError_t launch_begin(const MuonArgs& a, const MuonKind& k, cudaStream_t stream) {
  if (!k.step) return k.in_f32 ? begin<false, true, true>(a, stream) : begin<false, false, true>(a, stream);
  if (k.in_f32) return k.m_f32 ? begin<true, true, true>(a, stream) : begin<true, true, false>(a, stream);
  return k.m_f32 ? begin<true, false, true>(a, stream) : begin<true, false, false>(a, stream);
}

cudaError_t launch_finish(const MuonArgs& a, const MuonKind& k, cudaStream_t stream) {
  if (!k.step) return k.w_f32 ? finish<false, true, false>(a, stream) : finish<false, false, false>(a, stream);
  if (k.w_f32) return finish<true, true, false>(a, stream);
  return k.stochastic ? finish<true, false, true>(a, stream) : finish<true, false, false>(a, stream);
}

}  // namespace mpadam
