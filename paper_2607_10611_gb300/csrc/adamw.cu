// adamw.cu -- AdamW over a list of tensors, with moments in binary32 or in 8
// bits, and the global norm of a list of gradients.
//
// Per element, every operation rounded on its own in binary32 (include/mpadam.h):
//   g' = g s        m' = b1 m + (1 - b1) g'        v' = b2 v + (1 - b2) (g' g')
//   r' = sqrt(v')   w' = (w - kwd w) - (ka m') / (r' c2 + eps)
// In 8 bits the moments are held as m and r = sqrt(v), E4M3 codes with one
// power-of-two scale per 128 elements: the root halves the second moment's
// range, and the update needs it anyway.
#include "adamw.h"
#include "step_kernel.cuh"

namespace mpadam {

namespace {

constexpr int kThreads8 = kListTile / 8;  // 8 elements a thread

__device__ __forceinline__ const void* grad_of(const GradTable& g, int k) { return g.grads ? g.grads[k] : g.inline_grads[k]; }

// 8 values at p[at ..], `left` of them inside; whole and aligned ones in vector loads.
template <bool F32>
__device__ __forceinline__ void load8(const void* p, int64_t at, int64_t left, bool vec, float (&x)[8]) {
  if (F32) {
    const float* q = static_cast<const float*>(p) + at;
    if (vec && left >= 8) {
      const float4 a = __ldcs(reinterpret_cast<const float4*>(q)), b = __ldcs(reinterpret_cast<const float4*>(q) + 1);
      x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = j < left ? q[j] : 0.0f;
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    if (vec && left >= 8) {
      const uint4 a = __ldcs(reinterpret_cast<const uint4*>(q));
      const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) x[2 * j] = bf16_lo(u[j]), x[2 * j + 1] = bf16_hi(u[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = j < left ? __uint_as_float((uint32_t)q[j] << 16) : 0.0f;
    }
  }
}

__device__ __forceinline__ void store8_f32(void* p, int64_t at, int64_t left, bool vec, const float (&x)[8]) {
  float* q = static_cast<float*>(p) + at;
  if (vec && left >= 8) {
    __stcs(reinterpret_cast<float4*>(q), make_float4(x[0], x[1], x[2], x[3]));
    __stcs(reinterpret_cast<float4*>(q) + 1, make_float4(x[4], x[5], x[6], x[7]));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) q[j] = x[j];
  }
}
// Packed BF16 pairs.
__device__ __forceinline__ void store8_bf16(void* p, int64_t at, int64_t left, bool vec, const uint32_t (&u)[4]) {
  uint16_t* q = static_cast<uint16_t*>(p) + at;
  if (vec && left >= 8) {
    __stcs(reinterpret_cast<uint4*>(q), make_uint4(u[0], u[1], u[2], u[3]));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) q[j] = (uint16_t)(u[j / 2] >> (16 * (j & 1)));
  }
}
__device__ __forceinline__ uint2 load8_codes(const uint8_t* q, int64_t left, bool vec) {
  if (vec && left >= 8) return __ldcs(reinterpret_cast<const uint2*>(q));
  uint32_t u[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (j < left) u[j / 4] |= (uint32_t)q[j] << (8 * (j & 3));
  return make_uint2(u[0], u[1]);
}
__device__ __forceinline__ void store8_codes(uint8_t* q, int64_t left, bool vec, uint2 c) {
  if (vec && left >= 8) {
    __stcs(reinterpret_cast<uint2*>(q), c);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < left) q[j] = (uint8_t)((j < 4 ? c.x : c.y) >> (8 * (j & 3)));
  }
}

// 8 E4M3 codes times 2^(scale - 127).
__device__ __forceinline__ void decode8(uint2 c, uint32_t scale, float (&x)[8]) {
  const float s = __uint_as_float(scale == 0 ? 0x00400000u : scale << 23);
  const uint32_t u[2] = {c.x, c.y};
  e4m3x8_to_f32(u, x);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = __fmul_rn(x[j], s);
}

// The largest finite |x| (as bits) of the 16 lanes that own a block of 128, and the block's exponent from it: the
// smallest k >= -127 with A <= 448 2^k (448 = 1.75 2^8: the addition carries into the exponent where the mantissa is
// above 1.75); 0 where all are 0.
__device__ __forceinline__ int block_exponent(const float (&x)[8]) {
  uint32_t a = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t b = __float_as_uint(x[j]) & 0x7FFFFFFFu;
    a = max(a, b < 0x7F800000u ? b : 0u);
  }
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) a = max(a, __shfl_xor_sync(~0u, a, d));
  return a == 0 ? 0 : max(-127, (int)((a + 0x1FFFFFu) >> 23) - 135);
}

// Stochastic rounding onto E4M3's grid by 16 random bits r: they are added below the grid's last bit and the rest is
// cut off.  Below 2^-6 the grid is even with step 2^-9, as it is in [2^-6, 2^-5), where the value is moved for it.
__device__ __forceinline__ float e4m3_stochastic(float y, uint32_t r) {
  const float a = fabsf(y);
  const float off = a < 0x1p-6f ? 0x1p-6f : 0.0f;
  const uint32_t b = __float_as_uint(__fadd_rn(a, off)) + (r << 4);
  const float z = __fsub_rn(__uint_as_float(b & ~0xFFFFFu), off);
  return a <= 448.0f ? copysignf(z, y) : y;
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
  uint16_t h;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h) : "f"(hi), "f"(lo));
  return h;
}

// 8 values as codes under the block exponent k; lanes: their random bits, in the half of each word that `shift` names.
// keep: a value above 0 is never stored as 0 (the second moment's root, which the update divides by).
template <bool SR, bool KEEP>
__device__ __forceinline__ uint2 encode8(const float (&x)[8], int k, const uint32_t (&lanes)[8], int shift) {
  const float inv = __uint_as_float((uint32_t)(127 - k) << 23);
  uint32_t c[2] = {0, 0};
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    float y[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      y[i] = __fmul_rn(x[j + i], inv);
      if (SR) y[i] = e4m3_stochastic(y[i], (lanes[j + i] >> shift) & 0xFFFFu);
      if (KEEP && x[j + i] > 0.0f) y[i] = fmaxf(y[i], 0x1p-9f);
    }
    c[j / 4] |= e4m3x2(y[0], y[1]) << (8 * (j & 3));
  }
  return make_uint2(c[0], c[1]);
}

template <bool W32, bool G32, bool LOW, bool SR, bool STATE_SR>
__global__ void __launch_bounds__(kThreads8) adamw_kernel(const __grid_constant__ AdamwArgs p) {
  float mult = 1.0f;
  if (p.grad_scale) {
    mult = *p.grad_scale;
    if (mult != mult) return;  // the norm was not finite: the step is skipped
  }
  const AdamwScalars& s = p.s;
  for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
    const int k = p.tile_tensor[t];
    const ListTensor& d = p.tensors[k];
    const void* grad = grad_of(p.g, k);
    const int64_t at = (t - d.tile0) * kListTile + threadIdx.x * 8;
    const int64_t left = d.numel - at;
    const bool vec = d.aligned, gvec = (reinterpret_cast<uintptr_t>(grad) & 15) == 0;
    float w[8], g[8], m[8], v[8], r[8];
    load8<G32>(grad, at, left, gvec, g);
    load8<W32>(d.w, at, left, vec, w);
    uint8_t *mc = nullptr, *vc = nullptr;
    int64_t block = at / 128;
    if (LOW) {
      mc = static_cast<uint8_t*>(d.m) + at;
      vc = static_cast<uint8_t*>(d.v) + at;
      const uint32_t ms = left > 0 ? d.m_scale[block] : 127u, vs = left > 0 ? d.v_scale[block] : 127u;
      decode8(load8_codes(mc, left, vec), ms, m);
      decode8(load8_codes(vc, left, vec), vs, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], v[j]);
    } else {
      load8<true>(d.m, at, left, vec, m);
      load8<true>(d.v, at, left, vec, v);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float gs = p.grad_scale ? __fmul_rn(g[j], mult) : g[j];
      m[j] = __fadd_rn(__fmul_rn(m[j], s.b1), __fmul_rn(gs, s.omb1));
      v[j] = __fadd_rn(__fmul_rn(v[j], s.b2), __fmul_rn(__fmul_rn(gs, gs), s.omb2));
      r[j] = __fsqrt_rn(v[j]);
      const float u = __fdiv_rn(__fmul_rn(m[j], s.ka), __fadd_rn(__fmul_rn(r[j], s.c2), s.eps));
      const float base = s.kwd != 0.0f ? __fsub_rn(w[j], __fmul_rn(w[j], s.kwd)) : w[j];
      w[j] = __fsub_rn(base, u);
    }
    const int64_t gi = d.goff + at;
    if (LOW) {
      uint32_t lanes[8] = {};
      if (STATE_SR) {
        const uint64_t b = (uint64_t)gi >> 2;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint4 x = philox4x32_10((uint32_t)(b + i), (uint32_t)((b + i) >> 32) | 0x80000000u, p.t_lo, p.t_hi, p.rk0, p.rk1);
          lanes[4 * i] = x.x, lanes[4 * i + 1] = x.y, lanes[4 * i + 2] = x.z, lanes[4 * i + 3] = x.w;
        }
      }
      const int km = block_exponent(m), kv = block_exponent(r);
      store8_codes(mc, left, vec, encode8<STATE_SR, false>(m, km, lanes, 0));
      store8_codes(vc, left, vec, encode8<STATE_SR, true>(r, kv, lanes, 16));
      if ((threadIdx.x & 15) == 0 && left > 0) {
        d.m_scale[block] = (uint8_t)(km + 127);
        d.v_scale[block] = (uint8_t)(kv + 127);
      }
    } else {
      store8_f32(d.m, at, left, vec, m);
      store8_f32(d.v, at, left, vec, v);
    }
    if (W32) store8_f32(d.w, at, left, vec, w);
    if (!W32 || d.compute) {
      uint32_t u[4];
      if (!W32 && SR) {
        const uint64_t b = (uint64_t)gi >> 3;
        const uint4 x = philox4x32_10((uint32_t)b, (uint32_t)(b >> 32), p.t_lo, p.t_hi, p.rk0, p.rk1);
        const uint32_t rnd[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          u[j] = __byte_perm(bf16_sr_sum(w[2 * j], ~rnd[j] & 0xFFFFu), bf16_sr_sum(w[2 * j + 1], ~rnd[j] >> 16), 0x7632);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = bf16x2_rn(w[2 * j], w[2 * j + 1]);
      }
      if (!W32) store8_bf16(d.w, at, left, vec, u);
      else store8_bf16(d.compute, at, left, vec, u);
    }
  }
}

template <bool G32>
__global__ void __launch_bounds__(kThreads8) grad_norm_kernel(const __grid_constant__ NormArgs p) {
  __shared__ double part[kThreads8 / 32];
  __shared__ bool last;
  float acc[4] = {};
  for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
    const int k = p.tile_tensor[t];
    const ListTensor& d = p.tensors[k];
    const void* grad = grad_of(p.g, k);
    const int64_t at = (t - d.tile0) * kListTile + threadIdx.x * 8;
    float g[8];
    load8<G32>(grad, at, d.numel - at, (reinterpret_cast<uintptr_t>(grad) & 15) == 0, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j & 3] = __fmaf_rn(g[j], g[j], acc[j & 3]);
  }
  auto block_sum = [&](double x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0;
    for (int w = 0; w < kThreads8 / 32; ++w) x += part[w];
    return x;
  };
  const double mine = block_sum(((double)acc[0] + acc[1]) + ((double)acc[2] + acc[3]));
  if (threadIdx.x == 0) {
    p.partial[blockIdx.x] = mine;
    __threadfence();
    last = atomicAdd(p.done, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double x = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads8) x += __ldcg(p.partial + i);
  x = block_sum(x);
  if (threadIdx.x == 0) {
    const double norm = sqrt(x);
    const float n = (float)norm;
    p.out[0] = n;
    p.out[1] = isfinite(n) ? (norm > (double)p.max_norm ? (float)((double)p.max_norm / norm) : 1.0f) : __uint_as_float(0x7FC00000u);
    *p.done = 0;
  }
}

struct FillArgs {
  const void** table;
  int32_t first, count;
  const void* grads[kInlineGrads];
};
__global__ void fill_kernel(const __grid_constant__ FillArgs a) {
  for (int i = threadIdx.x; i < a.count; i += blockDim.x) a.table[a.first + i] = a.grads[i];
}

template <bool W32, bool G32, bool LOW>
void* pick(bool sr, bool state_sr) {
  if (W32) sr = false;
  if (!LOW) state_sr = false;
  if (sr) return state_sr ? (void*)adamw_kernel<W32, G32, LOW, !W32, LOW> : (void*)adamw_kernel<W32, G32, LOW, !W32, false>;
  return state_sr ? (void*)adamw_kernel<W32, G32, LOW, false, LOW> : (void*)adamw_kernel<W32, G32, LOW, false, false>;
}
template <bool W32, bool G32>
void* pick(const AdamwKind& k) {
  return k.state_e4m3 ? pick<W32, G32, true>(k.sr, k.state_sr) : pick<W32, G32, false>(k.sr, k.state_sr);
}

}  // namespace

cudaError_t launch_adamw(const AdamwArgs& a, const AdamwKind& k, cudaStream_t stream) {
  void* kernel = k.w_f32 ? (k.g_f32 ? pick<true, true>(k) : pick<true, false>(k))
                         : (k.g_f32 ? pick<false, true>(k) : pick<false, false>(k));
  void* params[] = {const_cast<AdamwArgs*>(&a)};
  const int64_t grid = a.tiles < 152 * 8 ? a.tiles : 152 * 8;
  return cudaLaunchKernel(kernel, dim3((unsigned)grid), dim3(kThreads8), params, 0, stream);
}

cudaError_t launch_grad_norm(const NormArgs& a, cudaStream_t stream) {
  const unsigned grid = (unsigned)(a.tiles < kNormCtas ? (a.tiles ? a.tiles : 1) : kNormCtas);
  if (a.g_f32) grad_norm_kernel<true><<<grid, kThreads8, 0, stream>>>(a);
  else grad_norm_kernel<false><<<grid, kThreads8, 0, stream>>>(a);
  return cudaGetLastError();
}

cudaError_t fill_grads(const void** table, const void* const* grads, int32_t first, int32_t count, cudaStream_t stream) {
  FillArgs f;
  f.table = table;
  f.first = first;
  f.count = count;
  for (int32_t i = 0; i < count; ++i) f.grads[i] = grads[i];
  fill_kernel<<<1, 128, 0, stream>>>(f);
  return cudaGetLastError();
}

}  // namespace mpadam
