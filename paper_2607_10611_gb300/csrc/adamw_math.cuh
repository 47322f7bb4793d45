// adamw_math.cuh -- the AdamW step's arithmetic on packed binary32 pairs.
#pragma once

#include "step_kernel.cuh"

namespace mpadam {

__device__ __forceinline__ float rsqrt_approx_ftz(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ f32x2 both(float x) { return pk(x, x); }

// x y rounded by itself, also where a sum follows.  A mul.rn.f32x2 whose result
// an add.rn.f32x2 takes came out as one fused operation, and so did a fused one
// with a constant -0; so the -0 is a value that only the launch knows.
__device__ __forceinline__ f32x2 prod2(f32x2 x, f32x2 y, f32x2 minus_zero) { return fma2_rn(x, y, minus_zero); }

// Correctly rounded square roots of two values in [0, 2^32): a Newton step with
// an exact residual from the hardware's 1 / sqrt (P. Markstein, "Computation of
// elementary functions on the IBM RISC System/6000 processor", IBM J. R&D 34(1),
// 1990).  Values are scaled by 2^96 first, so that neither they nor the residual
// is subnormal; the root's scale, 2^48, comes off exactly.  The scaled value and
// root are held negated: fma(s, s, t) is then minus the residual.  From 2^32 on
// the scaled value is infinite and the result NaN.  That every result is the
// correctly rounded one is tested for each of the 1.3 10^9 binary32 values in
// the range (tests/test_gpu_adamw.py).  Five instructions a value, against
// eleven.
__device__ __forceinline__ f32x2 root2(f32x2 v) {
  const f32x2 t = mul2_rn(v, both(-0x1p96f));
  float t0, t1;
  unpk(t, t0, t1);
  const f32x2 y = pk(rsqrt_approx_ftz(fmaxf(fabsf(t0), 0x1p-60f)), rsqrt_approx_ftz(fmaxf(fabsf(t1), 0x1p-60f)));
  const f32x2 s = mul2_rn(t, y);
  const f32x2 e = fma2_rn(s, s, t);
  return fma2_rn(fma2_rn(e, mul2_rn(y, both(0.5f)), s), both(-0x1p-48f), 0ull);  // (the sum makes the root of 0 positive)
}

// a / d rounded correctly, for nd = -d with d in [2^-100, 2^100], and a = 0 or
// |a| >= 2^-100 with a quotient that is neither subnormal nor too large (a
// quotient that overflows comes out as no finite value), in the same paper's way: y, the reciprocal after one Newton
// step, is the correctly rounded one (tested for every mantissa,
// tests/test_gpu_adamw.py); a quotient within one unit that is corrected with its
// exact remainder and such a reciprocal then is too.  Six instructions for two
// values, and the hardware's reciprocals.
__device__ __forceinline__ f32x2 reciprocal2(f32x2 nd) {
  float d0, d1;
  unpk(nd, d0, d1);
  const f32x2 y = pk(rcp_approx_ftz(-d0), rcp_approx_ftz(-d1));
  return fma2_rn(fma2_rn(nd, y, both(1.0f)), y, y);
}
__device__ __forceinline__ f32x2 quotient2(f32x2 a, f32x2 nd) {
  const f32x2 y = reciprocal2(nd);
  const f32x2 q = mul2_rn(a, y);
  return fma2_rn(fma2_rn(nd, q, a), y, q);
}

// Stochastic rounding by the hardware's conversions: the random bits are added
// below the result's last bit and the rest is cut off.  These two are what the
// step defines (and what its general code computes in integers) for finite BF16
// results, and for E4M3 ones of values up to 448 that are 0, at least 2^-6, or
// multiples of 2^-29 below that; tested for every such value
// (tests/test_gpu_adamw.py).  rs_bf16x2: lo by the random word's low half, hi by
// its high half.  rs_codes: a code in byte 0 by the low half, one in byte 2 by
// the high half; the other two bytes are 0.
__device__ __forceinline__ uint32_t rs_bf16x2(float lo, float hi, uint32_t rnd) {
  uint32_t d;
  asm("cvt.rs.bf16x2.f32 %0, %1, %2, %3;" : "=r"(d) : "f"(hi), "f"(lo), "r"(rnd));
  return d;
}
__device__ __forceinline__ uint32_t rs_codes(float lo, float hi, uint32_t rnd) {
  uint32_t d;
  asm("cvt.rs.satfinite.e4m3x4.f32 %0, {%3, %1, %3, %2}, %4;" : "=r"(d) : "f"(hi), "f"(lo), "f"(0.0f), "r"(rnd));
  return d;
}
// Values below 2^-6 onto the multiples of 2^-29, as the sum with 2^-6 rounds them.
__device__ __forceinline__ float settle(float y) {
  const float a = fabsf(y);
  return a < 0x1p-6f ? copysignf(__fsub_rn(__fadd_rn(a, 0x1p-6f), 0x1p-6f), y) : y;
}

}  // namespace mpadam
