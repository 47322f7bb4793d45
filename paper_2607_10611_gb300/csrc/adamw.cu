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
#include "adamw_math.cuh"
#include "launch.h"

namespace mpadam {

namespace {

__device__ __forceinline__ void wait_for_earlier_kernels() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// mbar_wait for a whole warp, which goes on or leaves with all its lanes.  (With the vote behind the lanes' loops, a 7B-width
// shard's step in 8 bits takes 1906 us, so 1845.)
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) {
  for (uint32_t i = 0; i < kSpinLimit; ++i)
    if (__all_sync(~0u, mbar_try_wait(bar, parity))) return true;
  return false;
}

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

// vec32: the array is on a 32-byte boundary, so that a thread's 8 values go in one access and fill a sector; vec: on a
// 16-byte one, as views of flat buffers may be: two accesses.  GPT-2's step takes 557 us in
// the first way, 562 in the second, 1030 in single words.
__device__ __forceinline__ void store8_f32(void* p, int64_t at, int64_t left, bool vec, bool vec32, const float (&x)[8]) {
  float* q = static_cast<float*>(p) + at;
  if (vec32 && left >= 8) {
    uint32_t u[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = __float_as_uint(x[j]);
    st8(q, u);
  } else if (vec && left >= 8) {
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

// The values of 8 E4M3 codes, and of an E8M0 scale.
__device__ __forceinline__ void decode8(uint2 c, float (&x)[8]) {
  const uint32_t u[2] = {c.x, c.y};
  e4m3x8_to_f32(u, x);
}
// The squares of 8 E4M3 codes' values, exactly: one product of half-precision operands each, in binary32.
__device__ __forceinline__ void decode8_squares(uint2 c, float (&x)[8]) {
  const uint32_t u[2] = {c.x, c.y};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    asm("{\n .reg .b16 a, b, lo, hi;\n .reg .b32 p, q;\n mov.b32 {a, b}, %4;\n"
        " cvt.rn.f16x2.e4m3x2 p, a;\n cvt.rn.f16x2.e4m3x2 q, b;\n"
        " mov.b32 {lo, hi}, p;\n fma.rn.f32.f16 %0, lo, lo, 0f00000000;\n fma.rn.f32.f16 %1, hi, hi, 0f00000000;\n"
        " mov.b32 {lo, hi}, q;\n fma.rn.f32.f16 %2, lo, lo, 0f00000000;\n fma.rn.f32.f16 %3, hi, hi, 0f00000000;\n}"
        : "=f"(x[4 * i]), "=f"(x[4 * i + 1]), "=f"(x[4 * i + 2]), "=f"(x[4 * i + 3])
        : "r"(u[i]));
  }
}
__device__ __forceinline__ float scale_value(uint32_t scale) { return __uint_as_float(scale == 0 ? 0x00400000u : scale << 23); }

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

// ---------------------------------------------------------------------------
// The step.  Every CTA walks its share of the tiles.  A producer warp brings each
// tile's arrays into a ring in shared memory by bulk copies (with the tile's
// place, its pointers and its blocks' scales beside them, whose addresses need
// not be aligned); the consumer warps update 8 elements a thread and store
// straight to global memory.  Arrays that are off a 16-byte boundary, and ends
// that do not fill one, are read by the consumers themselves.  With binary32
// moments memory bounds it: GPT-2 with binary32 weights and the BF16 copy (28
// bytes an element) takes 555 us (6.3 TB/s, 0.94 of the copy's rate), 537 of them
// between a launch's first access and its last.
// ---------------------------------------------------------------------------
template <bool LOW>
struct StepShape {
  static constexpr int kTile = adamw_tile(LOW);
  static constexpr int kConsumers = kTile / 8;       // 15 warps; with 8-bit moments 11, and two CTAs per SM
  static constexpr int kThreads = kConsumers + 32;
  static constexpr int kCtas = LOW ? 2 : 1;          // per SM
  static constexpr int kSmem = LOW ? 100 * 1024 : 200 * 1024;  // of the ring, at most
  static_assert(kTile % 256 == 0 && kTile / 128 <= 32, "whole warps; a lane of the producer per block");
};
constexpr int kStepMaxStages = 8;

// What the consumers need to know of a stage's tile.  Pointers are to its first element or block.
struct TileHead {
  const uint8_t* grad;
  uint8_t *w, *m, *v;
  uint16_t* compute;
  uint8_t *m_scale, *v_scale;
  int64_t left, goff;  // the elements from here to the tensor's end, the first one's global index
  int32_t staged[4];   // elements of w, g, m, v that are in the stage
  // 1: w, m, v, compute on 16-byte boundaries; 2: the gradient; 4: w, m, v on 32-byte ones; 8: the tile is full, all of it
  // is in the stage, and every store can be a vector's
  uint32_t flags;
  int32_t pad;
  uint8_t scales[2][32];
};

template <bool W32, bool G32, bool LOW>
struct StepRing {
  static constexpr int kW = W32 ? 4 : 2, kG = G32 ? 4 : 2, kS = LOW ? 1 : 4;
  static constexpr int kOffW = (sizeof(TileHead) + 127) / 128 * 128;
  static constexpr int kTile = StepShape<LOW>::kTile;
  static constexpr int kOffG = kOffW + kTile * kW, kOffM = kOffG + kTile * kG, kOffV = kOffM + kTile * kS;
  static constexpr int kBytes = kOffV + kTile * kS;
  static constexpr int kFit = StepShape<LOW>::kSmem / kBytes;
  static constexpr int kStages = kFit < kStepMaxStages ? kFit : kStepMaxStages;
  static_assert(kStages >= 3, "a ring of at least three tiles");
};

// 8 values of an array: from the stage where they are whole in it, else from memory.
template <bool F32>
__device__ __forceinline__ void take8(uint32_t stage, int in, int staged, const void* p, int64_t left, bool vec, float (&x)[8]) {
  if (in + 8 <= staged) {
    uint32_t a[4];
    if (F32) {
      uint32_t b[4];
      lds4(stage + in * 4, a);
      lds4(stage + in * 4 + 16, b);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = __uint_as_float(a[j]), x[4 + j] = __uint_as_float(b[j]);
    } else {
      lds4(stage + in * 2, a);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[2 * j] = bf16_lo(a[j]), x[2 * j + 1] = bf16_hi(a[j]);
    }
  } else {
    load8<F32>(p, in, left, vec, x);
  }
}
__device__ __forceinline__ uint2 take8_codes(uint32_t stage, int in, int staged, const uint8_t* p, int64_t left, bool vec) {
  if (in + 8 > staged) return load8_codes(p + in, left, vec);
  uint32_t a[2];
  lds2(stage + in, a);
  return make_uint2(a[0], a[1]);
}

// Philox4x32-10 of the step's counters {lo, hi, t}.  What the first two rounds make of t alone comes with the launch,
// so that it takes no registers: with them, fewer of the loop's values are spilled.
__device__ __forceinline__ uint4 philox_of_step(const AdamwArgs& p, uint32_t lo, uint32_t hi) {
  const uint64_t a = (uint64_t)lo * kPhiloxM0, c = (uint64_t)(p.round1[0] ^ hi) * kPhiloxM0;
  const uint64_t b = (uint64_t)((uint32_t)(a >> 32) ^ p.round1[1]) * kPhiloxM1;
  uint32_t x0 = (uint32_t)(b >> 32) ^ p.round1[2], x1 = (uint32_t)b, x2 = (uint32_t)(c >> 32) ^ (uint32_t)a ^ p.rk1[1], x3 = (uint32_t)c;
#pragma unroll
  for (int r = 2; r < kPhiloxRounds; ++r) {
    const uint64_t pa = (uint64_t)x0 * kPhiloxM0, pb = (uint64_t)x2 * kPhiloxM1;
    x0 = (uint32_t)(pb >> 32) ^ x1 ^ p.rk0[r];
    x2 = (uint32_t)(pa >> 32) ^ x3 ^ p.rk1[r];
    x1 = (uint32_t)pb, x3 = (uint32_t)pa;
  }
  return make_uint4(x0, x1, x2, x3);
}
// The 16 random bits of 8 weights, two to a word, and the 32 of 8 elements' moments (gi: the first one's global index).
__device__ __forceinline__ void weight_lanes(const AdamwArgs& p, int64_t gi, uint32_t (&r)[4]) {
  const uint64_t b = (uint64_t)gi >> 3;
  const uint4 x = philox_of_step(p, (uint32_t)b, (uint32_t)(b >> 32));
  r[0] = x.x, r[1] = x.y, r[2] = x.z, r[3] = x.w;
}
__device__ __forceinline__ void state_lanes(const AdamwArgs& p, int64_t gi, uint32_t (&r)[8]) {
  const uint64_t b = (uint64_t)gi >> 2;  // even: both blocks have the same high word
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint4 x = philox_of_step(p, (uint32_t)b + i, (uint32_t)(b >> 32) | 0x80000000u);
    r[4 * i] = x.x, r[4 * i + 1] = x.y, r[4 * i + 2] = x.z, r[4 * i + 3] = x.w;
  }
}
__device__ __forceinline__ uint32_t bf16x2_stochastic(float lo, float hi, uint32_t rnd) {
  return __byte_perm(bf16_sr_sum(lo, ~rnd & 0xFFFFu), bf16_sr_sum(hi, ~rnd >> 16), 0x7632);
}

// The canonical weight from the updated first moment and root.
__device__ __forceinline__ float new_weight(const AdamwScalars& c, float w, float m, float r) {
  const float u = __fdiv_rn(__fmul_rn(m, c.ka), __fadd_rn(__fmul_rn(r, c.c2), c.eps));
  return __fsub_rn(c.kwd != 0.0f ? __fsub_rn(w, __fmul_rn(w, c.kwd)) : w, u);
}

// ---------------------------------------------------------------------------
// The update of 8 weights with 8-bit moments, where an element has 10 bytes (with
// BF16 weights) and instructions are the bound: the same results, bit for bit,
// with little more than half of the instructions.  A 7B-width shard of 667 M
// weights, all rounded stochastically, takes 1847 us (3.6 TB/s; 2970 by the general
// code; its bytes alone would take 1003): 70 instructions an element, of which 14
// are the three Philox blocks of 8 elements and 14 packed.  Both take two issue
// slots, or the multiplier pipe for two cycles: 63 % of cycles issue, and four
// fifths of the slots are taken.
//
// Two elements at a time.  Old codes' scales go into beta1 and beta2: scales are
// powers of two and a code's square has 8 bits, so b1 (code s) = (b1 s) code and
// b2 (code s)^2 = (b2 s^2) code^2 bit for bit, for scales from 2^-47 to 2^23
// and betas of 0 or at least 2^-30, where nothing is subnormal or overflows.  Other scales, weights that are not
// finite (as where a moment is not) and second moments from 2^32 on send the warp
// to the general code (false).  Quotients are correctly rounded where the first
// moment times the rate is at least 2^-100.  A smaller one's quotient is off by
// less than 2^-99 / eps, which no weight of 2^-70 / eps or more notices: it stays
// as the decay left it.  Smaller weights beside such moments (zeros beside zeros
// among them, whose sign counts) send the warp to the general code, too.
//
// Branches around single operations (a gradient multiplier, weight decay, weights
// off the common range) stand before or after the loop over pairs, never in it, and
// call nothing.  A step over 202 M weights: 677 us, with the rounding conversions
// 631, one branch around each loop 611, no call 572, squares from half-precision
// products 566, Philox's first rounds from the launch 561.  No gain: the root's
// scaling folded into its neighbours, parts of tiles claimed by whichever warp is
// free (5 % slower), tiles of 2048 to 2560 with more registers a thread.
//
// Codes of the moments come from the rounding conversions (adamw_math.cuh).  A
// thread with a value below 2^-6 of its block's scale (about 1 in 500; zeros count)
// settles its values first.
// ---------------------------------------------------------------------------
template <bool W32, bool SR, bool STATE_SR>
__device__ __forceinline__ bool fast_update(const AdamwArgs& p, float mult, int64_t gi, int64_t left, bool vec, bool vec32,
                                            const float (&w)[8], const float (&g)[8], const float (&m0)[8],
                                            const float (&q0)[8], uint32_t km0, uint32_t kr0, const TileHead& h, int in) {
  const AdamwScalars& c = p.s;
  float m[8], r[8], x[8];
  f32x2 fin = 0;
  const float sm = scale_value(km0), sr = scale_value(kr0);
  const f32x2 b1 = both(__fmul_rn(c.b1, sm)), b2 = both(__fmul_rn(c.b2, __fmul_rn(sr, sr)));
  const f32x2 nz = p.minus_zero, mult2 = both(mult), nkwd = both(-c.kwd), nka = both(-c.ka);
  f32x2 gs[4], bs[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) gs[j] = pk(g[2 * j], g[2 * j + 1]), bs[j] = pk(w[2 * j], w[2 * j + 1]);
  if (p.grad_scale) {
#pragma unroll
    for (int j = 0; j < 4; ++j) gs[j] = mul2_rn(gs[j], mult2);
  }
  if (c.kwd != 0.0f) {
#pragma unroll
    for (int j = 0; j < 4; ++j) bs[j] = add2_rn(bs[j], prod2(bs[j], nkwd, nz));
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x2 gg = gs[j];
    const f32x2 mm = add2_rn(prod2(pk(m0[2 * j], m0[2 * j + 1]), b1, nz), prod2(gg, both(c.omb1), nz));
    const f32x2 vv = add2_rn(prod2(pk(q0[2 * j], q0[2 * j + 1]), b2, nz), prod2(mul2_rn(gg, gg), both(c.omb2), nz));
    const f32x2 rr = root2(vv);
    unpk(mm, m[2 * j], m[2 * j + 1]);
    unpk(rr, r[2 * j], r[2 * j + 1]);
    const f32x2 nd = add2_rn(prod2(rr, both(-c.c2), nz), both(-c.eps));
    const f32x2 base = bs[j];
    const f32x2 wn = add2_rn(base, quotient2(mul2_rn(mm, nka), nd));
    fin = fma2_rn(wn, 0ull, fin);
    unpk(wn, x[2 * j], x[2 * j + 1]);
  }
  // Both blocks' exponents from the 16 lanes' maxima, as 16-bit halves of a word: 0 where all are 0, else k + 135.
  float am = 0.0f, ar = 0.0f, lm = __uint_as_float(0x7F800000u), lr = lm;
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    am = fmaxf(fmaxf(am, fabsf(m[j])), fabsf(m[j + 1]));
    ar = fmaxf(fmaxf(ar, r[j]), r[j + 1]);
    lm = fminf(fminf(lm, fabsf(m[j])), fabsf(m[j + 1]));
    lr = fminf(fminf(lr, r[j]), r[j + 1]);
  }
  bool odd = cert_not_finite(fin) || min(km0, kr0) < 80u || max(km0, kr0) > 150u;
  if (__fmul_rn(lm, c.ka) < 0x1p-100f) {
    float lx = fabsf(x[0]);
#pragma unroll
    for (int j = 1; j < 8; ++j) lx = fminf(lx, fabsf(x[j]));
    odd |= __fmul_rn(lx, c.eps) < 0x1p-70f;
  }
  if (__any_sync(~0u, odd)) return false;
  uint32_t u[4];
  if (!W32 && SR) {
    uint32_t rnd[4];
    weight_lanes(p, gi, rnd);
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = rs_bf16x2(x[2 * j], x[2 * j + 1], ~rnd[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = bf16x2_rn(x[2 * j], x[2 * j + 1]);
  }
  if (W32) {
    store8_f32(h.w, in, left, vec, vec32, x);
    if (h.compute) store8_bf16(h.compute, in, left, vec, u);
  } else {
    store8_bf16(h.w, in, left, vec, u);
  }

  uint32_t lanes[8] = {};
  if (STATE_SR) state_lanes(p, gi, lanes);
  auto biased = [](float a) { return a == 0.0f ? 0u : max(8u, (__float_as_uint(a) + 0x1FFFFFu) >> 23); };
  uint32_t k2 = biased(am) | biased(ar) << 16;
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) k2 = __vmaxu2(k2, __shfl_xor_sync(~0u, k2, d));
  const int km = (k2 & 0xFFFFu) ? (int)(k2 & 0xFFFFu) - 135 : 0, kr = k2 >> 16 ? (int)(k2 >> 16) - 135 : 0;
  const float im = __uint_as_float((uint32_t)(127 - km) << 23), ir = __uint_as_float((uint32_t)(127 - kr) << 23);
  const bool small = STATE_SR ? fminf(__fmul_rn(lm, im), __fmul_rn(lr, ir)) < 0x1p-6f : __fmul_rn(lr, ir) < 0x1p-9f;
  float y[8], z[8];
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    unpk(mul2_rn(pk(m[j], m[j + 1]), both(im)), y[j], y[j + 1]);
    unpk(mul2_rn(pk(r[j], r[j + 1]), both(ir)), z[j], z[j + 1]);
  }
  if (small) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (STATE_SR) y[j] = settle(y[j]), z[j] = settle(z[j]);
      if (r[j] > 0.0f) z[j] = fmaxf(z[j], 0x1p-9f);  // never stored as 0
    }
  }
  uint32_t a[4], b[4];  // two codes each, in the low bytes (of b, with stochastic rounding, the high ones)
  constexpr uint32_t kHalves = STATE_SR ? 0x7632 : 0x5410;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (STATE_SR) {
      a[j] = b[j] = __byte_perm(rs_codes(y[2 * j], z[2 * j], lanes[2 * j]), rs_codes(y[2 * j + 1], z[2 * j + 1], lanes[2 * j + 1]),
                                0x6240);
    } else {
      a[j] = e4m3x2(y[2 * j], y[2 * j + 1]);
      b[j] = e4m3x2(z[2 * j], z[2 * j + 1]);
    }
  }
  store8_codes(h.m + in, left, vec, make_uint2(__byte_perm(a[0], a[1], 0x5410), __byte_perm(a[2], a[3], 0x5410)));
  store8_codes(h.v + in, left, vec, make_uint2(__byte_perm(b[0], b[1], kHalves), __byte_perm(b[2], b[3], kHalves)));
  if ((threadIdx.x & 15) == 0 && left > 0) {
    h.m_scale[threadIdx.x >> 4] = (uint8_t)(km + 127);
    h.v_scale[threadIdx.x >> 4] = (uint8_t)(kr + 127);
  }
  return true;
}

template <bool W32, bool G32, bool LOW, bool SR, bool STATE_SR>
__global__ void __launch_bounds__(StepShape<LOW>::kThreads, StepShape<LOW>::kCtas)
    adamw_kernel(const __grid_constant__ AdamwArgs p) {
  using R = StepRing<W32, G32, LOW>;
  constexpr int kTile = StepShape<LOW>::kTile, kConsumers = StepShape<LOW>::kConsumers;
  extern __shared__ uint8_t smem_raw[];
  __shared__ alignas(8) uint64_t bars[2 * R::kStages];
  const uint32_t smem = (smem_addr(smem_raw) + 127u) & ~127u;
  uint8_t* ring = smem_raw + (smem - smem_addr(smem_raw));
  const uint32_t bar0 = smem_addr(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (R::kStages + s); };
  if (threadIdx.x == 0) {
    for (int s = 0; s < R::kStages; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), kConsumers / 32);
    }
    mbar_init_fence();
  }
  __syncthreads();
  wait_for_earlier_kernels();
  float mult = 1.0f;
  if (p.grad_scale) {
    mult = *p.grad_scale;
    if (mult != mult) return;  // the norm was not finite: the step is skipped
  }
  // Every gridDim.x-th tile: the CTAs walk the list side by side.
  const int64_t count = (p.tiles - blockIdx.x + gridDim.x - 1) / gridDim.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (warp == kConsumers / 32) {
    // Each lane looks up one of the next 32 tiles, so that the chain of loads (the tile's tensor, its pointers, its
    // gradient) is waited for once in 32 tiles, and half of those early.
    struct Place {
      const uint8_t* grad;
      uint8_t *w, *m, *v, *ms, *vs;
      uint16_t* compute;
      int64_t at, left, goff;
      uint32_t vec;
    };
    auto look_up = [&](int64_t i) {
      Place x{};
      if (i < count) {
        const int64_t t = blockIdx.x + i * gridDim.x;
        const int k = p.tile_tensor[t];
        const ListTensor d = p.tensors[k];
        x.grad = static_cast<const uint8_t*>(grad_of(p.g, k));
        x.w = static_cast<uint8_t*>(d.w), x.m = static_cast<uint8_t*>(d.m), x.v = static_cast<uint8_t*>(d.v);
        x.ms = d.m_scale, x.vs = d.v_scale, x.compute = d.compute;
        x.at = (t - d.tile0) * kTile, x.left = d.numel - x.at, x.goff = d.goff;
        x.vec = d.aligned | ((reinterpret_cast<uintptr_t>(x.grad) & 15) == 0 ? 2u : 0u);
      }
      return x;
    };
    const uint64_t policy = evict_first_policy();
    Place mine = look_up(lane), next{};
    int s = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int64_t i = 0; i < count; ++i) {
      const int owner = (int)(i & 31);
      if (owner == 16) next = look_up(i + 16 + lane);
      if (owner == 0 && i > 0) mine = next;
      uint32_t ms = 127, vs = 127;
      if (LOW) {
        const int blocks = __shfl_sync(~0u, (int)((min(mine.left, (int64_t)kTile) + 127) / 128), owner);
        const uint64_t mp = __shfl_sync(~0u, reinterpret_cast<uint64_t>(mine.ms + mine.at / 128), owner);
        const uint64_t vp = __shfl_sync(~0u, reinterpret_cast<uint64_t>(mine.vs + mine.at / 128), owner);
        if (lane < blocks) {
          ms = reinterpret_cast<const uint8_t*>(mp)[lane];
          vs = reinterpret_cast<const uint8_t*>(vp)[lane];
        }
      }
      if (!warp_wait(empty(s), phase ^ 1)) { ok = false; break; }
      TileHead& h = *reinterpret_cast<TileHead*>(ring + s * R::kBytes);
      if (LOW) {
        h.scales[0][lane] = (uint8_t)ms;
        h.scales[1][lane] = (uint8_t)vs;
      }
      __syncwarp();
      if (lane == owner) {
        const Place& d = mine;
        const int n = (int)min((int64_t)kTile, d.left);
        auto whole = [&](const void* q, int size) { return (reinterpret_cast<uintptr_t>(q) & 15) ? 0 : n * size / 16 * 16; };
        const uint8_t *w = d.w + d.at * R::kW, *g = d.grad + d.at * R::kG, *m = d.m + d.at * R::kS, *v = d.v + d.at * R::kS;
        const int bw = whole(w, R::kW), bg = whole(g, R::kG), bm = whole(m, R::kS), bv = whole(v, R::kS);
        h.grad = g;
        h.w = const_cast<uint8_t*>(w), h.m = const_cast<uint8_t*>(m), h.v = const_cast<uint8_t*>(v);
        h.compute = d.compute ? d.compute + d.at : nullptr;
        h.m_scale = d.ms + d.at / 128, h.v_scale = d.vs + d.at / 128;
        h.left = d.left, h.goff = d.goff + d.at;
        h.staged[0] = bw / R::kW, h.staged[1] = bg / R::kG, h.staged[2] = bm / R::kS, h.staged[3] = bv / R::kS;
        const bool full_tile = n == kTile && bw == kTile * R::kW && bg == kTile * R::kG && bm == kTile * R::kS && bv == kTile * R::kS;
        h.flags = d.vec | (full_tile && (d.vec & 3) == 3 && (!W32 || (d.vec & 4)) ? 8u : 0u);
        const uint32_t st = smem + s * R::kBytes;
        mbar_expect_tx(full(s), bw + bg + bm + bv);
        if (bw) tma_load(st + R::kOffW, w, bw, full(s), policy);
        if (bg) tma_load(st + R::kOffG, g, bg, full(s), policy);
        if (bm) tma_load(st + R::kOffM, m, bm, full(s), policy);
        if (bv) tma_load(st + R::kOffV, v, bv, full(s), policy);
        mbar_arrive(full(s));
      }
      __syncwarp();
      if (++s == R::kStages) { s = 0; phase ^= 1; }
    }
    if (!ok) {
      if (lane == 0) atomicOr(p.err, 1);
      // the copies in flight, before the block's memory goes (a stage that was never filled has nothing in flight)
      for (int i = 0; i < R::kStages && i < count; ++i) {
        if (s == 0) { s = R::kStages; phase ^= 1; }
        --s;
        mbar_wait(full(s), phase);
      }
    }
    return;
  }

  const AdamwScalars& c = p.s;
  const int in = threadIdx.x * 8;
  int s = 0;
  uint32_t phase = 0;
  const int n32 = (int)count;
  for (int i = 0; i < n32; ++i) {
    if (!warp_wait(full(s), phase)) {
      if (lane == 0) atomicOr(p.err, 2);
      // the copies in flight, before the block's memory goes: the producer may be done, with every stage filled
      for (int n = min(n32 - i, R::kStages); n > 0; --n) {
        warp_wait(full(s), phase);
        if (++s == R::kStages) { s = 0; phase ^= 1; }
      }
      return;
    }
    const TileHead& h = *reinterpret_cast<const TileHead*>(ring + s * R::kBytes);
    const uint32_t st = smem + s * R::kBytes;
    const int64_t left = h.left - in;
    if (warp * 256 >= h.left) {  // nothing of the tile for this warp
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(s));
      if (++s == R::kStages) { s = 0; phase ^= 1; }
      continue;
    }
    const uint32_t flags = h.flags;
    const bool vec = flags & 1, gvec = flags & 2, vec32 = flags & 4;
    const int64_t gi = h.goff + in;
    uint32_t km0 = 127, kr0 = 127;
    float w[8], g[8], m[8], v[8];
    auto take_all = [&](const int (&staged)[4], bool squares) {  // (squares: v as its codes' squares)
      take8<G32>(st + R::kOffG, in, staged[1], h.grad, left, gvec, g);
      take8<W32>(st + R::kOffW, in, staged[0], h.w, left, vec, w);
      if (LOW) {
        decode8(take8_codes(st + R::kOffM, in, staged[2], h.m, left, vec), m);
        const uint2 codes = take8_codes(st + R::kOffV, in, staged[3], h.v, left, vec);
        if (squares) decode8_squares(codes, v);
        else decode8(codes, v);
        km0 = h.scales[0][threadIdx.x >> 4];
        kr0 = h.scales[1][threadIdx.x >> 4];
      } else {
        take8<true>(st + R::kOffM, in, staged[2], h.m, left, vec, m);
        take8<true>(st + R::kOffV, in, staged[3], h.v, left, vec, v);
      }
    };
    // With 8-bit moments the stage is kept to the end: what is needed again is read from it again, not kept in registers.
    auto release = [&] {
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(s));
      if (++s == R::kStages) { s = 0; phase ^= 1; }
    };
    if constexpr (LOW) {
      if (p.plain) {
        bool done;
        if (flags & 8) {  // no look at the tile's end or at alignments
          constexpr int kAll[4] = {1 << 30, 1 << 30, 1 << 30, 1 << 30};
          take_all(kAll, true);
          done = fast_update<W32, SR, STATE_SR>(p, mult, gi, 8, true, true, w, g, m, v, km0, kr0, h, in);
        } else {
          take_all(h.staged, true);
          done = fast_update<W32, SR, STATE_SR>(p, mult, gi, left, vec, vec32, w, g, m, v, km0, kr0, h, in);
        }
        if (done) {
          release();
          continue;
        }
      }
    }
    take_all(h.staged, false);
    uint8_t *const hw = h.w, *const hm = h.m, *const hv = h.v, *const ms = h.m_scale, *const vs = h.v_scale;
    uint16_t* const compute = h.compute;
    if constexpr (!LOW) release();
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (LOW) {
        m[j] = __fmul_rn(m[j], scale_value(km0));
        v[j] = __fmul_rn(v[j], scale_value(kr0));
        v[j] = __fmul_rn(v[j], v[j]);
      }
      const float gs = p.grad_scale ? __fmul_rn(g[j], mult) : g[j];
      m[j] = __fadd_rn(__fmul_rn(m[j], c.b1), __fmul_rn(gs, c.omb1));
      v[j] = __fadd_rn(__fmul_rn(v[j], c.b2), __fmul_rn(__fmul_rn(gs, gs), c.omb2));
      r[j] = __fsqrt_rn(v[j]);
      w[j] = new_weight(c, w[j], m[j], r[j]);
    }
    if (LOW) {
      uint32_t lanes[8] = {};
      if (STATE_SR) state_lanes(p, gi, lanes);
      const int km = block_exponent(m), kv = block_exponent(r);
      store8_codes(hm + in, left, vec, encode8<STATE_SR, false>(m, km, lanes, 0));
      store8_codes(hv + in, left, vec, encode8<STATE_SR, true>(r, kv, lanes, 16));
      if ((threadIdx.x & 15) == 0 && left > 0) {
        ms[threadIdx.x >> 4] = (uint8_t)(km + 127);
        vs[threadIdx.x >> 4] = (uint8_t)(kv + 127);
      }
    } else {
      store8_f32(hm, in, left, vec, vec32, m);
      store8_f32(hv, in, left, vec, vec32, v);
    }
    if (W32) store8_f32(hw, in, left, vec, vec32, w);
    if (!W32 || compute) {
      uint32_t u[4];
      if (!W32 && SR) {
        uint32_t rnd[4];
        weight_lanes(p, gi, rnd);
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = bf16x2_stochastic(w[2 * j], w[2 * j + 1], rnd[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = bf16x2_rn(w[2 * j], w[2 * j + 1]);
      }
      if (!W32) store8_bf16(hw, in, left, vec, u);
      else store8_bf16(compute, in, left, vec, u);
    }
    if constexpr (LOW) release();
  }
}

// ---------------------------------------------------------------------------
// The norm.  Each warp walks a run of tiles of 2048 elements, all of a tile's
// loads in flight at once, and adds a tile's squares in eight binary32 sums a
// thread, eight to each; these meet in binary64, with a partial sum per CTA, which
// the CTA that comes last adds up in order.  (Over a whole run in binary32, small
// squares of BF16 lost more to rounding than they gained: a norm over 4.3 10^9
// gradients came out 2 10^-6 too small.)  The runs depend on the list alone, so the
// result's bits do.
// Memory bounds it: 405 M BF16 gradients take 120 us (6.8 TB/s, 1.01 of the copy's
// rate; by CTAs of 2048 elements in turn, a chain of loads each, 234), 4000 ragged
// tensors of 86 M 33 (5.2 TB/s) behind 46 of the caller's look at them.
// ---------------------------------------------------------------------------
constexpr int kNormThreads = 256;
constexpr int kNormWarps = kNormThreads / 32;

template <bool G32>
__global__ void __launch_bounds__(kNormThreads, 5) grad_norm_kernel(const __grid_constant__ NormArgs p) {
  __shared__ double part[kNormWarps];
  __shared__ bool last;
  wait_for_earlier_kernels();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t walker = (int64_t)blockIdx.x * kNormWarps + warp, walkers = (int64_t)gridDim.x * kNormWarps;
  const int64_t t0 = p.tiles * walker / walkers, t1 = p.tiles * (walker + 1) / walkers;
  double sum = 0.0;
  constexpr int kSize = G32 ? 4 : 2, kPer = 16 / kSize, kRow = 32 * kPer, kLoads = kNormTile / kRow;
  for (int64_t base = t0; base < t1; base += 32) {
    // Each lane looks up one of the next 32 tiles: where it starts, and how many elements it has.
    const uint8_t* at = nullptr;
    int elements = 0;
    if (base + lane < t1) {
      const int k = p.tile_tensor[base + lane];
      const int64_t first = (base + lane - p.tensors[k].tile0) * kNormTile;
      at = static_cast<const uint8_t*>(grad_of(p.g, k)) + first * kSize;
      elements = (int)min((int64_t)kNormTile, p.tensors[k].numel - first);
    }
    const int here = (int)min((int64_t)32, t1 - base);
    for (int i = 0; i < here; ++i) {
      const uint8_t* q = reinterpret_cast<const uint8_t*>(__shfl_sync(~0u, reinterpret_cast<uint64_t>(at), i));
      const int n = __shfl_sync(~0u, elements, i);
      const bool vec = (reinterpret_cast<uintptr_t>(q) & 15) == 0;
      float acc[8] = {};
      // The squares of a lane's vector r.
      auto add = [&](const uint4& x, int r) {
        const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (G32) {
            const float a = __uint_as_float(u[j]);
            acc[4 * (r & 1) + j] = __fmaf_rn(a, a, acc[4 * (r & 1) + j]);
          } else {
            const float a = bf16_lo(u[j]), b = bf16_hi(u[j]);
            acc[2 * j] = __fmaf_rn(a, a, acc[2 * j]);
            acc[2 * j + 1] = __fmaf_rn(b, b, acc[2 * j + 1]);
          }
        }
      };
      if (vec && n == kNormTile) {
        uint4 x[kLoads];
#pragma unroll
        for (int r = 0; r < kLoads; ++r) x[r] = __ldcs(reinterpret_cast<const uint4*>(q) + r * 32 + lane);
#pragma unroll
        for (int r = 0; r < kLoads; ++r) add(x[r], r);
      } else {
        // The same elements in the same sums, whether they can be read in vectors or not: no alignment changes a bit.
#pragma unroll 1
        for (int r0 = 0; r0 * kRow < n; r0 += 4) {
          uint4 x[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int e = (r0 + r) * kRow + lane * kPer;
            uint32_t u[4] = {0, 0, 0, 0};
            if (vec && e + kPer <= n) {
              const uint4 y = __ldcs(reinterpret_cast<const uint4*>(q + e * kSize));
              u[0] = y.x, u[1] = y.y, u[2] = y.z, u[3] = y.w;
            } else if (e < n) {
#pragma unroll
              for (int j = 0; j < kPer; ++j)
                if (e + j < n) {
                  if (G32) u[j] = reinterpret_cast<const uint32_t*>(q)[e + j];
                  else u[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(q)[e + j] << (16 * (j & 1));
                }
            }
            x[r] = make_uint4(u[0], u[1], u[2], u[3]);
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) add(x[r], r);
        }
      }
      sum += (double)__fadd_rn(__fadd_rn(__fadd_rn(acc[0], acc[1]), __fadd_rn(acc[2], acc[3])),
                               __fadd_rn(__fadd_rn(acc[4], acc[5]), __fadd_rn(acc[6], acc[7])));
    }
  }
  auto block_sum = [&](double x) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    __syncthreads();
    if (lane == 0) part[warp] = x;
    __syncthreads();
    x = 0.0;
    for (int w = 0; w < kNormWarps; ++w) x += part[w];
    return x;
  };
  const double mine = block_sum(sum);
  if (threadIdx.x == 0) {
    p.partial[blockIdx.x] = mine;
    __threadfence();
    last = atomicAdd(p.done, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!last) return;
  __threadfence();
  double x = 0.0;
  for (int i = threadIdx.x; i < (int)gridDim.x; i += kNormThreads) x += __ldcg(p.partial + i);
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

struct StepKernel {
  const void* f;
  int smem, threads, ctas;
};
template <bool W32, bool G32, bool LOW>
StepKernel pick(bool sr, bool state_sr) {
  if (W32) sr = false;
  if (!LOW) state_sr = false;
  using R = StepRing<W32, G32, LOW>;
  const void* f = sr ? (state_sr ? (const void*)adamw_kernel<W32, G32, LOW, !W32, LOW> : (const void*)adamw_kernel<W32, G32, LOW, !W32, false>)
                     : (state_sr ? (const void*)adamw_kernel<W32, G32, LOW, false, LOW> : (const void*)adamw_kernel<W32, G32, LOW, false, false>);
  return {f, R::kStages * R::kBytes + 128, StepShape<LOW>::kThreads, StepShape<LOW>::kCtas};
}
template <bool W32, bool G32>
StepKernel pick(const AdamwKind& k) {
  return k.state_e4m3 ? pick<W32, G32, true>(k.sr, k.state_sr) : pick<W32, G32, false>(k.sr, k.state_sr);
}
StepKernel pick(const AdamwKind& k) {
  return k.w_f32 ? (k.g_f32 ? pick<true, true>(k) : pick<true, false>(k)) : (k.g_f32 ? pick<false, true>(k) : pick<false, false>(k));
}

}  // namespace

cudaError_t prepare_adamw(const AdamwKind& k, int32_t* sms) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev);
  const StepKernel kernel = pick(k);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel.f, cudaFuncAttributeMaxDynamicSharedMemorySize, kernel.smem);
  return e;
}

cudaError_t launch_adamw(const AdamwArgs& a, const AdamwKind& k, int32_t sms, cudaStream_t stream) {
  const StepKernel kernel = pick(k);
  const int64_t most = (int64_t)sms * kernel.ctas;
  const unsigned grid = (unsigned)(a.tiles < most ? a.tiles : most);
  return launch_dependent(kernel.f, grid, (unsigned)kernel.threads, 0, kernel.smem, &a, stream);
}

cudaError_t launch_grad_norm(const NormArgs& a, cudaStream_t stream) {
  const int64_t wanted = (a.tiles + kNormWarps - 1) / kNormWarps;
  const unsigned grid = (unsigned)(wanted < 1 ? 1 : wanted < kNormCtas ? wanted : kNormCtas);
  return launch_dependent(a.g_f32 ? (const void*)grad_norm_kernel<true> : (const void*)grad_norm_kernel<false>, grid, kNormThreads,
                          0, 0, &a, stream);
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
