// muon_products.cu -- the three products of a Newton-Schulz step (muon.h) over a
// list of matrices, one launch each:
//   A = X X^T,   B = a I + b A + c A A,   X <- B X
// of X's first part; a times its second part is added to the last.  A and B are
// symmetric: their tiles on and below the diagonal are computed and stored in
// both places.
#include <algorithm>
#include <atomic>

#include "launch.h"
#include "muon.h"
#include "tcgen05.cuh"

namespace mpadam {

namespace {

constexpr int kPairs = 76;      // GB300: two SMs each
constexpr int kStepK = 64;      // values of k per stage: a row of one 128-byte swizzle atom
constexpr int kStages = 6;
constexpr int kBoxBytes = 64 * 64 * 2;
constexpr int kStageBytes = 4 * kBoxBytes;  // 128 rows of either operand
constexpr int kDynSmem = kStages * kStageBytes + 1024;
constexpr uint32_t kStageTx = 2 * kStageBytes;  // of both CTAs
constexpr int kEpiWarps = 8;
constexpr int kProductThreads = 32 * (4 + kEpiWarps);  // a producer and an issuing warp (and two idle ones), then the epilogue

enum ProductError : int32_t { kErrCopy = 1, kErrStage = 2, kErrAcc = 4 };

// The steps' coefficients (K. Jordan et al., "Muon: An optimizer for hidden layers in neural networks", 2024).
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;

// An operand whose rows run along m (or n) instead of k: chunks of 64 of them 8192 bytes apart, groups of 8 values of k 1024.
__device__ __forceinline__ uint32_t desc_low_mn(uint32_t addr) { return addr >> 4 | (uint32_t)(kBoxBytes >> 4) << 16; }

__device__ __forceinline__ void pair_mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}

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

// WHICH: 1, 2, 3, the product.  A tile is [256 rows m, 256 columns n] of
//   1: X X^T, 2: A A, 3: X^T B (B is symmetric: the transpose of B X, whose rows then run along the lanes)
// Lane m of a warp holds column by column n: stores of a column go to 32
// neighbouring elements of the row n of the result (of the transposed place in a
// symmetric one).
template <int WHICH>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1) product_kernel(const __grid_constant__ ProductArgs p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ alignas(8) uint64_t bars[2 * kStages + 5];
  __shared__ uint32_t tmem_base_s;
  __shared__ int32_t failed;
  const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const uint32_t bar0 = smem_addr(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };               // the leader's alone
  auto empty = [&](int s) { return bar0 + 8u * (kStages + s); };  // each CTA's own
  auto acc_full = [&](int a) { return bar0 + 8u * (2 * kStages + a); };
  auto acc_free = [&](int a) { return bar0 + 8u * (2 * kStages + 2 + a); };
  const uint32_t drained = bar0 + 8u * (2 * kStages + 4);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(acc_full(a), 1);
      mbar_init(acc_free(a), 2 * kEpiWarps);
    }
    mbar_init(drained, 1);
    failed = 0;
    mbar_init_fence();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base_s)), "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  wait_for_earlier_kernels();

  const int pairs = gridDim.x / 2;
  volatile int32_t* stop = &failed;
  auto steps_of = [&](const NewtonTile& t) {
    const NewtonMatrix& q = p.matrices[t.matrix];
    return ((WHICH == 1 ? q.c : q.r) + kStepK - 1) / kStepK;
  };

  if (warp == 0) {
    if (lane == 0) {
      int s = 0, issued = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int i = blockIdx.x / 2; i < p.count && ok; i += pairs) {
        if (*stop) { ok = false; break; }
        const NewtonTile t = p.tiles[i];
        const NewtonMatrix& q = p.matrices[t.matrix];
        const CUtensorMap* first = WHICH == 2 ? &q.a : &q.x[p.from];
        const CUtensorMap* second = WHICH == 1 ? &q.x[p.from] : WHICH == 2 ? &q.a : &q.b;
        const int m0 = t.tm * kNewtonTile + (int)rank * 128, n0 = t.tn * kNewtonTile + (int)rank * 128, steps = steps_of(t);
        for (int k = 0; k < steps; ++k) {
          if (!mbar_wait(empty(s), phase ^ 1)) { ok = false; break; }
          const uint32_t st = smem + s * kStageBytes, bar = peer_addr(full(s), 0);
          if (rank == 0) mbar_arrive_tx(full(s), kStageTx);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (WHICH == 3) pair_load_2d(st + h * kBoxBytes, first, m0 + 64 * h, k * kStepK, bar);
            else pair_load_2d(st + h * kBoxBytes, first, k * kStepK, m0 + 64 * h, bar);
            pair_load_2d(st + (2 + h) * kBoxBytes, second, k * kStepK, n0 + 64 * h, bar);
          }
          ++issued;
          if (++s == kStages) { s = 0; phase ^= 1; }
        }
      }
      if (!ok) {
        *stop = 1;
        atomicOr(p.err, kErrStage);
        // the copies in flight: the leader sees both CTAs' last stages arrive, the other one waits for it in the end
        for (int i = 0; i < min(issued, kStages); ++i) {
          if (s == 0) { s = kStages; phase ^= 1; }
          --s;
          if (rank == 0) mbar_wait(full(s), phase);
        }
      }
    }
  } else if (warp == 1 && rank == 0) {
    const bool issue = elected();
    // FP16 operands, binary32 sums, 256 x 256; product 3's first operand runs along m
    constexpr uint32_t id = 1u << 4 | (WHICH == 3 ? 1u << 15 : 0u) | (uint32_t)(kNewtonTile >> 3) << 17 | (uint32_t)(kNewtonTile >> 4) << 24;
    int s = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    int i = blockIdx.x / 2, at = -1;  // the tile, and its step whose operands were given up
    for (; i < p.count; i += pairs) {
      const int steps = steps_of(p.tiles[i]);
      if (!warp_wait_cluster(acc_free(acc), acc_phase ^ 1)) { at = 0; break; }
      tc_fence_after();
      const uint32_t d = tmem + acc * kNewtonTile;
      for (int k = 0; k < steps; ++k) {
        if (!warp_wait(full(s), phase)) { at = k; break; }
        tc_fence_after();
        if (issue) {
          const uint32_t st = smem + s * kStageBytes;
          const uint32_t first = WHICH == 3 ? desc_low_mn(st) : desc_low(st), second = desc_low(st + 2 * kBoxBytes);
          constexpr uint32_t kAdvance = WHICH == 3 ? 2048 >> 4 : 32 >> 4;  // 16 values of k
#pragma unroll
          for (int j = 0; j < kStepK / 16; ++j)
            pair_mma_f16(d, desc(first + kAdvance * j, kOperandHigh), desc(second + 2 * j, kOperandHigh), id, j > 0 || k > 0);
          pair_commit(empty(s));
        }
        if (++s == kStages) { s = 0; phase ^= 1; }
      }
      if (at >= 0) break;
      if (issue) pair_commit(acc_full(acc));
      if (++acc == 2) { acc = 0; acc_phase ^= 1; }
    }
    if (at >= 0) {
      // The products in flight, then both CTAs' copies that are still to come (the producers fill every stage again, unless
      // they have seen the stop), before their memory goes; then the epilogue is woken up to find that it has nothing to store.
      if (issue) {
        atomicOr(p.err, kErrCopy);
        pair_commit(drained);
      }
      warp_wait(drained, 0);
      int64_t left = -at;
      for (int t = i; t < p.count && left < kStages; t += pairs) left += steps_of(p.tiles[t]);
      for (int n = 0; n < (int)min(left, (int64_t)kStages); ++n) {
        warp_wait(full(s), phase);
        if (++s == kStages) { s = 0; phase ^= 1; }
      }
      if (issue) {
        for (uint32_t r = 0; r < 2; ++r) {
          sts_cluster(peer_addr(smem_addr(&failed), r), 1);
          mbar_arrive_cluster(peer_addr(acc_full(acc), r));
        }
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, half = (warp - 4) >> 2;
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int i = blockIdx.x / 2; i < p.count; i += pairs) {
      const NewtonTile t = p.tiles[i];
      const NewtonMatrix& q = p.matrices[t.matrix];
      const int m = t.tm * kNewtonTile + (int)rank * 128 + quarter * 32 + lane, n0 = t.tn * kNewtonTile + half * 128;
      const int rows = q.r, last_m = WHICH == 3 ? q.c : q.r;
      const int64_t ld = WHICH == 3 ? q.ld : q.lda;
      // What is added to the sums, X's second part or A, a column of the tile at a time: fetched ahead, whatever is in the
      // way of the stores.
      const uint16_t* addend = WHICH == 3 ? q.lo : q.ga;
      const bool adds = WHICH == 2 || (WHICH == 3 && p.use_lo);
      uint16_t ahead[32];
      auto fetch = [&](int c) {
        const uint16_t* from = addend + (int64_t)(n0 + c) * ld + m;
#pragma unroll
        for (int j = 0; j < 32; ++j) ahead[j] = adds && m < last_m && n0 + c + j < rows ? from[j * ld] : (uint16_t)0;
      };
      if (WHICH != 1) fetch(0);
      if (!warp_wait_cluster(acc_full(acc), acc_phase) || *stop) {
        if (lane == 0) { atomicOr(p.err, kErrAcc); *stop = 1; }
        break;
      }
      tc_fence_after();
      const uint32_t from = tmem + acc * kNewtonTile + half * 128 + ((uint32_t)(quarter * 32) << 16);
#pragma unroll 1
      for (int c = 0; c < 128; c += 32) {
        uint32_t r[32];
        uint16_t add[32];
        __syncwarp();
        tmem_load32(from + c, r);
        if (WHICH != 1) {
#pragma unroll
          for (int j = 0; j < 32; ++j) add[j] = ahead[j];
          if (c + 32 < 128) fetch(c + 32);
        }
        tmem_wait_load();
        const int n = n0 + c, here = min(32, rows - n);  // columns of the tile: rows of the result
        if (here <= 0 || m >= last_m) continue;
        const int64_t at = (int64_t)n * ld + m;
        if (WHICH == 3) {
          uint16_t *hi = q.hi[p.from ^ 1] + at, *lo = q.lo + at;
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            if (j >= here) break;
            const float y = __fmaf_rn(kA, of_half(add[j]), __fmul_rn(__uint_as_float(r[j]), kFromHeld));
            const uint16_t h = half_of(y);
            hi[j * ld] = h;
            if (p.keep_lo) lo[j * ld] = half_of(__fsub_rn(y, of_half(h)));
          }
        } else {
          uint16_t* out = WHICH == 1 ? q.ga : q.gb;
          uint16_t h[32];
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            float y = __fmul_rn(__uint_as_float(r[j]), kFromHeld);
            if (WHICH == 2) {
              y = __fmaf_rn(kC, y, __fmul_rn(kB, of_half(add[j])));
              if (n + j == m) y = __fadd_rn(y, kA * kHeld);
            }
            h[j] = half_of(y);
            if (j < here) out[at + j * ld] = h[j];
          }
          if (t.tm != t.tn) {  // (the row's padding has room for whole vectors)
            uint4* row = reinterpret_cast<uint4*>(out + (int64_t)m * ld + n);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              if (8 * j >= here) break;
              uint32_t u[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) u[k] = h[8 * j + 2 * k] | (uint32_t)h[8 * j + 2 * k + 1] << 16;
              row[j] = make_uint4(u[0], u[1], u[2], u[3]);
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(peer_addr(acc_free(acc), 0));
      if (++acc == 2) { acc = 0; acc_phase ^= 1; }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

template <int WHICH>
cudaError_t launch(const ProductArgs& a, cudaStream_t stream) {
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem((const void*)product_kernel<WHICH>, kDynSmem, ready);
  if (e != cudaSuccess) return e;
  return launch_dependent((const void*)product_kernel<WHICH>, 2 * (unsigned)std::min(a.count, kPairs), kProductThreads, 0, kDynSmem, &a,
                          stream);
}

}  // namespace

cudaError_t launch_product(int which, const ProductArgs& a, cudaStream_t stream) {
  return which == 1 ? launch<1>(a, stream) : which == 2 ? launch<2>(a, stream) : launch<3>(a, stream);
}

}  // namespace mpadam
