// fp8_matmul.cu -- D[m, n] (+)= A[m, k] B[n, k]^T for E4M3 matrices with a
// power-of-two scale per block of 128 along k:
//   D_ij = sum over blocks c of 2^(ea_ic + eb_jc) sum over k in c of A_ik B_jk.
// The tensor cores apply the scales themselves (block-scaled tcgen05.mma: one
// E8M0 scale per row and 32 values of k, four such steps sharing a block's
// scale) and accumulate in binary32.
//
// Layout of a tile.  The rows of b lie along the 128 lanes of tensor memory and
// the rows of a along its columns, so that a warp that reads a column holds 32
// neighbouring elements of a row of D and stores them straight from registers.
// It also makes the a side the one whose tile may be small: a single token is a
// tile of 16 columns and no tensor work is spent on rows that are not there.
#include <algorithm>
#include <atomic>

#include "fp8.h"
#include "launch.h"
#include "step_kernel.cuh"

namespace mpadam {

namespace {

constexpr int kTileN = 128;   // rows of b per tile (lanes of tensor memory)
constexpr int kTileK = 128;   // values of k per stage (bytes of a row: one 128-byte swizzle atom)
constexpr int kSms = 152;      // GB300
constexpr int kEpiWarps = 8;
constexpr int kMatmulThreads = 32 * (4 + kEpiWarps);  // a producer and an issuing warp (and two idle ones), then the epilogue

enum MatmulError : int32_t { kErrCopy = 1, kErrStage = 2, kErrAcc = 4 };

__device__ int32_t g_matmul_error;

template <int TM>
struct Shape {
  static constexpr int kScaleTilesA = (TM + 127) / 128;
  static constexpr int kScaleBytes = kScaleTile * (1 + kScaleTilesA);
  static constexpr int kStageBytes = (kTileN + TM) * kTileK + 1024;  // codes, then scales; keeps 1024-byte alignment
  static constexpr int kStages = TM >= 128 ? 3 : TM >= 64 ? 4 : 5;   // two CTAs an SM
  // Tensor memory: the accumulator, then two sets of scales (4 columns for b, 4 for a).
  static constexpr int kScaleCols = 4 + 4 * kScaleTilesA;
  static constexpr int kUsedCols = TM + 2 * kScaleCols;
  static constexpr int kCols = kUsedCols <= 32 ? 32 : kUsedCols <= 64 ? 64 : kUsedCols <= 128 ? 128 : 256;
  static constexpr int kDynSmem = kStages * kStageBytes + 1024;
  static_assert(kScaleBytes <= 1024 && TM * kTileN * 4 <= kStages * kStageBytes, "scales and partial sums fit");
};

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void mbar_arrive_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.release.cta.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Descriptor of an operand tile in shared memory: rows of 128 bytes in the
// 128-byte swizzle, groups of 8 rows 1024 bytes apart.  Its low word holds the
// address (in units of 16 bytes; blocks' shared memory ends below 2^18), its
// high word is a constant.
constexpr uint32_t kOperandHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
// Descriptor of a tile of scales: 32 rows of 16 bytes, no swizzle, groups of 8 rows 128 bytes apart.
constexpr uint32_t kScaleHigh = (128 >> 4) | 1u << 14;
__device__ __forceinline__ uint32_t desc_low(uint32_t addr) { return addr >> 4 | 1u << 16; }
__device__ __forceinline__ uint64_t desc(uint32_t low, uint32_t high) { return (uint64_t)high << 32 | low; }
// One lane of the warp, always the same one; to be called by whole warps.
__device__ __forceinline__ bool elected() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}
// Scales of 128 rows into four columns, the same in each quarter of the lanes.
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                           uint32_t add) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
      " tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(add)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

// 16 columns of this warp's 32 lanes.
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
// mbar_wait for a whole warp: false in every lane where one gave up.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(~0u, mbar_wait(bar, parity)); }
// The address of `addr` in the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// What earlier kernels of the stream wrote may be used from here on: launches may begin before those have ended.
__device__ __forceinline__ void wait_for_earlier_kernels() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Instruction descriptor: E4M3 operands, E8M0 scales, m = 128 lanes, n = TM columns; the scales' byte of the two
// operands' 32-bit columns.
template <int TM>
__device__ __forceinline__ uint32_t instr_desc(uint32_t byte) {
  return (uint32_t)(TM >> 3) << 17 | 1u << 23 | (uint32_t)(kTileN >> 4) << 24 | byte << 4 | byte << 29;
}

// ---------------------------------------------------------------------------
// Tiles of 128 x TM, one CTA each, or, where tiles alone leave SMs idle, the 1,
// 2, 4 or 8 CTAs of a cluster: each takes a run of k, writes its sums to its
// shared memory and adds up all CTAs' for its share of the tile's lanes, in the
// CTAs' order, so that the same product gives the same bits.  A token through
// 11008 x 4096 (45 MB of codes) takes 12 us, 3.4 of them before the first copy
// and after the last; then an SM's intake of about 60 GB/s bounds it.  Two CTAs fit an
// SM: one's first copies and last stores run under the other's products.  Tiles
// of fewer than 128 rows of a are for an a that has no more (matmul_plan), so
// that every tile starts with its scale tile.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float4 lds_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ void sts_cluster(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
// Sums of all CTAs of a cluster over four neighbouring lanes, in the CTAs' order; all loads in flight at once.
template <int SPLIT>
__device__ __forceinline__ float4 cluster_sum(uint32_t addr) {
  float4 v[SPLIT];
#pragma unroll
  for (int s = 0; s < SPLIT; ++s) v[s] = lds_cluster(peer_addr(addr, s));
#pragma unroll
  for (int s = 1; s < SPLIT; ++s) {
    v[0].x = __fadd_rn(v[0].x, v[s].x), v[0].y = __fadd_rn(v[0].y, v[s].y);
    v[0].z = __fadd_rn(v[0].z, v[s].z), v[0].w = __fadd_rn(v[0].w, v[s].w);
  }
  return v[0];
}

template <int TM, bool F32>
__global__ void __launch_bounds__(kMatmulThreads, 2) matmul_kernel(const __grid_constant__ MatmulArgs p) {
  using S = Shape<TM>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ alignas(8) uint64_t bars[2 * S::kStages + 2];
  __shared__ uint32_t tmem_base_s;
  __shared__ int32_t failed;
  const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t bar0 = smem_addr(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };
  auto empty = [&](int s) { return bar0 + 8u * (S::kStages + s); };
  const uint32_t acc_full = bar0 + 8u * (2 * S::kStages), drained = acc_full + 8;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    mbar_init(acc_full, 1);
    mbar_init(drained, 1);
    failed = 0;
    mbar_init_fence();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_base_s)),
                 "r"((uint32_t)S::kCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_s;
  const uint32_t tmem_scales = tmem + TM;
  // After a's quantisation, which lets this kernel begin once it has itself waited for all before it, only a has to be
  // waited for, by the thread that copies it (d is not touched before a has been used).
  if (!p.b_early) wait_for_earlier_kernels();

  const int tiles_m = (p.m + TM - 1) / TM;
  const int tile = blockIdx.x / p.split, rank = blockIdx.x % p.split;
  const int tn = tile / tiles_m, tm = tile % tiles_m;
  const int steps_all = (p.k + kTileK - 1) / kTileK, groups = (steps_all + 3) / 4;
  const int k0 = 4 * (int)((int64_t)groups * rank / p.split), k1 = min(steps_all, 4 * (int)((int64_t)groups * (rank + 1) / p.split));
  volatile int32_t* stop = &failed;

  if (warp == 0) {
    if (lane == 0) {
      auto load_b = [&](int s, int k) {
        const uint32_t st = smem + s * S::kStageBytes;
        mbar_arrive_tx(full(s), (kTileN + TM) * kTileK + ((k & 3) == 0 ? S::kScaleBytes : 0));
        tma_load_2d(st, &p.b, k * kTileK, tn * kTileN, full(s));
        if ((k & 3) == 0)
          bulk_load(st + (kTileN + TM) * kTileK, p.sb + ((int64_t)tn * groups + (k >> 2)) * kScaleTile, kScaleTile, full(s));
      };
      auto load_a = [&](int s, int k) {
        const uint32_t st = smem + s * S::kStageBytes;
        tma_load_2d(st + kTileN * kTileK, &p.a, k * kTileK, tm * TM, full(s));
        if ((k & 3) == 0)
          bulk_load(st + (kTileN + TM) * kTileK + kScaleTile, p.sa + ((int64_t)tm * groups + (k >> 2)) * kScaleTile, kScaleTile,
                    full(s));
      };
      int k = k0;
      if (p.b_early) {
        const int ahead = min(S::kStages, k1 - k0);
        for (int i = 0; i < ahead; ++i) load_b(i, k0 + i);
        wait_for_earlier_kernels();
        for (int i = 0; i < ahead; ++i) load_a(i, k0 + i);
        k += ahead;
      }
      int s = (k - k0) % S::kStages;
      uint32_t phase = (k - k0) / S::kStages;
      for (; k < k1; ++k) {
        if (!mbar_wait(empty(s), phase ^ 1)) break;
        load_b(s, k);
        load_a(s, k);
        if (++s == S::kStages) { s = 0; phase ^= 1; }
      }
      if (k < k1) {
        *stop = 1;
        atomicOr(p.err, kErrStage);
        // the copies in flight, those of the last stages, before the block's memory goes
        for (int i = 0; i < min(k - k0, S::kStages); ++i) {
          if (s == 0) { s = S::kStages; phase ^= 1; }
          --s;
          mbar_wait(full(s), phase);
        }
      }
    }
  } else if (warp == 1) {
    // The whole warp walks the stages, so that addresses stay in uniform registers, and one lane issues.
    const bool issue = elected();
    const uint32_t low0 = desc_low(smem);
    int s = 0;
    uint32_t phase = 0;
    int at = k1;  // the step whose operands were given up
    for (int kg = k0; kg < at; kg += 4) {
      const uint32_t sb = tmem_scales + ((kg >> 2) & 1) * S::kScaleCols, sa = sb + 4;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (kg + j >= k1) break;
        if (!warp_wait(full(s), phase)) { at = kg + j; break; }
        tc_fence_after();
        if (issue) {
          const uint32_t low = low0 + s * (S::kStageBytes >> 4);
          if (j == 0) {
            const uint32_t sc = low + ((kTileN + TM) * kTileK >> 4);
            copy_scales(sb, desc(sc, kScaleHigh));
            copy_scales(sa, desc(sc + (kScaleTile >> 4), kScaleHigh));
          }
#pragma unroll
          for (int i = 0; i < kTileK / 32; ++i)
            mma_scaled(tmem, desc(low + 2 * i, kOperandHigh), desc(low + (kTileN * kTileK >> 4) + 2 * i, kOperandHigh),
                       instr_desc<TM>(j), sb, sa, j > 0 || i > 0 || kg > k0);
          mma_commit(empty(s));
        }
        if (++s == S::kStages) { s = 0; phase ^= 1; }
      }
    }
    if (at == k1) {
      if (issue) mma_commit(acc_full);
    } else {
      // The products and copies in flight, before their memory goes (once the products are done, the producer fills every
      // stage again); then the epilogue is woken up to find that it has nothing to store.
      if (issue) {
        atomicOr(p.err, kErrCopy);
        mma_commit(drained);
      }
      warp_wait(drained, 0);
      for (const int end = min(k1, at + S::kStages); at < end; ++at) {
        warp_wait(full(s), phase);
        if (++s == S::kStages) { s = 0; phase ^= 1; }
      }
      if (issue) {
        *stop = 1;
        mbar_arrive(acc_full);
      }
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, half = (warp - 4) >> 2;
    constexpr int kHalf = TM / 2 >= 16 ? TM / 2 : 16;  // columns of one warp
    if (!warp_wait(acc_full, 0)) {
      if (lane == 0) { atomicOr(p.err, kErrAcc); *stop = 1; }
    } else if (!*stop && half * kHalf < TM) {
      tc_fence_after();
      const int n = tn * kTileN + quarter * 32 + lane;
      for (int c = half * kHalf; c < half * kHalf + kHalf; c += 16) {
        const int m0 = tm * TM + c;
        if (m0 >= p.m) break;
        uint32_t r[16];
        __syncwarp();
        tmem_load16(tmem + c + ((uint32_t)(quarter * 32) << 16), r);
        tmem_wait_load();
        const int rows = min(16, p.m - m0);
        if (p.split > 1) {  // the stages' memory is free: every copy has been used
#pragma unroll
          for (int j = 0; j < 16; ++j) sts_u32(smem + ((c + j) * kTileN + quarter * 32 + lane) * 4, r[j]);
        } else if (n < p.n) {
          const int64_t at = (int64_t)m0 * p.ldd + n;
          if (F32) {
            float* d = static_cast<float*>(p.d) + at;
            if (p.accumulate) {
              float old[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) old[j] = j < rows ? d[j * p.ldd] : 0.0f;
#pragma unroll
              for (int j = 0; j < 16; ++j) r[j] = __float_as_uint(__fadd_rn(old[j], __uint_as_float(r[j])));
            }
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (j < rows) d[j * p.ldd] = __uint_as_float(r[j]);
          } else {
            uint16_t* d = static_cast<uint16_t*>(p.d) + at;
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (j < rows) d[j * p.ldd] = (uint16_t)bf16x2_rn(__uint_as_float(r[j]), 0.0f);
          }
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)S::kCols) : "memory");
  if (p.split > 1) {
    if (threadIdx.x == 0 && *stop) {  // no sum without this CTA's share
      for (int s = 0; s < p.split; ++s) sts_cluster(peer_addr(smem_addr(&failed), s), 1);
    }
    cluster_sync();
    const int width = kTileN / p.split, rows = *stop ? 0 : min(TM, p.m - tm * TM);
#pragma unroll 2
    for (int e = threadIdx.x; e < rows * width / 4; e += kMatmulThreads) {
      const int j = 4 * e / width, l = rank * width + 4 * e % width, n = tn * kTileN + l;
      const uint32_t at = smem + (j * kTileN + l) * 4;
      const float4 v = p.split == 2 ? cluster_sum<2>(at) : p.split == 4 ? cluster_sum<4>(at) : cluster_sum<8>(at);
      const float x[4] = {v.x, v.y, v.z, v.w};
      const int64_t to = (int64_t)(tm * TM + j) * p.ldd + n;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (n + i >= p.n) break;
        if (F32) {
          float* d = static_cast<float*>(p.d) + to + i;
          *d = p.accumulate ? __fadd_rn(*d, x[i]) : x[i];
        } else {
          static_cast<uint16_t*>(p.d)[to + i] = (uint16_t)bf16x2_rn(x[i], 0.0f);
        }
      }
    }
    cluster_sync();  // nobody leaves while its sums are read
  }
}

// ---------------------------------------------------------------------------
// Tiles of 256 x TM by pairs of CTAs: the two SMs' tensor cores work on one
// product of 256 lanes (128 in each SM's tensor memory) by TM columns, each SM
// holding half of either operand.  A stage is then 32 KB for 2 x 128 x 128 x 256
// multiply-adds an SM, against 48 KB where one CTA makes a tile of 128 x 256.
// 8192 x 11008 x 4096 takes 225 us (3.28 PFLOP/s) after a pause and 257 (2.87)
// in a long run, where the power limit lowers the clock; 8192 cubed 303 us (3.63
// PFLOP/s, the tensor pipe active in 85 % of all cycles).  The rest: about 3000
// cycles a tile until the accumulator has been read out, and last waves that are not full.
// ---------------------------------------------------------------------------
constexpr int kPairTileN = 256;
constexpr int kPairStages = 6;
constexpr int kGroupRows = 8;  // row tiles of a that neighbouring clusters share out, so that they meet in L2

template <int TM>
struct PairShape {
  // Two accumulators where tensor memory has room for them beside the scales: the next tile's products then need not
  // wait until this one's have been read out (about 3000 cycles a tile).
  static constexpr int kAccs = TM > 192 ? 1 : 2;
  static constexpr int kScaleTilesA = 2;  // 128-row tiles that TM rows from a multiple of TM may touch
  static constexpr int kScaleCols = 4 + 4 * kScaleTilesA;
  static constexpr int kBytesB = 128 * kTileK, kBytesA = TM / 2 * kTileK, kBytesScales = kScaleTile * (1 + kScaleTilesA);
  static constexpr int kStageBytes = kBytesB + kBytesA + 2048;  // b's rows, a's rows, scales of 128 rows of b and of a's
  static constexpr int kDynSmem = kPairStages * kStageBytes + 1024;
  static constexpr uint32_t kTx = 2 * (kBytesB + kBytesA), kScaleTx = 2 * kBytesScales;  // of both CTAs
  static_assert(kStageBytes % 1024 == 0 && kBytesScales <= 2048, "layout of a stage");
  // A column of scales holds 32 rows, and a product's scales have to start at an even column (an odd one is a misaligned
  // address), so tiles start at multiples of 64 rows.
  static_assert(TM == 256 || TM == 192, "tiles start at multiples of 64 rows, in at most two scale tiles");
  static_assert(kAccs * TM + 2 * kScaleCols <= 512, "tensor memory");
};

__device__ __forceinline__ void pair_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void pair_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void pair_copy_scales(uint32_t tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void pair_mma_scaled(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                                uint32_t add) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %6, 0;\n"
      " tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(add)
      : "memory");
}
// Arrives at `bar` in both CTAs when all that was issued before is done.
__device__ __forceinline__ void pair_commit(uint32_t bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
      "h"((uint16_t)3)
      : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity) {
  for (uint32_t i = 0; i < kSpinLimit; ++i) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n"
        " selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    if (ok) return true;
  }
  return false;
}
__device__ __forceinline__ bool warp_wait_cluster(uint32_t bar, uint32_t parity) {
  return __all_sync(~0u, mbar_wait_cluster(bar, parity));
}
// 32 columns of this warp's 32 lanes.
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
      "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
        "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
        "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}

// Tile t's place: kGroupRows row tiles of a at a time, all of b's before the next ones.
__device__ __forceinline__ void pair_place(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
  const int group = t / (kGroupRows * tiles_n), first = group * kGroupRows;
  const int rows = min(kGroupRows, tiles_m - first), in = t - group * kGroupRows * tiles_n;
  tm = first + in % rows;
  tn = in / rows;
}

template <int TM, bool F32>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kMatmulThreads, 1)
    matmul_pair_kernel(const __grid_constant__ MatmulArgs p) {
  using S = PairShape<TM>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ alignas(8) uint64_t bars[2 * kPairStages + 2 * S::kAccs + 1];
  __shared__ uint32_t tmem_base_s;
  __shared__ int32_t failed;
  const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const uint32_t bar0 = smem_addr(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };                   // the leader's alone
  auto empty = [&](int s) { return bar0 + 8u * (kPairStages + s); };  // each CTA's own
  auto acc_full = [&](int a) { return bar0 + 8u * (2 * kPairStages + a); };
  auto acc_free = [&](int a) { return bar0 + 8u * (2 * kPairStages + S::kAccs + a); };
  const uint32_t drained = bar0 + 8u * (2 * kPairStages + 2 * S::kAccs);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kPairStages; ++s) {
      mbar_init(full(s), 1);
      mbar_init(empty(s), 1);
    }
    for (int a = 0; a < S::kAccs; ++a) {
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

  const int tiles_n = (p.n + kPairTileN - 1) / kPairTileN, tiles_m = (p.m + TM - 1) / TM;
  const int tiles = tiles_n * tiles_m, pairs = gridDim.x / 2;
  const int steps = (p.k + kTileK - 1) / kTileK;
  volatile int32_t* stop = &failed;

  if (warp == 0) {
    if (lane == 0) {
      int s = 0, issued = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int t = blockIdx.x / 2; t < tiles && ok; t += pairs) {
        if (*stop) { ok = false; break; }
        int tm, tn;
        pair_place(t, tiles_m, tiles_n, tm, tn);
        for (int k = 0; k < steps; ++k) {
          if (!mbar_wait(empty(s), phase ^ 1)) { ok = false; break; }
          const uint32_t st = smem + s * S::kStageBytes, bar = peer_addr(full(s), 0);
          const bool scales = (k & 3) == 0;
          if (rank == 0) mbar_arrive_tx(full(s), S::kTx + (scales ? S::kScaleTx : 0));
          pair_load_2d(st, &p.b, k * kTileK, tn * kPairTileN + (int)rank * 128, bar);
          pair_load_2d(st + S::kBytesB, &p.a, k * kTileK, tm * TM + (int)rank * (TM / 2), bar);
          if (scales) {
            const uint32_t sc = st + S::kBytesB + S::kBytesA;
            pair_load_3d(sc, &p.sb_map, 0, k >> 2, tn * 2 + (int)rank, bar);
            pair_load_3d(sc + kScaleTile, &p.sa_map, 0, k >> 2, tm * TM / 128, bar);
          }
          ++issued;
          if (++s == kPairStages) { s = 0; phase ^= 1; }
        }
      }
      if (!ok) {
        *stop = 1;
        atomicOr(p.err, kErrStage);
        // the copies in flight: the leader sees both CTAs' last stages arrive, the other one waits for it in the end
        for (int i = 0; i < min(issued, kPairStages); ++i) {
          if (s == 0) { s = kPairStages; phase ^= 1; }
          --s;
          if (rank == 0) mbar_wait(full(s), phase);
        }
      }
    }
  } else if (warp == 1 && rank == 0) {
    const bool issue = elected();  // as in matmul_kernel
    const uint32_t low0 = desc_low(smem);
    int s = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    int t = blockIdx.x / 2, at = steps;  // the tile, and its step whose operands were given up
    for (; t < tiles; t += pairs) {
      if (!warp_wait_cluster(acc_free(acc), acc_phase ^ 1)) { at = 0; break; }
      tc_fence_after();
      const uint32_t d = tmem + acc * TM;
      int tm, tn;
      pair_place(t, tiles_m, tiles_n, tm, tn);
      const uint32_t col = (uint32_t)(tm * TM % 128) / 32;  // 0 or 2
      for (int g = 0; 4 * g < at; ++g) {
        const uint32_t sb = tmem + S::kAccs * TM + (g & 1) * S::kScaleCols, sa = sb + 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int k = 4 * g + j;
          if (k >= steps) break;
          if (!warp_wait(full(s), phase)) { at = k; break; }
          tc_fence_after();
          if (issue) {
            const uint32_t low = low0 + s * (S::kStageBytes >> 4);
            if (j == 0) {
              const uint32_t sc = low + ((S::kBytesB + S::kBytesA) >> 4);
              pair_copy_scales(sb, desc(sc, kScaleHigh));
#pragma unroll
              for (int i = 0; i < S::kScaleTilesA; ++i)
                pair_copy_scales(sa + 4 * i, desc(sc + (i + 1) * (kScaleTile >> 4), kScaleHigh));
            }
            const uint32_t id = (uint32_t)(TM >> 3) << 17 | 1u << 23 | (uint32_t)(kPairTileN >> 4) << 24 | (uint32_t)j << 4 |
                                (uint32_t)j << 29;
#pragma unroll
            for (int i = 0; i < kTileK / 32; ++i)
              pair_mma_scaled(d, desc(low + 2 * i, kOperandHigh), desc(low + (S::kBytesB >> 4) + 2 * i, kOperandHigh), id, sb,
                              sa + col, j > 0 || i > 0 || g > 0);
            pair_commit(empty(s));
          }
          if (++s == kPairStages) { s = 0; phase ^= 1; }
        }
      }
      if (at < steps) break;
      if (issue) pair_commit(acc_full(acc));
      if (++acc == S::kAccs) { acc = 0; acc_phase ^= 1; }
    }
    if (at < steps) {
      // As in matmul_kernel, for both CTAs: their copies arrive here.
      if (issue) {
        atomicOr(p.err, kErrCopy);
        pair_commit(drained);
      }
      warp_wait(drained, 0);
      const int64_t left = (int64_t)((tiles - 1 - t) / pairs) * steps + steps - at;
      for (int i = 0; i < (int)min(left, (int64_t)kPairStages); ++i) {
        warp_wait(full(s), phase);
        if (++s == kPairStages) { s = 0; phase ^= 1; }
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
    constexpr int kHalf = TM / 2;  // columns of one warp
    int acc = 0;
    uint32_t acc_phase = 0;
    for (int t = blockIdx.x / 2; t < tiles; t += pairs) {
      if (!warp_wait_cluster(acc_full(acc), acc_phase) || *stop) {
        if (lane == 0) { atomicOr(p.err, kErrAcc); *stop = 1; }
        break;
      }
      tc_fence_after();
      int tm, tn;
      pair_place(t, tiles_m, tiles_n, tm, tn);
      const int n = tn * kPairTileN + (int)rank * 128 + quarter * 32 + lane, m0 = tm * TM + half * kHalf;
      // All of this warp's values first, so that the accumulator is free again.
      uint32_t r[kHalf];
      const uint32_t from = tmem + acc * TM + half * kHalf + ((uint32_t)(quarter * 32) << 16);
#pragma unroll
      for (int c = 0; c < kHalf / 32; ++c) tmem_load32(from + 32 * c, r + 32 * c);
      tmem_wait_load();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(peer_addr(acc_free(acc), 0));
      if (++acc == S::kAccs) { acc = 0; acc_phase ^= 1; }
      const int rows = min(kHalf, p.m - m0);
      if (n < p.n && rows > 0) {
        const int64_t at = (int64_t)m0 * p.ldd + n;
        if (F32) {
          float* d = static_cast<float*>(p.d) + at;
          if (p.accumulate) {
#pragma unroll
            for (int c = 0; c < kHalf; c += 16) {
              float old[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) old[j] = c + j < rows ? d[(c + j) * p.ldd] : 0.0f;
#pragma unroll
              for (int j = 0; j < 16; ++j) r[c + j] = __float_as_uint(__fadd_rn(old[j], __uint_as_float(r[c + j])));
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (c + j < rows) d[(c + j) * p.ldd] = __uint_as_float(r[c + j]);
            }
          } else {
#pragma unroll
            for (int j = 0; j < kHalf; ++j)
              if (j < rows) d[j * p.ldd] = __uint_as_float(r[j]);
          }
        } else {
          uint16_t* d = static_cast<uint16_t*>(p.d) + at;
#pragma unroll
          for (int j = 0; j < kHalf; ++j)
            if (j < rows) d[j * p.ldd] = (uint16_t)bf16x2_rn(__uint_as_float(r[j]), 0.0f);
        }
      }
      __syncwarp();
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// Lets a kernel use `bytes` of shared memory on the current device, once.
template <typename K>
cudaError_t allow_smem(K* kernel, int bytes, std::atomic<uint64_t>& ready) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (ready.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) ready.fetch_or(bit);
  return e;
}

template <int TM, bool F32>
cudaError_t launch_pair(const MatmulArgs& a, cudaStream_t stream) {
  using S = PairShape<TM>;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem(matmul_pair_kernel<TM, F32>, S::kDynSmem, ready);
  if (e != cudaSuccess) return e;
  const int64_t tiles = (int64_t)((a.n + kPairTileN - 1) / kPairTileN) * ((a.m + TM - 1) / TM);
  return launch_dependent((const void*)matmul_pair_kernel<TM, F32>, 2 * (unsigned)std::min<int64_t>(tiles, kSms / 2), kMatmulThreads,
                          0, S::kDynSmem, &a, stream);
}

template <int TM>
cudaError_t launch_pair(const MatmulArgs& a, cudaStream_t stream) {
  return a.f32 ? launch_pair<TM, true>(a, stream) : launch_pair<TM, false>(a, stream);
}

template <int TM, bool F32>
cudaError_t launch(const MatmulArgs& a, cudaStream_t stream) {
  using S = Shape<TM>;
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem(matmul_kernel<TM, F32>, S::kDynSmem, ready);
  if (e != cudaSuccess) return e;
  const int64_t tiles = (int64_t)((a.n + kTileN - 1) / kTileN) * ((a.m + TM - 1) / TM);
  return launch_dependent((const void*)matmul_kernel<TM, F32>, (unsigned)(tiles * a.split), kMatmulThreads, a.split, S::kDynSmem, &a,
                          stream);
}

template <int TM>
cudaError_t launch(const MatmulArgs& a, cudaStream_t stream) {
  return a.f32 ? launch<TM, true>(a, stream) : launch<TM, false>(a, stream);
}

// Columns of a pair's tile: those with which all of a product's waves take less, by the time of one wave of each size
// (fitted to 16 to 64 steps of k on shapes from 2048 to 11008: 7.4, 12.1, 17.1 and 23.0 us with 256 columns and 16, 32, 44
// and 64 steps, 5.8, 9.5, 12.2 and 17.5 with 192).  4096 cubed takes 53.6 us with 256 and 47.5 with 192, 8192 x 2048 x
// 5632 68.3 and 61.0, 8192 cubed 322.6 and 333.1, 2048 x 5632 x 8192 70.3 and 75.8.
int pair_tile(int64_t m, int64_t n, int64_t k) {
  auto time = [&](int tm, double step, double tile) {
    const int64_t tiles = ((m + tm - 1) / tm) * ((n + kPairTileN - 1) / kPairTileN);
    return (double)((tiles + kSms / 2 - 1) / (kSms / 2)) * ((double)((k + kTileK - 1) / kTileK) * step + tile);
  };
  return time(192, 0.245, 1.86) < time(256, 0.326, 2.2) ? 192 : 256;
}

}  // namespace

MatmulPlan matmul_plan(int64_t m, int64_t n, int64_t k) {
  // Pairs of CTAs from 40 tiles of 256 x 256 on, about half of what runs at once (36 tiles, 1023 x 2304 x 768: 8.2 us
  // by pairs, 6.8 by single CTAs; 40, 1280 x 2048 x 4096: 15.0 and 15.9; 43, 256 x 11008 x 4096: 17.3 and 19.2).  Else
  // tiles of 128 x up to 128, a tile's k shared out among CTAs while all of them run at once with one an SM: an SM takes
  // in about 60 GB/s, so idle ones cost (1 x 4096 x 4096 10.3 us by 32 CTAs, 6.2 by 128), but with a second CTA on many
  // SMs the others wait (1024 x 2048 x 2048 8.9 us by 128, 12.3 by 256).  Eight SMs with two are worth it up to 64 rows of
  // a or with a long k: 1 x 5120 x 4096 6.1 us by 160 CTAs, 7.4 by 80; 1 x 10240 x 4096 7.8 and 9.5; 128 x 10240 x 11008
  // 28.7 and 35.9; they cost where sums of 128 rows are joined after a short k (128 x 2560 x 4096 11.1 and 7.9).
  const int64_t large = ((m + 255) / 256) * ((n + 255) / 256);
  if (m > 128 && large >= 40) return {pair_tile(m, n, k), 1, true};
  const int tile = m <= 16 ? 16 : m <= 32 ? 32 : m <= 64 ? 64 : 128;
  const int64_t tiles = ((m + tile - 1) / tile) * ((n + kTileN - 1) / kTileN), groups = (k + 511) / 512;
  int split = 1;
  while (split < 8 && 2 * split <= groups && 2 * split * tiles <= kSms + 8) split *= 2;
  return {tile, split, false};
}

cudaError_t launch_matmul(MatmulArgs& a, const MatmulPlan& plan, cudaStream_t stream) {
  if (plan.pair) return plan.tile == 256 ? launch_pair<256>(a, stream) : launch_pair<192>(a, stream);
  a.split = plan.split;
  switch (plan.tile) {
    case 16: return launch<16>(a, stream);
    case 32: return launch<32>(a, stream);
    case 64: return launch<64>(a, stream);
    default: return launch<128>(a, stream);
  }
}

cudaError_t matmul_error_word(int32_t** p) {
  return cudaGetSymbolAddress(reinterpret_cast<void**>(p), g_matmul_error);
}

}  // namespace mpadam
