// muon_products.cu -- the products of all Newton-Schulz steps (muon.h) over a
// list of matrices, in one launch:
//   A = X X^T,   B = a I + b A + c A A,   X <- B X
// of X's first part; a times its second part is added to the last.  A and B are
// symmetric: only their tiles on and below the diagonal are computed and stored, and
// read as they lie or turned (an operand of the tensor cores may run along either of
// its sides).
//
// The host lists every tile of every product in an order in which it can be made
// (muon_schedule.h), and pairs of CTAs take them from that list one after another
// by a counter.  Every 256 rows of a matrix have a counter of their own, which every
// warp that has stored a part of a result in them raises, and a tile says how far
// those of its operands' rows have to be; who takes it waits for that (bounded).
//   A's tile (i, j) waits for rows i and j of X, B's for rows i and j of A, X's
//   tile (i, n) for row i of B, and so for all that B's row was made of.
// What a tile writes over was read only by tiles that those rows waited for.
// Whatever a tile waits for is ahead of it in the list and taken by a pair that
// runs, so the first tile that is not done can always go on, however many pairs run
// at once.  One launch a product left the last wave of each to itself, 10 us of
// launch, first copies and last stores each time, and X, A and B of a whole list out
// of L2 in between.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "launch.h"
#include "muon.h"
#include "tcgen05.cuh"

namespace mpadam {

namespace {

constexpr int kStepK = kNewtonStepK;  // a row of one 128-byte swizzle atom
constexpr int kStages = 5;
constexpr int kBoxBytes = 64 * 64 * 2;
constexpr int kStageBytes = 4 * kBoxBytes;  // 128 rows of either operand
constexpr uint32_t kStageTx = 2 * kStageBytes;  // of both CTAs
constexpr int kEpiWarps = 8;
static_assert(2 * kEpiWarps == kSignals, "every epilogue warp of a pair says when it has stored its part");
constexpr int kPatchBytes = 32 * 64 * 2;        // rows of one 128-byte swizzle atom
constexpr int kPatches = 2;                     // of a warp, in a tile
constexpr int kEpiBytes = kPatches * kPatchBytes;
static_assert(64 * kPatches * 2 == kNewtonTile, "two warps side by side");
constexpr int kDynSmem = kStages * kStageBytes + kEpiWarps * kEpiBytes + 1024;
constexpr int kProductThreads = 32 * (4 + kEpiWarps);  // producer, issuer, the one who takes tiles, their maps', then the epilogue
constexpr int kSlots = 3;                       // tiles that a pair has taken ahead of its epilogue
constexpr int kReaders = 2 * kEpiWarps + 5;     // of a slot: epilogue warps, a producer and the maps' warp in both CTAs, the issuer

enum ProductError : int32_t { kErrCopy = 1, kErrStage = 2, kErrAcc = 4, kErrSlot = 8, kErrTurn = 16 };

// The steps' coefficients (K. Jordan et al., "Muon: An optimizer for hidden layers in neural networks", 2024).
constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;

// An operand whose rows run along n instead of k: chunks of 64 of them 8192 bytes apart, groups of 8 values of k 1024.
__device__ __forceinline__ uint32_t desc_low_mn(uint32_t addr) { return addr >> 4 | (uint32_t)(kBoxBytes >> 4) << 16; }

__device__ __forceinline__ void pair_mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}

// Bytes that a barrier waits for as if a copy had brought them.
__device__ __forceinline__ void mbar_complete_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.complete_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

__device__ __forceinline__ void sts_v4(uint32_t addr, const uint32_t (&v)[4]) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ uint4 lds_v4(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
// What this thread wrote to shared memory may be read by copies from here on.
__device__ __forceinline__ void fence_for_copies() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, int x, int y, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(src)
               : "memory");
}
__device__ __forceinline__ void commit_stores() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// This thread's stores, but for the last LEFT groups, have read what they store; or all have stored it.
template <int LEFT>
__device__ __forceinline__ void wait_for_reads() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void wait_for_stores() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// A tensor map that the host copied to memory may be used by this block's copies from here on; what the SM kept of
// another one that lay there before may not.
__device__ __forceinline__ void acquire_map(const CUtensorMap* map) {
  asm volatile("fence.proxy.tensormap::generic.acquire.sys [%0], 128;" ::"l"(map) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  uint32_t h;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(h) : "f"(hi), "f"(lo));
  return h;
}
__device__ __forceinline__ float2 of_half2(uint32_t h) {
  float2 x;
  asm("{\n .reg .f16 lo, hi;\n mov.b32 {lo, hi}, %2;\n cvt.f32.f16 %0, lo;\n cvt.f32.f16 %1, hi;\n}" : "=f"(x.x), "=f"(x.y) : "r"(h));
  return x;
}

__device__ __forceinline__ uint32_t load_relaxed(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void fence_gpu() { asm volatile("fence.acq_rel.gpu;" ::: "memory"); }
__device__ __forceinline__ void add_one_release(uint32_t* p) { asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(p) : "memory"); }
// Between this thread's ordinary accesses to global memory and copies: in either direction.
__device__ __forceinline__ void fence_copies_global() { asm volatile("fence.proxy.async.global;" ::: "memory"); }

// A tile is 256 rows m by 256 columns n of a product's result, by a pair of CTAs;
// a warp of the epilogue takes 32 rows, a row a lane, and 128 columns, in two
// patches.  What is added to a patch's sums (A, or X's second part) is copied to
// shared memory as the tile begins, the results take its place there and are copied
// out; X's second part is held in registers until the first has gone.  Copies know
// the matrix's edges (nothing lies beyond them, nothing is stored there).  Shared
// memory's bandwidth is what this competes for: the products read 64 bytes a cycle
// of it and the operands' copies write as many.  A row a lane straight from and to
// memory (a line of L1 for 16 bytes), and results stored turned as well, took 8 us of
// a warp's time a tile; this takes 3, and a Muon step of half of GPT-2's hidden
// matrices 770 us, where it took 1087.
// One lane of the pair takes tiles and waits for their rows, so that nobody else has
// to look.
// Within a tile 64 values of k take 526 (A, B) to 565 cycles (X) at 4096 x 11008, of
// which the products are 512; in half of GPT-2's hidden matrices 590 to 670, with an
// epilogue every twelve of them.  The kernel takes 1.85 ms for 4096 x 11008 after a
// pause (1.69 PFLOP/s), 2.1 in a long run, where the power limit lowers the clock.
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kProductThreads, 1) newton_kernel(const __grid_constant__ ProductArgs p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ alignas(8) uint64_t bars[2 * kStages + 5 + 3 * kSlots + kEpiWarps];
  __shared__ alignas(16) int4 slots[kSlots];
  __shared__ uint32_t tmem_base_s;
  __shared__ int32_t failed;
  __shared__ int32_t asked[2];  // steps whose copies a CTA has asked for, when it asks for no more; the leader's alone
  const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const uint32_t bar0 = smem_addr(bars);
  auto full = [&](int s) { return bar0 + 8u * s; };               // the leader's alone
  auto empty = [&](int s) { return bar0 + 8u * (kStages + s); };  // each CTA's own
  auto acc_full = [&](int a) { return bar0 + 8u * (2 * kStages + a); };
  auto acc_free = [&](int a) { return bar0 + 8u * (2 * kStages + 2 + a); };
  const uint32_t drained = bar0 + 8u * (2 * kStages + 4);
  auto slot_full = [&](int s) { return bar0 + 8u * (2 * kStages + 5 + s); };           // each CTA's own
  auto slot_free = [&](int s) { return bar0 + 8u * (2 * kStages + 5 + kSlots + s); };  // the leader's alone
  auto slot_ready = [&](int s) { return bar0 + 8u * (2 * kStages + 5 + 2 * kSlots + s); };  // each CTA's own: rows and maps are there
  auto addend_full = [&](int w) { return bar0 + 8u * (2 * kStages + 5 + 3 * kSlots + w); };

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
    for (int s = 0; s < kSlots; ++s) {
      mbar_init(slot_full(s), 1);
      mbar_init(slot_free(s), kReaders);
      mbar_init(slot_ready(s), 2);
    }
    for (int w = 0; w < kEpiWarps; ++w) mbar_init(addend_full(w), 1);
    failed = asked[0] = asked[1] = 0;
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

  volatile int32_t* stop = &failed;
  // Nobody waits for long once someone of the pair has given up.
  auto stop_both = [&] {
    for (uint32_t r = 0; r < 2; ++r) sts_cluster(peer_addr(smem_addr(&failed), r), 1);
  };
  auto give_up = [&](int32_t why) {
    atomicOr(p.err, why);
    stop_both();
  };
  auto wait = [&](uint32_t bar, uint32_t parity) {
    for (uint32_t i = 0; i < kSpinLimit; ++i) {
      if (mbar_try_wait(bar, parity)) return true;
      if (*stop) return false;
    }
    return false;
  };
  auto wait_cluster = [&](uint32_t bar, uint32_t parity) {
    for (uint32_t i = 0; i < kSpinLimit; ++i) {
      if (mbar_try_wait_cluster(bar, parity)) return true;
      if (*stop) return false;
    }
    return false;
  };
  auto tile_of = [](int4 v) {
    return NewtonTile{v.x, (uint16_t)v.y, (uint16_t)((uint32_t)v.y >> 16), v.z, (uint32_t)v.w};
  };
  auto tile_in = [&](int s) {
    const volatile int4& v = slots[s];
    return tile_of(make_int4(v.x, v.y, v.z, v.w));
  };
  // The pair's n-th tile, when its turn has come; matrix < 0: there are no more.  By whole warps, or by one lane (whole = false).
  auto read_slot = [&](int n, NewtonTile& t, bool whole) {
    const int s = n % kSlots;
    bool ok = wait_cluster(slot_ready(s), (uint32_t)(n / kSlots) & 1);
    if (whole) ok = __all_sync(~0u, ok);
    if (!ok) return false;
    t = tile_in(s);
    if (!whole || lane == 0) mbar_arrive_cluster(peer_addr(slot_free(s), 0));
    return true;
  };
  // Until the rows that the tile is made of have come as far as they have to.
  auto wait_turn = [&](const NewtonTile& t) {
    const uint32_t* count = p.progress + __ldg(&p.matrices[t.matrix].row0);
    const uint32_t *one = count + t.tm, *two = t.which() == 3 ? one : count + t.tn;
    for (uint32_t i = 0; i < kSpinLimit; ++i) {
      const uint32_t a = load_relaxed(one), b = load_relaxed(two);
      if (a >= t.need && b >= t.need) {  // (loads that acquire empty L1 every time)
        fence_gpu();
        return true;
      }
      if (*stop || ((i & 63) == 63 && *static_cast<volatile int32_t*>(p.err))) return false;
    }
    return false;
  };

  if (warp == 0) {
    if (lane == 0) {
      const uint32_t full0 = peer_addr(full(0), 0);
      int s = 0, steps_asked = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int n = 0; ok; ++n) {
        NewtonTile t;
        if (!read_slot(n, t, false)) { give_up(kErrSlot); ok = false; break; }
        if (t.matrix < 0) break;
        const NewtonMatrix& q = p.matrices[t.matrix];
        const int which = t.which(), from = t.from(), steps = t.steps_k();
        const CUtensorMap* first = which == 1 ? &q.x[from] : which == 2 ? &q.a : &q.b;
        const CUtensorMap* turned = which == 2 ? &q.a_along : &q.b_along;
        const CUtensorMap* second = which == 2 ? turned : &q.x_along[from];
        fence_copies_global();  // what others stored, and the slot's writer waited for, before what is copied here
        const int m0 = t.tm * kNewtonTile + (int)rank * 128, n0 = t.tn * kNewtonTile + (int)rank * 128;
        // (Loops of their own: a choice of maps within one took 130 cycles more a step.)
        auto load = [&](int k, int end, auto first_turned, auto second_turned) {
          for (; k < end && ok; ++k) {
            if (!wait(empty(s), phase ^ 1)) { give_up(kErrStage); ok = false; break; }
            const uint32_t st = smem + s * kStageBytes, to = st + kStageBytes / 2, bar = full0 + 8u * s;
            const int x = k * kStepK;
            if (rank == 0) mbar_arrive_tx(full(s), kStageTx);
            if (decltype(first_turned)::value) {
              pair_load_2d(st, turned, m0, x, bar);
              pair_load_2d(st + kBoxBytes, turned, m0 + 64, x, bar);
            } else {
              pair_load_2d(st, first, x, m0, bar);
            }
            if (decltype(second_turned)::value) {
              pair_load_2d(to, second, n0, x, bar);
              pair_load_2d(to + kBoxBytes, second, n0 + 64, x, bar);
            } else {
              pair_load_2d(to, first, x, n0, bar);
            }
            ++steps_asked;
            if (++s == kStages) { s = 0; phase ^= 1; }
          }
        };
        constexpr std::true_type yes;
        constexpr std::false_type no;
        const int plain = which == 1 ? steps : which == 2 ? min(steps, t.turned_from(t.tn)) : 0;
        const int half = which == 1 ? steps : min(steps, t.turned_from(t.tm));
        load(0, plain, no, no);
        load(plain, half, no, yes);
        load(half, steps, yes, yes);
      }
      sts_cluster(peer_addr(smem_addr(&asked[rank]), 0), (uint32_t)steps_asked);
    }
  } else if (warp == 2 && rank == 0) {
    if (lane == 0) {
      for (int n = 0;; ++n) {
        const int s = n % kSlots;
        if (!wait_cluster(slot_free(s), (uint32_t)(n / kSlots) & 1 ^ 1)) { give_up(kErrSlot); break; }
        const uint32_t i = atomicAdd(p.taken, 1u);
        const bool more = i < (uint32_t)p.count;
        const int4 v = more ? __ldg(reinterpret_cast<const int4*>(p.tiles) + i) : make_int4(-1, 0, 0, 0);
        for (uint32_t r = 0; r < 2; ++r) {
          const uint32_t to = peer_addr(smem_addr(&slots[s]), r);
          sts_cluster(to, (uint32_t)v.x), sts_cluster(to + 4, (uint32_t)v.y), sts_cluster(to + 8, (uint32_t)v.z), sts_cluster(to + 12, (uint32_t)v.w);
          mbar_arrive_cluster(peer_addr(slot_full(s), r));
        }
        if (more && !wait_turn(tile_of(v))) { give_up(kErrTurn); break; }
        for (uint32_t r = 0; r < 2; ++r) mbar_arrive_cluster(peer_addr(slot_ready(s), r));
        if (!more) break;
      }
    }
  } else if (warp == 3) {
    // A tile's tensor maps, before its turn.  They lie in memory that the host filled (its copy was complete before the launch),
    // where another list's may have lain that this SM still holds: a block acquires those of a matrix's product when it first
    // comes to a tile of it, then fetches them, since one that the SM does not hold costs half a microsecond.  Acquiring takes
    // 20 ns a map: 200 matrices of 256 x 256 take 290 us, with all maps of a matrix at once 313, with all of the list's as a
    // block begins 320 (1000 of 64 x 64 650 and 900).
    // What was acquired last, a lane's share each: of the products whose numbers are the same modulo kMet the last one.
    constexpr int kMet = 8 * 32;
    int32_t met[kMet / 32];
#pragma unroll
    for (int i = 0; i < kMet / 32; ++i) met[i] = -1;
    for (int n = 0;; ++n) {
      const int s = n % kSlots;
      if (!__all_sync(~0u, wait_cluster(slot_full(s), (uint32_t)(n / kSlots) & 1))) {
        if (lane == 0) give_up(kErrSlot);
        break;
      }
      const NewtonTile t = tile_in(s);
      if (t.matrix >= 0) {
        const int32_t key = (t.matrix - p.first) * 5 + (t.which() == 2 ? 4 : t.which() - 1 + t.from());  // (B reads no X)
        const int owner = key % 32, at = key % kMet / 32;
        int32_t last = -1;
#pragma unroll
        for (int i = 0; i < kMet / 32; ++i)
          if (i == at) last = met[i];
        const bool known = __shfl_sync(~0u, last, owner) == key;
        if (lane < kTileMaps) {
          const CUtensorMap* map = newton_map(p.matrices + t.matrix, tile_map(t.which(), t.from(), lane));
          if (!known) acquire_map(map);
          prefetch_map(map);
        }
#pragma unroll
        for (int i = 0; i < kMet / 32; ++i)
          if (i == at && lane == owner) met[i] = key;
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive_cluster(peer_addr(slot_ready(s), rank));
        mbar_arrive_cluster(peer_addr(slot_free(s), 0));
      }
      if (t.matrix < 0) break;
    }
  } else if (warp == 1 && rank == 0) {
    const bool issue = elected();
    // FP16 operands, binary32 sums, 256 x 256
    constexpr uint32_t kInstr = 1u << 4 | (uint32_t)(kNewtonTile >> 3) << 17 | (uint32_t)(kNewtonTile >> 4) << 24;
    int s = 0, acc = 0;
    uint32_t phase = 0, acc_phase = 0;
    bool ok = true;
    for (int n = 0; ok; ++n) {
      NewtonTile t;
      if (!read_slot(n, t, true)) { ok = false; break; }
      if (t.matrix < 0) break;
      const int steps = t.steps_k();
      if (!__all_sync(~0u, wait_cluster(acc_free(acc), acc_phase ^ 1))) { ok = false; break; }
      tc_fence_after();
      const uint32_t d = tmem + acc * kNewtonTile;
      for (int k = 0; k < steps; ++k) {
        if (!__all_sync(~0u, wait(full(s), phase))) { ok = false; break; }
        tc_fence_after();
        if (issue) {
          const uint32_t st = smem + s * kStageBytes, second_at = st + kStageBytes / 2;
          const bool first_along = t.which() != 1 && k >= t.turned_from(t.tm);
          const bool second_along = t.which() == 3 || (t.which() == 2 && k >= t.turned_from(t.tn));
          const uint32_t first = first_along ? desc_low_mn(st) : desc_low(st), second = second_along ? desc_low_mn(second_at) : desc_low(second_at);
          const uint32_t on1 = first_along ? 2048 >> 4 : 32 >> 4, on2 = second_along ? 2048 >> 4 : 32 >> 4;  // 16 values of k
          const uint32_t id = kInstr | (first_along ? 1u << 15 : 0u) | (second_along ? 1u << 16 : 0u);
#pragma unroll
          for (int j = 0; j < kStepK / 16; ++j)
            pair_mma_f16(d, desc(first + on1 * j, kOperandHigh), desc(second + on2 * j, kOperandHigh), id, j > 0 || k > 0);
          pair_commit(empty(s));
        }
        if (++s == kStages) { s = 0; phase ^= 1; }
      }
      if (!ok) break;
      if (issue) pair_commit(acc_full(acc));
      if (++acc == 2) { acc = 0; acc_phase ^= 1; }
    }
    if (issue) {
      if (!ok) give_up(kErrCopy);
      pair_commit(drained);
    }
  } else if (warp >= 4) {
    const int quarter = warp & 3, half = (warp - 4) >> 2, who = warp - 4;
    const uint32_t places = smem + kStages * kStageBytes + who * kEpiBytes;
    int acc = 0;
    uint32_t acc_phase = 0, addend_phase = 0;
    for (int at = 0;; ++at) {
      NewtonTile t;
      if (!read_slot(at, t, true)) { if (lane == 0) give_up(kErrSlot); break; }
      if (t.matrix < 0) break;
      const NewtonMatrix& q = p.matrices[t.matrix];
      const int from = t.from();
      const int m = t.tm * kNewtonTile + (int)rank * 128 + quarter * 32, n0 = t.tn * kNewtonTile + half * 128;
      const int rows = q.r, cols = t.which() == 3 ? q.c : q.r, row0 = q.row0;
      const int patches = m < rows ? min(kPatches, (max(cols - n0, 0) + 63) / 64) : 0;
      const uint32_t sums = tmem + acc * kNewtonTile + half * 128 + ((uint32_t)(quarter * 32) << 16);
      const bool fetches = t.adds() && patches > 0;
      if (fetches && lane == 0) {  // (the places are free: the last tile's stores are done)
        fence_copies_global();
        mbar_arrive_tx(addend_full(who), patches * kPatchBytes);
        for (int b = 0; b < patches; ++b)
          tma_load_2d(places + b * kPatchBytes, t.which() == 2 ? &q.a_patch : &q.lo_patch, n0 + 64 * b, m, addend_full(who));
      }
      __syncwarp();
      bool ok = __all_sync(~0u, wait_cluster(acc_full(acc), acc_phase));
      if (fetches) {  // (seen to its end in any case: the copies are in flight)
        ok = __all_sync(~0u, mbar_wait(addend_full(who), addend_phase)) && ok;
        addend_phase ^= 1;
      }
      if (!ok) {
        if (lane == 0) give_up(kErrAcc);
        break;
      }
      tc_fence_after();
      auto freed = [&] {  // the sums are read
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(peer_addr(acc_free(acc), 0));
      };
      auto store = [&](const CUtensorMap* map, int b) {
        fence_for_copies();
        __syncwarp();
        if (lane == 0) {
          tma_store_2d(map, n0 + 64 * b, m, places + b * kPatchBytes);
          commit_stores();
        }
      };
      // 8 columns are 16 bytes of a row, in the copies' swizzle.
      auto place = [&](int b, int g) { return places + b * kPatchBytes + lane * 128 + (g ^ (lane & 7)) * 16; };
      auto make = [&](auto product, auto adding, auto keeping) {
        constexpr int kWhich = decltype(product)::value;
        constexpr bool kAdds = decltype(adding)::value, kKeepLo = decltype(keeping)::value;
        uint32_t rest[kPatches][32];
#pragma unroll
        for (int b = 0; b < kPatches; ++b) {
          if (b >= patches) break;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t r[32];
            tmem_load32(sums + 64 * b + 32 * h, r);
            tmem_wait_load();
            const bool diagonal = kWhich == 2 && n0 + 64 * b + 32 * h == m;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const uint32_t to = place(b, 4 * h + g);
              uint4 add = make_uint4(0, 0, 0, 0);
              if (kAdds) add = lds_v4(to);
              const uint32_t old[4] = {add.x, add.y, add.z, add.w};
              uint32_t sum[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const int k = 8 * g + 2 * j;
                float y0 = __fmul_rn(__uint_as_float(r[k]), kFromHeld), y1 = __fmul_rn(__uint_as_float(r[k + 1]), kFromHeld);
                const float2 a = of_half2(old[j]);
                if (kWhich == 2) {
                  y0 = __fmaf_rn(kC, y0, __fmul_rn(kB, a.x)), y1 = __fmaf_rn(kC, y1, __fmul_rn(kB, a.y));
                  if (diagonal) {
                    if (lane == k) y0 = __fadd_rn(y0, kA * kHeld);
                    if (lane == k + 1) y1 = __fadd_rn(y1, kA * kHeld);
                  }
                }
                if (kWhich == 3 && kAdds) y0 = __fmaf_rn(kA, a.x, y0), y1 = __fmaf_rn(kA, a.y, y1);
                sum[j] = half2_of(y0, y1);
                if (kKeepLo) {
                  const float2 held = of_half2(sum[j]);
                  rest[b][16 * h + 4 * g + j] = half2_of(__fsub_rn(y0, held.x), __fsub_rn(y1, held.y));
                }
              }
              sts_v4(to, sum);
            }
          }
          store(kWhich == 1 ? &q.a_patch : kWhich == 2 ? &q.b_patch : &q.x_patch[from ^ 1], b);
        }
        freed();
        if (kKeepLo) {  // X's second part takes the first's place once that has been read
#pragma unroll
          for (int b = 0; b < kPatches; ++b) {
            if (b >= patches) break;
            if (lane == 0) {
              if (b + 1 < patches) wait_for_reads<1>();
              else wait_for_reads<0>();
            }
            __syncwarp();
#pragma unroll
            for (int g = 0; g < 8; ++g) {
              const uint32_t some[4] = {rest[b][4 * g], rest[b][4 * g + 1], rest[b][4 * g + 2], rest[b][4 * g + 3]};
              sts_v4(place(b, g), some);
            }
            store(&q.lo_patch, b);
          }
        }
      };
      constexpr std::true_type yes;
      constexpr std::false_type no;
      if (t.which() == 1) make(std::integral_constant<int, 1>(), no, no);
      else if (t.which() == 2) make(std::integral_constant<int, 2>(), yes, no);
      else if (t.keep_lo()) make(std::integral_constant<int, 3>(), yes, yes);
      else if (t.adds()) make(std::integral_constant<int, 3>(), yes, no);
      else make(std::integral_constant<int, 3>(), no, no);
      if (lane == 0) {
        wait_for_stores();  // in memory now: its rows are that much further
        fence_copies_global();
        add_one_release(p.progress + row0 + t.tm);
        if (t.which() != 3 && t.tm != t.tn) add_one_release(p.progress + row0 + t.tn);
      }
      if (++acc == 2) { acc = 0; acc_phase ^= 1; }
    }
    if (lane == 0) wait_for_stores();
  }
  // The pair's end, the same whoever gave up, or nobody: any of the pair may have left its loop while what others asked for is in
  // flight.  Past the first barrier nobody asks for copies or products any more; memory goes past the second, when all
  // products are done (each CTA's own barrier has been arrived at) and all copies of operands have landed.  The epilogue's
  // warps have seen the ends of their own copies and stores.  (These waits are bounded too, by seconds: copies and products
  // end by themselves.)
  __syncwarp();
  tc_fence_before();
  cluster_sync();
  if (warp == 1) mbar_wait(drained, 0);
  if (warp == 0 && rank == 0 && lane == 0) {
    const volatile int32_t* by = asked;
    const int first = by[0], second = by[1], end = pair_end(first, second);
    for (int i = pair_open(first, second, kStages); i < end; ++i) {
      const PairStep what = pair_step(i, first, second);
      if (what == PairStep::kNoPeer) mbar_complete_tx(full(i % kStages), kStageTx / 2);
      if (what == PairStep::kNoLeader) mbar_arrive_tx(full(i % kStages), kStageTx / 2);
    }
    for (int i = pair_open(first, second, kStages); i < end; ++i) mbar_wait(full(i % kStages), (uint32_t)(i / kStages) & 1);
  }
  __syncwarp();
  cluster_sync();
  tc_fence_after();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

}  // namespace

cudaError_t launch_products(const ProductArgs& a, cudaStream_t stream) {
  static std::atomic<uint64_t> ready{0};
  const cudaError_t e = allow_smem((const void*)newton_kernel, kDynSmem, ready);
  if (e != cudaSuccess) return e;
  return launch_dependent((const void*)newton_kernel, 2 * (unsigned)std::min(a.count, kNewtonPairs), kProductThreads, 0, kDynSmem, &a, stream);
}

}  // namespace mpadam
