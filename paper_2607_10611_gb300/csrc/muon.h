// muon.h -- Newton-Schulz steps over a list of matrices and the Muon step around
// them: device tables and launch arguments (internal to the CUDA library; the C
// ABI is mpadam_orthogonal_* and mpadam_muon_* in include/mpadam.h).
//
// Every matrix is worked on lying down, [r, c] with r <= c (a tall one as its
// transpose), and held in FP16 times 2^14: X in two parts, a value's FP16 and the
// FP16 of what that leaves, A = X X^T and B = a I + b A + c A A in one.  The
// steps' polynomial keeps X's singular values, and so its values, below 1.21, A's
// below 1.45 and B's between 0.63 and 3.45, so nothing reaches 65504, and what
// lies below FP16's normal numbers is below 2^-28.  FP16 is as fast as BF16 on the tensor cores and
// rounds 8 times finer; X's second part, which only the sum a X takes, keeps the
// small singular values of matrices that a few large ones dominate: a 768 x 768
// of rank 32 and 1 % noise comes out with a relative error of 6e-4 after five
// steps, without the second part 2.2e-2, with BF16 0.18.
#pragma once

#include <cstddef>
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "adamw.h"

namespace mpadam {

constexpr float kHeld = 0x1p14f, kFromHeld = 0x1p-14f;

constexpr int kNewtonTile = 256;   // rows and columns of a product's tile, by a pair of CTAs
constexpr int kNewtonStepK = 64;   // values of k that are copied and multiplied at once
constexpr int kNewtonPairs = 76;   // GB300: two SMs each
constexpr int kTileRows = 64;      // rows and columns of a tile of the element-wise kernels
constexpr int kTileCols = 128;
constexpr int kSquaresPass = 8192; // elements that a block squares at once
constexpr int kMaxChunks = 1024;   // partial sums of a matrix's squares

// A matrix as the products see it.
struct alignas(128) NewtonMatrix {
  CUtensorMap x[2];    // X's first part before and after an odd step, A and B: a product's operands, boxes of 128 rows of 64
  CUtensorMap a, b;
  CUtensorMap x_along[2], a_along, b_along;            // the same where k runs along their columns: boxes of 64 x 64
  CUtensorMap x_patch[2], lo_patch, a_patch, b_patch;  // boxes of 32 rows of 64, what an epilogue's warp handles at once
  uint16_t* hi[2];     // X's first part, row stride ld
  uint16_t* lo;        // and its second
  uint16_t* ga;        // A and B, row stride lda
  uint16_t* gb;
  int64_t ld, lda;
  int32_t r, c;
  int32_t row0;        // its first counter: one for every 256 rows
};

// Its maps by their number.
constexpr int kNewtonMaps = 13;
static_assert(offsetof(NewtonMatrix, hi) == kNewtonMaps * sizeof(CUtensorMap), "nothing but maps before X's pointers");
__host__ __device__ inline const CUtensorMap* newton_map(const NewtonMatrix* q, int i) {
  return reinterpret_cast<const CUtensorMap*>(q) + i;
}

// Those that a tile of product `which` (1, 2, 3) copies by, where the step reads X `from`: operands as they lie and turned, the
// result, X's or A's part that is added to it (X's second part is stored too); fewer than kTileMaps come twice.
constexpr int kTileMaps = 5;
__host__ __device__ inline int tile_map(int which, int from, int i) {
  constexpr int kX = 0, kA = 2, kB = 3, kXAlong = 4, kAAlong = 6, kBAlong = 7, kXPatch = 8, kLoPatch = 10, kAPatch = 11, kBPatch = 12;
  if (which == 1) return i == 0 ? kX + from : kAPatch;
  if (which == 2) return i == 0 ? kA : i == 1 ? kAAlong : i == 2 ? kBPatch : kAPatch;
  return i == 0 ? kB : i == 1 ? kBAlong : i == 2 ? kXAlong + from : i == 3 ? kXPatch + (from ^ 1) : kLoPatch;
}

// A tile of a product: rows 256 tm and columns 256 tn of its result.
struct alignas(16) NewtonTile {
  int32_t matrix;
  uint16_t tm, tn;
  int32_t steps;   // of 64 values of k, times 32; and which product it is of (1, 2, 3), which X the step reads, whether something
                   // is added to the sums (A, X's second part), whether X's second part is stored
  uint32_t need;   // how far its operands' rows have to be: kSignals for every tile that was made of them

  static NewtonTile make(int32_t matrix, int tm, int tn, int steps, int which, int from, bool adds, bool keep_lo, uint32_t need) {
    return {matrix, (uint16_t)tm, (uint16_t)tn, steps << 5 | which << 3 | from << 2 | (int)adds << 1 | (int)keep_lo, need};
  }
  __host__ __device__ int steps_k() const { return steps >> 5; }
  __host__ __device__ int which() const { return steps >> 3 & 3; }
  __host__ __device__ int from() const { return steps >> 2 & 1; }
  __host__ __device__ bool adds() const { return steps >> 1 & 1; }
  __host__ __device__ bool keep_lo() const { return steps & 1; }
  // Products 2 and 3 read rows `tile` of A and B up to the diagonal's tile; from this step of k on, what lies above the
  // diagonal, they read what is below it, turned: k runs along its columns then.
  __host__ __device__ static int turned_from(int tile) { return (tile + 1) * (kNewtonTile / kNewtonStepK); }
};
constexpr uint32_t kSignals = 16;

// How a pair of CTAs that share operands in `stages` stages of shared memory ends.  Each CTA copies its half of a step's bytes,
// both halves to one barrier, on which the leader announces all of them as it asks for its own half.  When nobody asks for any
// more, CTA `rank` having asked for the first asked[rank] steps, every step before pair_open is whole (its stage was taken again)
// and the barriers of those from there on, a stage each, become whole once what will not come is made up for:
enum class PairStep { kWhole, kNoLeader, kNoPeer };  // both asked; the leader did not, so nothing is announced; the other CTA did not
__host__ __device__ inline int pair_end(int asked0, int asked1) { return asked0 > asked1 ? asked0 : asked1; }
__host__ __device__ inline int pair_open(int asked0, int asked1, int stages) {
  const int end = pair_end(asked0, asked1);
  return end > stages ? end - stages : 0;
}
__host__ __device__ inline PairStep pair_step(int step, int asked0, int asked1) {
  return step >= asked1 ? PairStep::kNoPeer : step >= asked0 ? PairStep::kNoLeader : PairStep::kWhole;
}

struct ProductArgs {
  const NewtonMatrix* matrices;  // the list's
  int32_t first;                 // the first one that the tiles belong to
  const NewtonTile* tiles;
  int32_t count;
  uint32_t* progress;  // of every 256 rows; 0 when the launch begins, and so is
  uint32_t* taken;     // the number of tiles that were taken
  int32_t* err;
};

// All products of the list: A = X X^T, B = a I + b A + c A A, X = B X and a times X's second part, step after step.
cudaError_t launch_products(const ProductArgs& a, cudaStream_t stream);

// A matrix as the element-wise kernels see it.
struct MuonMatrix {
  void* w;             // [rows, cols], or nullptr (orthogonalisation alone)
  void* m;
  uint16_t* compute;   // or nullptr
  uint16_t* hi[2];     // the products' X, transposed where tall
  uint16_t* lo;
  int64_t ld;
  int64_t goff;        // global index of element 0
  int64_t chunk0;      // its first partial sum
  int32_t chunks;
  int32_t chunk;       // elements of each (the last may have fewer)
  int32_t rows, cols;
  int32_t tile0;       // its first tile among the group's
  int32_t tiles_across;
  int32_t index;       // in the caller's list
  int32_t tall;
  float factor;        // of the learning rate
  uint32_t aligned;    // w, m and compute on 16-byte boundaries
};

// 1 / |U| times 2^14, as three factors that take a value of U to X's without
// leaving binary32's range on the way; and the chunks whose squares are summed (0
// between launches).
struct MuonNorm {
  float down0, down1, rest;
  uint32_t done;
};

struct MuonArgs {
  const MuonMatrix* matrices;
  const int32_t* owner;      // the matrix of each tile, or of each chunk
  int32_t count;
  double* partial;           // sums of squares, a chunk each
  MuonNorm* norms;           // of each matrix
  const float* grad_scale;   // or nullptr
  int32_t* err;              // the products' error word
  uint32_t* progress;        // the products' counters, which begin clears: `counters` of them
  int32_t counters;
  float beta, rest, lr, decay;
  int32_t nesterov, last;    // last: which X holds the result
  int64_t step;
  uint32_t rk0[kPhiloxRounds], rk1[kPhiloxRounds];
  GradTable in;              // gradients, or the matrices themselves
  GradTable out;             // where those go
};

struct MuonKind {
  bool step;                 // a Muon step; else orthogonalisation alone
  bool in_f32, m_f32, w_f32, stochastic;
};

cudaError_t launch_squares(const MuonArgs& a, const MuonKind& k, cudaStream_t stream);  // owner: of chunks
cudaError_t launch_begin(const MuonArgs& a, const MuonKind& k, cudaStream_t stream);    // of tiles, as below
cudaError_t launch_finish(const MuonArgs& a, const MuonKind& k, cudaStream_t stream);

}  // namespace mpadam
