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

#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "adamw.h"

namespace mpadam {

constexpr float kHeld = 0x1p14f, kFromHeld = 0x1p-14f;

constexpr int kNewtonTile = 256;   // rows and columns of a product's tile, by a pair of CTAs
constexpr int kElementTile = 64;   // rows and columns of a tile of the element-wise kernels
constexpr int kSquaresPass = 16384; // elements that a block squares at once
constexpr int kMaxChunks = 1024;   // partial sums of a matrix's squares

// A matrix as the products see it.
struct alignas(128) NewtonMatrix {
  CUtensorMap x[2];    // X before and after an odd step, boxes of 64 x 64
  CUtensorMap a, b;
  uint16_t* hi[2];     // X's first part, row stride ld
  uint16_t* lo;        // and its second
  uint16_t* ga;        // A and B, row stride lda
  uint16_t* gb;
  int64_t ld, lda;
  int32_t r, c;
};

struct NewtonTile {
  int32_t matrix, tm, tn, pad;
};

struct ProductArgs {
  const NewtonMatrix* matrices;
  const NewtonTile* tiles;
  int32_t count;
  int32_t from;        // which of a matrix's two X the step reads
  int32_t keep_lo;     // the third product writes X's second part
  int32_t use_lo;      // and reads it
  int32_t* err;
};

// The three products of a step: A = X X^T, B = a I + b A + c A A, X = B X and a times X's second part.
cudaError_t launch_product(int which, const ProductArgs& a, cudaStream_t stream);

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
