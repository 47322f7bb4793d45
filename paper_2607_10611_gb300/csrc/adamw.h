// adamw.h -- launch arguments of the AdamW step and of the gradient norm over a
// list of tensors (internal to the CUDA library; the C ABI is mpadam_adamw_* and
// mpadam_grad_norm_* in include/mpadam.h).
#pragma once

#include <cstdint>
#include <cuda_runtime.h>

#include "step_args.h"

namespace mpadam {

// Elements per tile; a tensor's last tile may be short.  A CTA takes a tile of a
// step (of this size by the moments' type), a warp one of the norm.
constexpr int adamw_tile(bool state_e4m3) { return state_e4m3 ? 2816 : 3840; }
constexpr uint32_t kPhiloxM0 = 0xD2511F53u, kPhiloxM1 = 0xCD9E8D57u;
constexpr int kNormTile = 2048;
constexpr int kInlineGrads = 448;    // gradient pointers that travel with one launch

// One tensor of the list. Its tiles are tile0, tile0 + 1, ...
struct ListTensor {
  void* w;
  void* m;
  void* v;
  uint8_t* m_scale;
  uint8_t* v_scale;
  uint16_t* compute;
  int64_t numel;
  int64_t goff;     // global index of element 0 (a multiple of 128)
  int64_t tile0;
  uint32_t aligned; // 1: every pointer is a multiple of 16 bytes; 4: w, m, v of 32
  uint32_t pad;
};

// Gradient pointers: in the launch itself, or (grads != nullptr) in device memory.
struct GradTable {
  const void* const* grads;
  const void* inline_grads[kInlineGrads];
};

struct AdamwScalars {
  float b1, b2, omb1, omb2, ka, c2, eps, kwd;
};

struct AdamwArgs {
  const ListTensor* tensors;
  const int32_t* tile_tensor;  // [tiles] the tensor each tile belongs to
  int64_t tiles;
  AdamwScalars s;
  uint64_t minus_zero;         // two binary32 -0 (see prod2)
  int32_t plain;               // eps and betas are in fast_update's range
  const float* grad_scale;     // device multiplier of the gradients, or nullptr
  int32_t* err;                // device error word
  uint32_t rk0[kPhiloxRounds], rk1[kPhiloxRounds];
  // the first Philox round's share of step t: the high word of t_lo M1 and t_hi, each with the round's key, and the low
  // word with the next round's
  uint32_t round1[3];
  GradTable g;
};

struct AdamwKind {
  bool w_f32, g_f32, state_e4m3, sr, state_sr;
};

// Makes the kernel of this kind ready on the current device (and counts its SMs), and launches it.
cudaError_t prepare_adamw(const AdamwKind& k, int32_t* sms);
cudaError_t launch_adamw(const AdamwArgs& a, const AdamwKind& k, int32_t sms, cudaStream_t stream);

struct NormArgs {
  const ListTensor* tensors;
  const int32_t* tile_tensor;
  int64_t tiles;
  double* partial;       // [ctas] of the launch
  uint32_t* done;        // CTAs that have written theirs; 0 between launches
  float* out;            // norm, multiplier
  float max_norm;
  int32_t g_f32;
  GradTable g;
};

constexpr int kNormCtas = 152 * 5;
cudaError_t launch_grad_norm(const NormArgs& a, cudaStream_t stream);

// Copies count gradient pointers into a device table at `first`.
cudaError_t fill_grads(const void** table, const void* const* grads, int32_t first, int32_t count, cudaStream_t stream);

}  // namespace mpadam
