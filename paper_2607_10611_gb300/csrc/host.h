// host.h -- what the host-side translation units share: the last error's
// message, and the allocations that tests can make fail (internal to the CUDA
// library; defined in mpadam_api.cu).
#pragma once

#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

#include "mpadam.h"

namespace mpadam {

// Records the message of this host thread's last error; returns code.
int32_t fail(int32_t code, const char* fmt, ...);
int32_t cuda_fail(cudaError_t e, const char* what);

// Every device and pinned allocation of the library goes through these.
cudaError_t dev_malloc(void** p, size_t bytes);
template <typename T>
cudaError_t dev_malloc(T** p, size_t bytes) {
  return dev_malloc(reinterpret_cast<void**>(p), bytes);
}

// a: a power of two
inline bool is_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Philox4x32-10 round keys: key + r * (0x9E3779B9, 0xBB67AE85), r = 0..9.
void round_keys(uint64_t seed, uint32_t* rk0, uint32_t* rk1);

}  // namespace mpadam
