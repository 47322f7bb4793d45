// list.h -- what the host sides of the list operators share: the device they
// were made on, their tables of pointers, and the driver's entry for tensor maps
// (internal to the CUDA library).
#pragma once

#include <algorithm>
#include <cstring>
#include <cuda.h>
#include <vector>

#include "adamw.h"
#include "host.h"

namespace mpadam {

inline int32_t check_device(int device) {
  int dev = -1;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
  if (dev != device) return fail(MPADAM_EINVAL, "current device %d differs from the state's device %d", dev, device);
  return MPADAM_OK;
}

// Pointers that come with every call: in the launch, or through a device table
// where there are more than kInlineGrads.
struct PointerTable {
  const void** table = nullptr;   // on the device, as many as the list has tensors (not used for short lists)
  std::vector<const void*> last;  // what it holds
  bool last_known = false, captured = false;

  // Pointers for a launch on `stream`: with it, or through the device table,
  // refilled when they changed.  A replayed graph fills the table as it was
  // captured, so once a fill was captured the table's content is not known.
  int32_t for_launch(GradTable* g, const void* const* pointers, int32_t n, cudaStream_t stream) {
    g->grads = nullptr;
    if (n <= kInlineGrads) {
      std::memcpy(g->inline_grads, pointers, sizeof(void*) * n);
      return MPADAM_OK;
    }
    g->grads = table;
    cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(stream, &st);
    if (e != cudaSuccess) return cuda_fail(e, "cudaStreamIsCapturing");
    if (st != cudaStreamCaptureStatusNone) captured = true;
    if (!captured && last_known && std::memcmp(last.data(), pointers, sizeof(void*) * n) == 0) return MPADAM_OK;
    last_known = false;
    for (int32_t i = 0; i < n; i += kInlineGrads) {
      e = fill_grads(table, pointers + i, i, std::min(kInlineGrads, n - i), stream);
      if (e != cudaSuccess) return cuda_fail(e, "launch of the pointer table's fill");
    }
    last.assign(pointers, pointers + n);
    last_known = true;
    return MPADAM_OK;
  }
};

using EncodeTiled = decltype(&cuTensorMapEncodeTiled);

// The driver's function, or nullptr.
inline EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

}  // namespace mpadam
