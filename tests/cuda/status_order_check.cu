// Test-only host program: the calls that a status function of STATUS_SOURCE (which this file includes) makes of the runtime,
// here by fakes that write down what they were asked for; one a line.  The error word reads as 4.
#include <cstdio>
#include <cuda_runtime.h>

namespace fakes {
inline cudaError_t said(const char* what) {
  std::printf("%s\n", what);
  return cudaSuccess;
}
inline cudaError_t device(int* d) {
  *d = 0;
  return cudaSuccess;
}
inline cudaError_t copied(void* to, size_t bytes, cudaMemcpyKind kind) {
  if (kind == cudaMemcpyDeviceToHost && bytes == sizeof(int32_t)) *static_cast<int32_t*>(to) = 4;
  return said("copy");
}
}  // namespace fakes

#define cudaGetDevice(d) fakes::device(d)
#define cudaDeviceSynchronize() fakes::said("wait for the device")
#define cudaStreamSynchronize(stream) fakes::said((stream) == cudaStreamLegacy ? "wait for the legacy stream" : "wait for a stream")
#define cudaMemcpy(to, from, bytes, kind) fakes::copied(to, bytes, kind)
#define cudaMemset(p, value, bytes) fakes::said("clear")
#define cudaFree(p) ((void)(p))
#include STATUS_SOURCE

int main() {
  int32_t code = 0, word = 0;
  (void)word;
  int32_t rc = 1;
#if defined(OF_ORTHOGONAL)
  static mpadam_orthogonal_state s;
  s.newton.args.err = &word;
  rc = mpadam_orthogonal_status(&s, &code);
#elif defined(OF_MUON)
  static mpadam_muon_state s;
  s.newton.args.err = &word;
  rc = mpadam_muon_status(&s, &code);
#endif
  std::printf("returned %d, code %d\n", rc, code);
}
