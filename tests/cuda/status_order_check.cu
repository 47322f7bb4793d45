// Test-only host program: the calls that a status function of STATUS_SOURCE (which this file includes), or one that sets how a
// state launches, makes of the runtime, here by fakes that write down what they were asked for; one a line.  The error word reads as 4.
#include <cstdio>
#include <string>
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

namespace {

int32_t word = 0;

int32_t run(const std::string& of, int32_t* code) {
#if defined(OF_muon_api)
  static mpadam_orthogonal_state orthogonal;
  static mpadam_muon_state muon;
  orthogonal.newton.args.err = muon.newton.args.err = &word;
  if (of == "orthogonal") return mpadam_orthogonal_status(&orthogonal, code);
  if (of == "muon") return mpadam_muon_status(&muon, code);
#elif defined(OF_train_api)
  static mpadam_adamw_state adamw;
  adamw.args.err = &word;
  if (of == "adamw") return mpadam_adamw_status(&adamw, code);
#else
  static mpadam_state state;
  static mpadam_toy_state toy;
  state.d_err = toy.a.err = &word;
  if (of == "step") return mpadam_device_status(&state, code);
  if (of == "toy") return mpadam_toy_status(&toy, code);
  *code = 4;
  if (of == "grid") return mpadam_set_grid(&state, 8);
  if (of == "pool") return mpadam_set_tail_pool(&state, 512, 4);
#endif
  return -1;
}

}  // namespace

int main(int, char** argv) {
  int32_t code = 0;
  const int32_t rc = run(argv[1], &code);
  std::printf("returned %d, code %d\n", rc, code);
}
