// train_api.cu -- host side of mpadam_adamw_*, mpadam_grad_norm_* and
// mpadam_e4m3_* (include/mpadam.h).
#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>
#include <vector>

#include "adamw.h"
#include "fp8.h"
#include "host.h"

using namespace mpadam;

namespace {

int32_t check_device(int device) {
  int dev = -1;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
  if (dev != device) return fail(MPADAM_EINVAL, "current device %d differs from the state's device %d", dev, device);
  return MPADAM_OK;
}

// What both list operators keep on the device: the tensors, each tile's tensor,
// and gradient pointers where they do not fit a launch.
struct List {
  int device = 0;
  int32_t n = 0;
  int64_t tiles = 0;
  size_t grad_size = 4;
  std::vector<int64_t> numel;
  uint8_t* memory = nullptr;  // one allocation: the tables below, then what the operator asked for, zeroed
  ListTensor* d_tensors = nullptr;
  int32_t* d_tile_tensor = nullptr;
  const void** d_grads = nullptr;
  void* extra = nullptr;
  std::vector<const void*> last;  // what d_grads holds
  bool last_known = false, captured = false;

  List() = default;
  List(const List&) = delete;
  ~List() { cudaFree(memory); }

  int32_t build(std::vector<ListTensor>& t, int32_t tile, size_t extra_bytes) {
    n = (int32_t)t.size();
    int64_t goff = 0;
    for (auto& x : t) {
      // checked before it is rounded up, and the sum after each: nothing here overflows
      const int64_t own = x.numel <= (int64_t)INT32_MAX * tile ? (x.numel + tile - 1) / tile : INT32_MAX;
      if (tiles + own >= INT32_MAX) return fail(MPADAM_EINVAL, "the list has too many elements");
      x.goff = goff;
      x.tile0 = tiles;
      goff += (x.numel + 127) / 128 * 128;
      tiles += own;
      numel.push_back(x.numel);
    }
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    auto pad = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t tensors_at = 0, extra_at = pad(sizeof(ListTensor) * n), owner_at = extra_at + pad(extra_bytes);
    const size_t upload = owner_at + sizeof(int32_t) * tiles, grads_at = pad(upload);
    const size_t bytes = grads_at + (n > kInlineGrads ? sizeof(void*) * n : 0);
    std::vector<uint8_t> host(upload);
    if (n) std::memcpy(host.data() + tensors_at, t.data(), sizeof(ListTensor) * n);
    int32_t* owner = reinterpret_cast<int32_t*>(host.data() + owner_at);
    for (int32_t k = 0; k < n; ++k) std::fill_n(owner + t[k].tile0, (t[k].numel + tile - 1) / tile, k);
    if (dev_malloc(&memory, std::max<size_t>(bytes, 256)) != cudaSuccess) {
      memory = nullptr;
      cudaGetLastError();
      return fail(MPADAM_EALLOC, "allocation of the list's tables failed");
    }
    if (upload) {
      e = cudaMemcpy(memory, host.data(), upload, cudaMemcpyHostToDevice);
      // a copy from pageable memory may return before it has arrived, and steps run on any stream
      if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);
      if (e != cudaSuccess) return cuda_fail(e, "upload of the list's tables");
    }
    d_tensors = reinterpret_cast<ListTensor*>(memory + tensors_at);
    d_tile_tensor = reinterpret_cast<int32_t*>(memory + owner_at);
    d_grads = reinterpret_cast<const void**>(memory + grads_at);
    extra = memory + extra_at;
    return MPADAM_OK;
  }

  int32_t check_grads(const void* const* grads) const {
    if (!grads) return fail(MPADAM_EINVAL, "grads is NULL");
    for (int32_t k = 0; k < n; ++k) {
      if (numel[k] == 0) continue;
      if (!grads[k]) return fail(MPADAM_EINVAL, "grads[%d] is NULL", k);
      if (!is_aligned(grads[k], grad_size)) return fail(MPADAM_EINVAL, "grads[%d] not aligned to its element size", k);
    }
    return MPADAM_OK;
  }

  // Gradient pointers for a launch on `stream`: with it, or through the device
  // table, refilled when they changed.  A replayed graph fills the table as it
  // was captured, so once a fill was captured the table's content is not known.
  int32_t grads_for(GradTable* g, const void* const* grads, cudaStream_t stream) {
    g->grads = nullptr;
    if (n <= kInlineGrads) {
      std::memcpy(g->inline_grads, grads, sizeof(void*) * n);
      return MPADAM_OK;
    }
    g->grads = d_grads;
    cudaStreamCaptureStatus st = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(stream, &st);
    if (e != cudaSuccess) return cuda_fail(e, "cudaStreamIsCapturing");
    if (st != cudaStreamCaptureStatusNone) captured = true;
    if (!captured && last_known && std::memcmp(last.data(), grads, sizeof(void*) * n) == 0) return MPADAM_OK;
    last_known = false;
    for (int32_t i = 0; i < n; i += kInlineGrads) {
      e = fill_grads(d_grads, grads + i, i, std::min(kInlineGrads, n - i), stream);
      if (e != cudaSuccess) return cuda_fail(e, "launch of the gradient table's fill");
    }
    last.assign(grads, grads + n);
    last_known = true;
    return MPADAM_OK;
  }
};

}  // namespace

struct mpadam_adamw_state {
  List list;
  mpadam_adamw_config cfg;
  AdamwKind kind;
  int32_t sms = 0;
  AdamwArgs args{};
};
struct mpadam_grad_norm_state {
  List list;
  NormArgs args{};
};

extern "C" int32_t mpadam_adamw_create(const mpadam_adamw_tensor* tensors, int32_t n, const mpadam_adamw_config* cfg,
                                       mpadam_adamw_state** out) {
  if (!out) return fail(MPADAM_EINVAL, "out is NULL");
  *out = nullptr;
  if (!cfg) return fail(MPADAM_EINVAL, "config is NULL");
  if (n < 0) return fail(MPADAM_EINVAL, "n must be >= 0");
  if (n > 0 && !tensors) return fail(MPADAM_EINVAL, "tensors is NULL");
  const mpadam_adamw_config& c = *cfg;
  auto f32_or = [](int32_t x, int32_t other) { return x == MPADAM_F32 || x == other; };
  if (!f32_or(c.weight_dtype, MPADAM_BF16)) return fail(MPADAM_EINVAL, "weight_dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", c.weight_dtype);
  if (!f32_or(c.grad_dtype, MPADAM_BF16)) return fail(MPADAM_EINVAL, "grad_dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", c.grad_dtype);
  if (!f32_or(c.state_dtype, MPADAM_E4M3)) return fail(MPADAM_EINVAL, "state_dtype must be MPADAM_F32 or MPADAM_E4M3 (got %d)", c.state_dtype);
  for (int32_t r : {c.rounding, c.state_rounding})
    if (r != MPADAM_ROUND_NEAREST && r != MPADAM_ROUND_STOCHASTIC)
      return fail(MPADAM_EINVAL, "rounding must be nearest (0) or stochastic (1) (got %d)", r);
  if (c.state_rounding == MPADAM_ROUND_STOCHASTIC && c.state_dtype != MPADAM_E4M3)
    return fail(MPADAM_EINVAL, "stochastic state rounding is for E4M3 states");
  if (c.reserved != 0) return fail(MPADAM_EINVAL, "reserved must be 0");
  if (!(c.beta1 >= 0.0f && c.beta1 < 1.0f)) return fail(MPADAM_EINVAL, "beta1 must be in [0, 1)");
  if (!(c.beta2 >= 0.0f && c.beta2 < 1.0f)) return fail(MPADAM_EINVAL, "beta2 must be in [0, 1)");
  if (!(std::isfinite(c.eps) && c.eps > 0.0f)) return fail(MPADAM_EINVAL, "eps must be finite and > 0");
  if (!(std::isfinite(c.weight_decay) && c.weight_decay >= 0.0f)) return fail(MPADAM_EINVAL, "weight_decay must be finite and >= 0");
  const size_t wsz = c.weight_dtype == MPADAM_F32 ? 4 : 2, ssz = c.state_dtype == MPADAM_F32 ? 4 : 1;
  try {
    std::vector<ListTensor> list((size_t)n);
    for (int32_t k = 0; k < n; ++k) {
      const mpadam_adamw_tensor& t = tensors[k];
      ListTensor& x = list[k];
      if (t.numel < 0) return fail(MPADAM_EINVAL, "tensor %d has a negative size", k);
      x = {t.w, t.m, t.v, t.m_scale, t.v_scale, t.compute, t.numel, 0, 0, 0, 0};
      if (c.state_dtype == MPADAM_F32 && (t.m_scale || t.v_scale)) return fail(MPADAM_EINVAL, "tensor %d: binary32 moments have no scales", k);
      if (t.compute && c.weight_dtype != MPADAM_F32) return fail(MPADAM_EINVAL, "tensor %d: a compute copy is for binary32 weights", k);
      if (t.numel == 0) continue;
      if (!t.w || !t.m || !t.v) return fail(MPADAM_EINVAL, "tensor %d has a NULL pointer", k);
      if (c.state_dtype == MPADAM_E4M3 && (!t.m_scale || !t.v_scale)) return fail(MPADAM_EINVAL, "tensor %d: 8-bit moments need their scales", k);
      if (!is_aligned(t.w, wsz) || !is_aligned(t.m, ssz) || !is_aligned(t.v, ssz) || !is_aligned(t.compute, 2))
        return fail(MPADAM_EINVAL, "tensor %d: a pointer is not aligned to its element size", k);
      x.aligned = (is_aligned(t.w, 16) && is_aligned(t.m, 16) && is_aligned(t.v, 16) && is_aligned(t.compute, 16) ? 1u : 0u) |
                  (is_aligned(t.w, 32) && is_aligned(t.m, 32) && is_aligned(t.v, 32) ? 4u : 0u);
    }
    std::unique_ptr<mpadam_adamw_state> s(new mpadam_adamw_state());
    s->cfg = c;
    s->list.grad_size = c.grad_dtype == MPADAM_F32 ? 4 : 2;
    const int32_t rc = s->list.build(list, adamw_tile(c.state_dtype == MPADAM_E4M3), sizeof(int32_t));
    if (rc) return rc;
    s->kind = {c.weight_dtype == MPADAM_F32, c.grad_dtype == MPADAM_F32, c.state_dtype == MPADAM_E4M3,
               c.rounding == MPADAM_ROUND_STOCHASTIC, c.state_rounding == MPADAM_ROUND_STOCHASTIC};
    const cudaError_t e = prepare_adamw(s->kind, &s->sms);
    if (e != cudaSuccess) return cuda_fail(e, "preparing the AdamW step");
    s->args.err = static_cast<int32_t*>(s->list.extra);
    s->args.tensors = s->list.d_tensors;
    s->args.tile_tensor = s->list.d_tile_tensor;
    s->args.tiles = s->list.tiles;
    s->args.minus_zero = 0x8000000080000000ull;
    round_keys(c.seed, s->args.rk0, s->args.rk1);
    *out = s.release();
  } catch (const std::bad_alloc&) {
    return fail(MPADAM_EALLOC, "host allocation failed");
  }
  return MPADAM_OK;
}

extern "C" int32_t mpadam_adamw_step(mpadam_adamw_state* s, const void* const* grads, int64_t step, float lr,
                                     const float* grad_scale, cudaStream_t stream) {
  if (!s) return fail(MPADAM_EINVAL, "state is NULL");
  if (step < 1) return fail(MPADAM_EINVAL, "step must be >= 1 (got %lld)", (long long)step);
  if (!(std::isfinite(lr) && lr >= 0.0f)) return fail(MPADAM_EINVAL, "lr must be finite and >= 0");
  if (!is_aligned(grad_scale, 4)) return fail(MPADAM_EINVAL, "grad_scale misaligned");
  if (s->list.tiles == 0) return MPADAM_OK;
  int32_t rc = s->list.check_grads(grads);
  if (rc) return rc;
  rc = check_device(s->list.device);
  if (rc) return rc;
  try {
    rc = s->list.grads_for(&s->args.g, grads, stream);
  } catch (const std::bad_alloc&) {
    return fail(MPADAM_EALLOC, "host allocation failed");
  }
  if (rc) return rc;
  const mpadam_adamw_config& c = s->cfg;
  const double b1 = c.beta1, b2 = c.beta2, t = (double)step;
  AdamwScalars& q = s->args.s;
  q.b1 = c.beta1;
  q.b2 = c.beta2;
  q.omb1 = (float)(1.0 - b1);
  q.omb2 = (float)(1.0 - b2);
  q.ka = (float)((double)lr / (1.0 - std::pow(b1, t)));
  q.c2 = (float)(1.0 / std::sqrt(1.0 - std::pow(b2, t)));
  q.eps = c.eps;
  q.kwd = (float)((double)lr * (double)c.weight_decay);
  // r' < 2^16 on the fast path: denominators lie in [2^-100, 2^25], and quotients of 2^-100 and more are not subnormal
  // betas of 2^-30 and more keep all their bits when old scales (2^-47 at least; the root's enters squared) go into them
  auto holds = [](float beta) { return beta == 0.0f || beta >= 0x1p-30f; };
  s->args.plain = c.eps >= 0x1p-100f && c.eps <= 0x1p20f && q.c2 <= 0x1p8f && holds(c.beta1) && holds(c.beta2);
  s->args.grad_scale = grad_scale;
  const uint64_t first = (uint64_t)(uint32_t)step * kPhiloxM1;
  s->args.round1[0] = (uint32_t)(first >> 32) ^ s->args.rk0[0];
  s->args.round1[1] = (uint32_t)((uint64_t)step >> 32) ^ s->args.rk1[0];
  s->args.round1[2] = (uint32_t)first ^ s->args.rk0[1];
  const cudaError_t e = launch_adamw(s->args, s->kind, s->sms, stream);
  if (e != cudaSuccess) return cuda_fail(e, "launch of the AdamW step");
  return MPADAM_OK;
}

extern "C" int32_t mpadam_adamw_status(mpadam_adamw_state* s, int32_t* code) {
  if (!s || !code) return fail(MPADAM_EINVAL, "state or code is NULL");
  *code = 0;
  const int32_t rc = check_device(s->list.device);
  if (rc) return rc;
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(code, s->args.err, sizeof(int32_t), cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && *code) e = cudaMemset(s->args.err, 0, sizeof(int32_t));
  return e == cudaSuccess ? MPADAM_OK : cuda_fail(e, "reading the error word");
}

extern "C" int32_t mpadam_adamw_destroy(mpadam_adamw_state* s) {
  if (!s) return MPADAM_OK;
  cudaDeviceSynchronize();
  delete s;
  return MPADAM_OK;
}

extern "C" int32_t mpadam_grad_norm_create(const int64_t* numel, int32_t n, int32_t grad_dtype, mpadam_grad_norm_state** out) {
  if (!out) return fail(MPADAM_EINVAL, "out is NULL");
  *out = nullptr;
  if (n < 0) return fail(MPADAM_EINVAL, "n must be >= 0");
  if (n > 0 && !numel) return fail(MPADAM_EINVAL, "numel is NULL");
  if (grad_dtype != MPADAM_F32 && grad_dtype != MPADAM_BF16)
    return fail(MPADAM_EINVAL, "grad_dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", grad_dtype);
  try {
    std::vector<ListTensor> list((size_t)n);
    for (int32_t k = 0; k < n; ++k) {
      if (numel[k] < 0) return fail(MPADAM_EINVAL, "tensor %d has a negative size", k);
      list[k] = ListTensor{};
      list[k].numel = numel[k];
    }
    std::unique_ptr<mpadam_grad_norm_state> s(new mpadam_grad_norm_state());
    s->list.grad_size = grad_dtype == MPADAM_F32 ? 4 : 2;
    // the partial sums, and the count of CTAs behind them
    const int32_t rc = s->list.build(list, kNormTile, sizeof(double) * (kNormCtas + 1));
    if (rc) return rc;
    NormArgs& a = s->args;
    a.partial = static_cast<double*>(s->list.extra);
    a.done = reinterpret_cast<uint32_t*>(a.partial + kNormCtas);
    a.tensors = s->list.d_tensors;
    a.tile_tensor = s->list.d_tile_tensor;
    a.tiles = s->list.tiles;
    a.g_f32 = grad_dtype == MPADAM_F32;
    *out = s.release();
  } catch (const std::bad_alloc&) {
    return fail(MPADAM_EALLOC, "host allocation failed");
  }
  return MPADAM_OK;
}

extern "C" int32_t mpadam_grad_norm(mpadam_grad_norm_state* s, const void* const* grads, float max_norm, float* out,
                                    cudaStream_t stream) {
  if (!s) return fail(MPADAM_EINVAL, "state is NULL");
  if (!out || !is_aligned(out, 4)) return fail(MPADAM_EINVAL, "out NULL or misaligned");
  if (!(max_norm > 0.0f)) return fail(MPADAM_EINVAL, "max_norm must be > 0 (+inf = never clip)");
  int32_t rc = s->list.tiles ? s->list.check_grads(grads) : MPADAM_OK;
  if (rc) return rc;
  rc = check_device(s->list.device);
  if (rc) return rc;
  if (s->list.tiles) {
    try {
      rc = s->list.grads_for(&s->args.g, grads, stream);
    } catch (const std::bad_alloc&) {
      return fail(MPADAM_EALLOC, "host allocation failed");
    }
    if (rc) return rc;
  }
  s->args.max_norm = max_norm;
  s->args.out = out;
  const cudaError_t e = launch_grad_norm(s->args, stream);
  if (e != cudaSuccess) return cuda_fail(e, "launch of the gradient norm");
  return MPADAM_OK;
}

extern "C" int32_t mpadam_grad_norm_destroy(mpadam_grad_norm_state* s) {
  if (!s) return MPADAM_OK;
  cudaDeviceSynchronize();
  delete s;
  return MPADAM_OK;
}

extern "C" int32_t mpadam_e4m3_quantize(const void* x, int32_t x_dtype, int64_t rows, int64_t cols, int64_t ld,
                                        int32_t square, uint8_t* q, uint8_t* s, int64_t ldq, uint8_t* qt, uint8_t* st,
                                        int64_t ldqt, cudaStream_t stream) {
  if (x_dtype != MPADAM_F32 && x_dtype != MPADAM_BF16)
    return fail(MPADAM_EINVAL, "x_dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", x_dtype);
  if (rows < 0 || cols < 0 || rows > INT32_MAX || cols > INT32_MAX) return fail(MPADAM_EINVAL, "rows and cols must be in [0, 2^31)");
  if (ld < cols) return fail(MPADAM_EINVAL, "ld must be >= cols");
  if (square != 0 && square != 1) return fail(MPADAM_EINVAL, "square must be 0 or 1");
  if (rows == 0 || cols == 0) return MPADAM_OK;
  if (!q && !qt) return fail(MPADAM_EINVAL, "q and qt are both NULL");
  if (!x || !is_aligned(x, x_dtype == MPADAM_F32 ? 4 : 2)) return fail(MPADAM_EINVAL, "x NULL or misaligned");
  if (q && (!s || !is_aligned(q, 16) || !is_aligned(s, 16) || ldq < cols || ldq % 16))
    return fail(MPADAM_EINVAL, "q, s must be 16-byte aligned and ldq a multiple of 16, >= cols");
  if (qt && (!st || !is_aligned(qt, 16) || !is_aligned(st, 16) || ldqt < rows || ldqt % 16))
    return fail(MPADAM_EINVAL, "qt, st must be 16-byte aligned and ldqt a multiple of 16, >= rows");
  if ((rows + 127) / 128 * ((cols + 127) / 128) > INT32_MAX) return fail(MPADAM_EINVAL, "the matrix has too many tiles");
  const QuantArgs a{x, rows, cols, ld, q, s, qt, st, ldq, ldqt, x_dtype == MPADAM_F32, square};
  const cudaError_t e = launch_quantize(a, stream);
  if (e != cudaSuccess) return cuda_fail(e, "launch of the quantisation");
  return MPADAM_OK;
}

namespace {

constexpr int64_t kMatmulMax = INT32_MAX - 1023;  // the kernels round sizes up to tiles in 32 bits

using EncodeTiled = decltype(&cuTensorMapEncodeTiled);

EncodeTiled encode_tiled() {
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

// Tensor map of scales, [row tiles, groups, 128 words], boxes of `box` row tiles of one group.
bool scale_map(CUtensorMap* map, const uint8_t* s, int64_t rows, int64_t k, int box) {
  const cuuint64_t groups = (cuuint64_t)(k + 511) / 512;
  const cuuint64_t dims[3] = {128, groups, (cuuint64_t)(rows + 127) / 128}, strides[2] = {kScaleTile, kScaleTile * groups};
  const cuuint32_t boxes[3] = {128, 1, (cuuint32_t)box}, steps[3] = {1, 1, 1};
  return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<uint8_t*>(s), dims, strides, boxes, steps,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tensor map of codes [rows, k], row stride ld bytes, boxes of `box` rows x 128 bytes in the 128-byte swizzle.
bool code_map(CUtensorMap* map, const uint8_t* q, int64_t rows, int64_t k, int64_t ld, int box) {
  const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t boxes[2] = {128, (cuuint32_t)box}, steps[2] = {1, 1};
  return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(q), dims, strides, boxes, steps,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

namespace {

// A product's arguments.
int32_t check_product(const mpadam_e4m3_product* p) {
  if (!p) return fail(MPADAM_EINVAL, "product is NULL");
  if (p->m < 0 || p->n < 0 || p->k < 0 || p->m > kMatmulMax || p->n > kMatmulMax || p->k > kMatmulMax)
    return fail(MPADAM_EINVAL, "m, n and k must be in [0, 2^31 - 1024]");
  if (p->d_dtype != MPADAM_F32 && p->d_dtype != MPADAM_BF16)
    return fail(MPADAM_EINVAL, "d_dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", p->d_dtype);
  if (p->accumulate != 0 && p->accumulate != 1) return fail(MPADAM_EINVAL, "accumulate must be 0 or 1");
  if (p->accumulate && p->d_dtype != MPADAM_F32) return fail(MPADAM_EINVAL, "accumulation needs a binary32 d");
  if (p->m == 0 || p->n == 0) return MPADAM_OK;
  if (!p->d || !is_aligned(p->d, p->d_dtype == MPADAM_F32 ? 4 : 2)) return fail(MPADAM_EINVAL, "d NULL or misaligned");
  if (p->ldd < p->n) return fail(MPADAM_EINVAL, "ldd must be >= n");
  if (p->k == 0) return MPADAM_OK;
  if (!p->a || !p->b || !p->a_scale || !p->b_scale || !is_aligned(p->a, 16) || !is_aligned(p->b, 16) ||
      !is_aligned(p->a_scale, 16) || !is_aligned(p->b_scale, 16))
    return fail(MPADAM_EINVAL, "codes and scales must be 16-byte aligned and not NULL");
  if (p->lda < p->k || p->ldb < p->k || p->lda % 16 || p->ldb % 16)
    return fail(MPADAM_EINVAL, "lda and ldb must be multiples of 16, >= k");
  return MPADAM_OK;
}

// Of checked arguments; b_early: the launch follows a's quantisation on the stream.
int32_t multiply(const mpadam_e4m3_product* p, bool b_early, cudaStream_t stream) {
  if (p->m == 0 || p->n == 0) return MPADAM_OK;
  const size_t dsz = p->d_dtype == MPADAM_F32 ? 4 : 2;
  if (p->k == 0) {
    if (p->accumulate) return MPADAM_OK;
    const cudaError_t e = cudaMemset2DAsync(p->d, (size_t)p->ldd * dsz, 0, (size_t)p->n * dsz, (size_t)p->m, stream);
    return e == cudaSuccess ? MPADAM_OK : cuda_fail(e, "clearing d");
  }
  MatmulArgs a;
  const MatmulPlan plan = matmul_plan(p->m, p->n, p->k);
  if (!encode_tiled()) return fail(MPADAM_EUNSUPPORTED, "the driver offers no cuTensorMapEncodeTiled");
  if (!code_map(&a.a, p->a, p->m, p->k, p->lda, plan.box()) || !code_map(&a.b, p->b, p->n, p->k, p->ldb, 128) ||
      (plan.pair && (!scale_map(&a.sa_map, p->a_scale, p->m, p->k, 2) || !scale_map(&a.sb_map, p->b_scale, p->n, p->k, 1))))
    return fail(MPADAM_EINVAL, "no tensor map for these codes");
  a.sa = p->a_scale;
  a.sb = p->b_scale;
  a.d = p->d;
  a.ldd = p->ldd;
  a.m = (int32_t)p->m;
  a.n = (int32_t)p->n;
  a.k = (int32_t)p->k;
  a.f32 = p->d_dtype == MPADAM_F32;
  a.accumulate = p->accumulate;
  a.b_early = b_early && !plan.pair;
  cudaError_t e = matmul_error_word(&a.err);
  if (e != cudaSuccess) return cuda_fail(e, "the products' error word");
  e = launch_matmul(a, plan, stream);
  if (e != cudaSuccess) return cuda_fail(e, "launch of the product");
  return MPADAM_OK;
}

}  // namespace

extern "C" int32_t mpadam_e4m3_matmul(const mpadam_e4m3_product* p, cudaStream_t stream) {
  const int32_t rc = check_product(p);
  return rc ? rc : multiply(p, false, stream);
}

extern "C" int32_t mpadam_e4m3_quantize_matmul(const void* x, int32_t x_dtype, int64_t ldx, const mpadam_e4m3_product* p,
                                               cudaStream_t stream) {
  int32_t rc = check_product(p);
  if (rc) return rc;
  rc = mpadam_e4m3_quantize(x, x_dtype, p->m, p->k, ldx, 0, const_cast<uint8_t*>(p->a), const_cast<uint8_t*>(p->a_scale), p->lda,
                            nullptr, nullptr, 0, stream);
  return rc ? rc : multiply(p, p->m > 0 && p->k > 0, stream);
}

extern "C" int32_t mpadam_e4m3_status(cudaStream_t stream, int32_t* code) {
  if (!code) return fail(MPADAM_EINVAL, "code is NULL");
  *code = 0;
  int32_t* err = nullptr;
  cudaError_t e = matmul_error_word(&err);
  if (e != cudaSuccess) return cuda_fail(e, "the products' error word");
  e = cudaMemcpyAsync(code, err, sizeof(int32_t), cudaMemcpyDeviceToHost, stream);
  if (e != cudaSuccess) return cuda_fail(e, "reading the error word");
  e = cudaMemsetAsync(err, 0, sizeof(int32_t), stream);
  if (e != cudaSuccess) return cuda_fail(e, "clearing the error word");
  e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return cuda_fail(e, "cudaStreamSynchronize");
  return MPADAM_OK;
}

extern "C" int32_t mpadam_debug_e4m3_plan(int64_t m, int64_t n, int64_t k, int32_t* plan) {
  if (!plan) return fail(MPADAM_EINVAL, "plan is NULL");
  if (m < 1 || n < 1 || k < 1 || m > kMatmulMax || n > kMatmulMax || k > kMatmulMax)
    return fail(MPADAM_EINVAL, "m, n and k must be in [1, 2^31 - 1024]");
  const MatmulPlan p = matmul_plan(m, n, k);
  plan[0] = p.tile, plan[1] = p.split, plan[2] = p.pair;
  return MPADAM_OK;
}
