// layer_api.cu -- host side of mpadam_layer_norm_* and mpadam_nvfp4_linear
// (include/mpadam.h).
#include <cmath>

#include "fp4.h"
#include "host.h"
#include "layer_norm.h"

using namespace mpadam;

namespace {

bool real(int32_t dtype) { return dtype == MPADAM_F32 || dtype == MPADAM_BF16; }
size_t size_of(int32_t dtype) { return dtype == MPADAM_F32 ? 4 : 2; }

// What the forward and the backward pass have in common; rows and cols are not 0 when `pointers`.
int32_t check_norm(int64_t rows, int64_t cols, int32_t x_dtype, int32_t w_dtype) {
  if (rows < 0 || cols < 0 || rows > INT32_MAX || cols > INT32_MAX) return fail(MPADAM_EINVAL, "rows and cols must be in [0, 2^31)");
  if (!real(x_dtype)) return fail(MPADAM_EINVAL, "x_dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", x_dtype);
  if (w_dtype != MPADAM_F32 && w_dtype != x_dtype) return fail(MPADAM_EINVAL, "w_dtype must be MPADAM_F32 or x's (got %d)", w_dtype);
  return MPADAM_OK;
}
// A matrix of `cols` columns that is there and has room for them between its rows.
int32_t check_rows(const char* name, const void* p, int64_t ld, int64_t cols, size_t size) {
  if (!p || !is_aligned(p, size)) return fail(MPADAM_EINVAL, "%s NULL or misaligned", name);
  if (ld < cols) return fail(MPADAM_EINVAL, "%s's row stride must be >= cols", name);
  return MPADAM_OK;
}

}  // namespace

extern "C" int32_t mpadam_layer_norm_forward(const mpadam_layer_norm* p, cudaStream_t stream) {
  if (!p) return fail(MPADAM_EINVAL, "the argument is NULL");
  int32_t rc = check_norm(p->rows, p->cols, p->x_dtype, p->w_dtype);
  if (rc) return rc;
  if (p->reserved != 0) return fail(MPADAM_EINVAL, "reserved must be 0");
  if (!(std::isfinite(p->eps) && p->eps >= 0.0f)) return fail(MPADAM_EINVAL, "eps must be finite and >= 0");
  if (!p->mean != !p->rstd) return fail(MPADAM_EINVAL, "mean and rstd come together or not at all");
  if (!is_aligned(p->mean, 4) || !is_aligned(p->rstd, 4)) return fail(MPADAM_EINVAL, "mean or rstd misaligned");
  if (!is_aligned(p->w, size_of(p->w_dtype)) || !is_aligned(p->b, size_of(p->w_dtype))) return fail(MPADAM_EINVAL, "w or b misaligned");
  if (p->rows == 0 || p->cols == 0) return MPADAM_OK;
  rc = check_rows("x", p->x, p->ldx, p->cols, size_of(p->x_dtype));
  if (!rc) rc = check_rows("y", p->y, p->ldy, p->cols, size_of(p->x_dtype));
  if (rc) return rc;
  const NormForwardArgs a{p->x, p->w, p->b, p->y, p->mean, p->rstd, p->rows, p->cols, p->ldx, p->ldy, p->eps,
                          (float)(1.0 / (double)p->cols), (float)p->cols, p->x_dtype == MPADAM_F32, p->w_dtype == MPADAM_F32};
  const cudaError_t e = launch_norm_forward(a, stream);
  return e == cudaSuccess ? MPADAM_OK : cuda_fail(e, "launch of the layer norm");
}

extern "C" int32_t mpadam_layer_norm_workspace(int64_t rows, int64_t cols, int64_t* bytes) {
  if (!bytes) return fail(MPADAM_EINVAL, "bytes is NULL");
  *bytes = 0;
  if (rows < 0 || cols < 0 || rows > INT32_MAX || cols > INT32_MAX) return fail(MPADAM_EINVAL, "rows and cols must be in [0, 2^31)");
  if (rows && cols) *bytes = (int64_t)norm_parts(rows, cols) * 2 * cols * (int64_t)sizeof(float);
  return MPADAM_OK;
}

extern "C" int32_t mpadam_layer_norm_backward(const mpadam_layer_norm_grad* p, cudaStream_t stream) {
  if (!p) return fail(MPADAM_EINVAL, "the argument is NULL");
  int32_t rc = check_norm(p->rows, p->cols, p->x_dtype, p->w_dtype);
  if (rc) return rc;
  const size_t xs = size_of(p->x_dtype), ws = size_of(p->w_dtype);
  if (!is_aligned(p->w, ws) || !is_aligned(p->dw, ws) || !is_aligned(p->db, ws)) return fail(MPADAM_EINVAL, "w, dw or db misaligned");
  if (p->cols == 0) return MPADAM_OK;
  if (p->rows == 0) {  // sums of nothing
    for (void* d : {p->dw, p->db}) {
      const cudaError_t e = d ? cudaMemsetAsync(d, 0, ws * (size_t)p->cols, stream) : cudaSuccess;
      if (e != cudaSuccess) return cuda_fail(e, "clearing dw and db");
    }
    return MPADAM_OK;
  }
  if (!p->dx && !p->dw && !p->db) return MPADAM_OK;
  rc = check_rows("x", p->x, p->ldx, p->cols, xs);
  if (!rc) rc = check_rows("dy", p->dy, p->lddy, p->cols, xs);
  if (!rc && p->dx) rc = check_rows("dx", p->dx, p->lddx, p->cols, xs);
  if (rc) return rc;
  if (!p->mean || !p->rstd || !is_aligned(p->mean, 4) || !is_aligned(p->rstd, 4)) return fail(MPADAM_EINVAL, "mean or rstd NULL or misaligned");
  const bool sums = p->dw || p->db;
  int64_t need = 0;
  mpadam_layer_norm_workspace(p->rows, p->cols, &need);
  if (sums && (!p->workspace || !is_aligned(p->workspace, 16) || p->workspace_bytes < need))
    return fail(MPADAM_EINVAL, "dw and db need a workspace of %lld bytes, 16-byte aligned", (long long)need);
  const int parts = norm_parts(p->rows, p->cols);
  float* partial = sums ? static_cast<float*>(p->workspace) : nullptr;
  const NormBackwardArgs a{p->x, p->dy, p->w, p->mean, p->rstd, p->dx, partial, p->rows, p->cols, p->ldx, p->lddy, p->lddx,
                           (float)(1.0 / (double)p->cols), p->x_dtype == MPADAM_F32, p->w_dtype == MPADAM_F32, parts};
  cudaError_t e = launch_norm_backward(a, stream);
  if (e != cudaSuccess) return cuda_fail(e, "launch of the layer norm's backward pass");
  if (sums) e = launch_norm_sums({partial, p->dw, p->db, p->cols, parts, p->w_dtype == MPADAM_F32}, stream);
  return e == cudaSuccess ? MPADAM_OK : cuda_fail(e, "launch of the layer norm's sums");
}

extern "C" int32_t mpadam_nvfp4_linear(const void* x, int32_t x_dtype, int64_t tokens, int64_t ldx, const mpadam_nvfp4_matrix* w,
                                       void* y, int64_t ldy, cudaStream_t stream) {
  if (!w) return fail(MPADAM_EINVAL, "w is NULL");
  if (!real(x_dtype)) return fail(MPADAM_EINVAL, "x_dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", x_dtype);
  if (tokens < 0 || tokens > (1 << 16)) return fail(MPADAM_EINVAL, "tokens must be in [0, 2^16]");
  if (w->rows < 0 || w->cols < 0 || w->rows > INT32_MAX || w->cols > INT32_MAX)
    return fail(MPADAM_EINVAL, "rows and cols must be in [0, 2^31)");
  if (!(std::isfinite(w->global_scale) && w->global_scale > 0.0f)) return fail(MPADAM_EINVAL, "global_scale must be finite and > 0");
  if (w->reserved != 0) return fail(MPADAM_EINVAL, "reserved must be 0");
  if (tokens == 0 || w->rows == 0) return MPADAM_OK;
  const size_t size = size_of(x_dtype);
  if (!y || !is_aligned(y, size) || ldy < w->rows) return fail(MPADAM_EINVAL, "y NULL or misaligned, or ldy < rows");
  if (w->cols == 0) {
    const cudaError_t e = cudaMemset2DAsync(y, (size_t)ldy * size, 0, (size_t)w->rows * size, (size_t)tokens, stream);
    return e == cudaSuccess ? MPADAM_OK : cuda_fail(e, "clearing y");
  }
  if (!x || !is_aligned(x, size) || ldx < w->cols) return fail(MPADAM_EINVAL, "x NULL or misaligned, or ldx < cols");
  if (!w->codes || !w->scales) return fail(MPADAM_EINVAL, "codes or scales NULL");
  const cudaError_t e = launch_fp4_linear({x, w->codes, w->scales, y, tokens, w->rows, w->cols, ldx, ldy, w->global_scale,
                                           x_dtype == MPADAM_F32, 0, 1}, stream);
  return e == cudaSuccess ? MPADAM_OK : cuda_fail(e, "launch of the product");
}
