// muon_api.cu -- host side of mpadam_orthogonal_* and mpadam_muon_*
// (include/mpadam.h): tables and workspace of a list of matrices, and the
// launches of a call.
#include <algorithm>
#include <cmath>
#include <memory>
#include <new>
#include <vector>

#include "list.h"
#include "muon.h"
#include "muon_schedule.h"

using namespace mpadam;

namespace {

constexpr int64_t kMaxSide = 1 << 20;
// Matrices share a workspace while theirs together stay below this; others follow when those are done.
constexpr int64_t kWorkspace = (int64_t)6 << 30;

struct Matrix {
  void* w;
  void* m;
  uint16_t* compute;
  int64_t rows, cols;
};

// Matrices whose products run together, and where their entries in the tables begin.
struct Group {
  int64_t chunk_owner = 0, tile_owner = 0, product = 0;
  int32_t first = 0, chunks = 0, tiles = 0, product_tiles = 0;
};

int64_t round_up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }

bool matrix_map(CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t boxes[2] = {64, (cuuint32_t)box_rows}, steps[2] = {1, 1};
  return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(p), dims, strides, boxes, steps,
                        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool matrix_maps(NewtonMatrix* m) {
  constexpr int kOperand = kNewtonTile / 2, kAlong = kNewtonStepK, kPatch = 32;
  auto x = [&](CUtensorMap* map, const void* p, int box_rows) { return matrix_map(map, p, m->r, m->c, m->ld, box_rows); };
  auto a = [&](CUtensorMap* map, const void* p, int box_rows) { return matrix_map(map, p, m->r, m->r, m->lda, box_rows); };
  bool ok = x(&m->lo_patch, m->lo, kPatch);
  for (int i = 0; i < 2; ++i)
    ok = ok && x(&m->x[i], m->hi[i], kOperand) && x(&m->x_along[i], m->hi[i], kAlong) && x(&m->x_patch[i], m->hi[i], kPatch);
  ok = ok && a(&m->a, m->ga, kOperand) && a(&m->a_along, m->ga, kAlong) && a(&m->a_patch, m->ga, kPatch);
  return ok && a(&m->b, m->gb, kOperand) && a(&m->b_along, m->gb, kAlong) && a(&m->b_patch, m->gb, kPatch);
}

// What both operators keep: the list, its tables on the device, the workspace.
struct Newton {
  int device = 0;
  int32_t n = 0, steps = 0;
  MuonKind kind{};
  std::vector<int64_t> numel;
  std::vector<Group> groups;
  uint8_t* memory = nullptr;
  uint8_t* workspace = nullptr;
  const NewtonMatrix* d_newton = nullptr;
  const int32_t* d_owners = nullptr;
  const NewtonTile* d_tiles = nullptr;
  PointerTable in, out;
  MuonArgs args{};

  Newton() = default;
  Newton(const Newton&) = delete;
  ~Newton() {
    cudaFree(memory);
    cudaFree(workspace);
  }

  // factor: of the learning rate, by a matrix's sizes.
  int32_t build(const std::vector<Matrix>& list, float (*factor)(int64_t, int64_t)) {
    n = (int32_t)list.size();
    cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    std::vector<MuonMatrix> matrices;
    std::vector<NewtonMatrix> newton;
    std::vector<int32_t> owners;
    std::vector<NewtonTile> tiles;
    std::vector<int64_t> offsets;  // of each matrix in the workspace
    int64_t goff = 0, used = 0, most = 0, chunks_most = 0, counters = 0;
    std::vector<std::pair<int32_t, int32_t>> members;  // of each group: first and last + 1
    for (int32_t k = 0; k < n; ++k) {
      const Matrix& x = list[k];
      const int64_t count = x.rows * x.cols;
      numel.push_back(count);
      MuonMatrix q{};
      q.w = x.w, q.m = x.m, q.compute = x.compute;
      q.goff = goff;
      goff += round_up(count, 128);
      if (!count) continue;
      q.rows = (int32_t)x.rows, q.cols = (int32_t)x.cols;
      q.tall = x.rows > x.cols;
      q.index = k;
      q.factor = factor ? factor(x.rows, x.cols) : 1.0f;
      q.aligned = is_aligned(x.w, 16) && is_aligned(x.m, 16) && is_aligned(x.compute, 16);
      // Four passes a block where a matrix has 64 such blocks: its end (a sum, a fence, a count) takes longer than a pass.
      q.chunk = (int32_t)std::max(round_up((count + kMaxChunks - 1) / kMaxChunks, kSquaresPass),
                                  std::min<int64_t>(4 * kSquaresPass, round_up(count / 64 + 1, kSquaresPass)));
      q.chunks = (int32_t)((count + q.chunk - 1) / q.chunk);
      q.tiles_across = (int32_t)((x.cols + kTileCols - 1) / kTileCols);
      NewtonMatrix m{};
      m.r = std::min(q.rows, q.cols), m.c = std::max(q.rows, q.cols);
      m.ld = q.ld = round_up(m.c, 64);
      m.lda = round_up(m.r, 64);
      m.row0 = (int32_t)counters;
      counters += newton_across(m.r);
      const int64_t bytes = 3 * round_up(2 * m.r * m.ld, 1024) + 2 * round_up(2 * m.r * m.lda, 1024);
      if (members.empty() || used + bytes > kWorkspace) {
        members.push_back({(int32_t)matrices.size(), (int32_t)matrices.size()});
        used = 0;
      }
      offsets.push_back(used);
      used += bytes;
      most = std::max(most, used);
      ++members.back().second;
      matrices.push_back(q);
      newton.push_back(m);
    }
    if (!encode_tiled() && !matrices.empty()) return fail(MPADAM_EUNSUPPORTED, "the driver offers no cuTensorMapEncodeTiled");
    if (most && dev_malloc(&workspace, (size_t)most) != cudaSuccess) {
      workspace = nullptr;
      cudaGetLastError();
      return fail(MPADAM_EALLOC, "allocation of a workspace of %lld bytes failed", (long long)most);
    }
    for (const auto& member : members) {
      Group g;
      g.first = member.first;
      g.chunk_owner = (int64_t)owners.size();
      for (int32_t k = member.first; k < member.second; ++k) {
        matrices[k].chunk0 = (int64_t)owners.size() - g.chunk_owner;
        owners.insert(owners.end(), matrices[k].chunks, k);
      }
      g.chunks = (int32_t)(owners.size() - g.chunk_owner);
      chunks_most = std::max<int64_t>(chunks_most, g.chunks);
      g.tile_owner = (int64_t)owners.size();
      for (int32_t k = member.first; k < member.second; ++k) {
        const int64_t down = (matrices[k].rows + kTileRows - 1) / kTileRows;
        const int64_t first = (int64_t)owners.size() - g.tile_owner;
        if (first + down * matrices[k].tiles_across >= INT32_MAX) return fail(MPADAM_EINVAL, "the list has too many elements");
        matrices[k].tile0 = (int32_t)first;
        owners.insert(owners.end(), down * matrices[k].tiles_across, k);
      }
      g.tiles = (int32_t)(owners.size() - g.tile_owner);
      int64_t count = 0;
      for (int32_t k = member.first; k < member.second; ++k)
        for (int which = 1; which <= 3; ++which) count += steps * newton_tiles(which, newton[k].r, newton[k].c);
      if (count >= INT32_MAX / (2 * kSignals)) return fail(MPADAM_EINVAL, "the list has too many elements");
      g.product = (int64_t)tiles.size();
      g.product_tiles = (int32_t)count;
      newton_schedule(newton, member.first, member.second, steps, kNewtonPairs, &tiles);
      groups.push_back(g);
    }
    for (size_t k = 0; k < matrices.size(); ++k) {
      NewtonMatrix& m = newton[k];
      uint8_t* at = workspace + offsets[k];
      const int64_t x = round_up(2 * m.r * m.ld, 1024), a = round_up(2 * m.r * m.lda, 1024);
      auto next = [&](int64_t bytes) {
        uint16_t* p = reinterpret_cast<uint16_t*>(at);
        at += bytes;
        return p;
      };
      m.hi[0] = next(x), m.hi[1] = next(x), m.lo = next(x), m.ga = next(a), m.gb = next(a);
      matrices[k].hi[0] = m.hi[0], matrices[k].hi[1] = m.hi[1];
      matrices[k].lo = m.lo;
      if (!matrix_maps(&m)) return fail(MPADAM_EINVAL, "no tensor map for a matrix of this size");
    }
    // one allocation: what is uploaded, then the partial sums, the error word and the tables of pointers
    const size_t newton_at = 0, matrices_at = newton_at + round_up(sizeof(NewtonMatrix) * newton.size(), 256);
    const size_t tiles_at = matrices_at + round_up(sizeof(MuonMatrix) * matrices.size(), 256);
    const size_t owners_at = tiles_at + round_up(sizeof(NewtonTile) * tiles.size(), 256);
    const size_t err_at = owners_at + round_up(sizeof(int32_t) * owners.size(), 256), norms_at = err_at + 256;
    const size_t progress_at = norms_at + round_up(sizeof(MuonNorm) * matrices.size(), 256);
    const size_t upload = progress_at + round_up(sizeof(uint32_t) * (counters + 1), 256);
    const size_t partial_at = upload, pointers_at = partial_at + round_up(sizeof(double) * chunks_most, 256);
    const size_t bytes = pointers_at + (n > kInlineGrads ? 2 * sizeof(void*) * n : 0);
    std::vector<uint8_t> host(upload);
    auto put = [&](size_t to, const void* from, size_t size) {
      if (size) std::memcpy(host.data() + to, from, size);
    };
    put(newton_at, newton.data(), sizeof(NewtonMatrix) * newton.size());
    put(matrices_at, matrices.data(), sizeof(MuonMatrix) * matrices.size());
    put(tiles_at, tiles.data(), sizeof(NewtonTile) * tiles.size());
    put(owners_at, owners.data(), sizeof(int32_t) * owners.size());
    if (dev_malloc(&memory, bytes) != cudaSuccess) {
      memory = nullptr;
      cudaGetLastError();
      return fail(MPADAM_EALLOC, "allocation of the list's tables failed");
    }
    e = cudaMemcpy(memory, host.data(), upload, cudaMemcpyHostToDevice);
    // a copy from pageable memory may return before it has arrived, and steps run on any stream
    if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);
    if (e != cudaSuccess) return cuda_fail(e, "upload of the list's tables");
    d_newton = reinterpret_cast<const NewtonMatrix*>(memory + newton_at);
    d_tiles = reinterpret_cast<const NewtonTile*>(memory + tiles_at);
    d_owners = reinterpret_cast<const int32_t*>(memory + owners_at);
    args.matrices = reinterpret_cast<const MuonMatrix*>(memory + matrices_at);
    args.partial = reinterpret_cast<double*>(memory + partial_at);
    args.err = reinterpret_cast<int32_t*>(memory + err_at);
    args.norms = reinterpret_cast<MuonNorm*>(memory + norms_at);
    args.progress = reinterpret_cast<uint32_t*>(memory + progress_at);
    args.counters = (int32_t)counters + 1;
    args.last = steps & 1;
    in.table = reinterpret_cast<const void**>(memory + pointers_at);
    out.table = in.table + n;
    return MPADAM_OK;
  }

  int32_t check_pointers(const void* const* p, const char* name, size_t size) const {
    if (!p) return fail(MPADAM_EINVAL, "%s is NULL", name);
    for (int32_t k = 0; k < n; ++k) {
      if (numel[k] == 0) continue;
      if (!p[k]) return fail(MPADAM_EINVAL, "%s[%d] is NULL", name, k);
      if (!is_aligned(p[k], size)) return fail(MPADAM_EINVAL, "%s[%d] not aligned to its element size", name, k);
    }
    return MPADAM_OK;
  }

  // All launches of a call.
  int32_t run(cudaStream_t stream) {
    for (const Group& g : groups) {
      args.owner = d_owners + g.chunk_owner;
      args.count = g.chunks;
      cudaError_t e = launch_squares(args, kind, stream);
      args.owner = d_owners + g.tile_owner;
      args.count = g.tiles;
      if (e == cudaSuccess) e = launch_begin(args, kind, stream);
      const ProductArgs p{d_newton, g.first, d_tiles + g.product, g.product_tiles, args.progress, args.progress + args.counters - 1, args.err};
      if (e == cudaSuccess) e = launch_products(p, stream);
      if (e == cudaSuccess) e = launch_finish(args, kind, stream);
      if (e != cudaSuccess) return cuda_fail(e, "launch of the Newton-Schulz steps");
    }
    return MPADAM_OK;
  }

  int32_t status(int32_t* code) {
    *code = 0;
    const int32_t rc = check_device(device);
    if (rc) return rc;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(code, args.err, sizeof(int32_t), cudaMemcpyDeviceToHost);
    if (e == cudaSuccess && *code) {
      e = cudaMemset(args.err, 0, sizeof(int32_t));
      // the clear is asynchronous, and the next call may be on a stream that does not wait for it
      if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);
    }
    return e == cudaSuccess ? MPADAM_OK : cuda_fail(e, "reading the error word");
  }
};

bool real(int32_t dtype) { return dtype == MPADAM_F32 || dtype == MPADAM_BF16; }

int32_t check_side(int32_t k, int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0 || rows > kMaxSide || cols > kMaxSide)
    return fail(MPADAM_EINVAL, "matrix %d: rows and columns must be in [0, 2^20]", k);
  return MPADAM_OK;
}

// Whether a step would write two of the list's arrays to the same memory.
bool any_overlap(const std::vector<Matrix>& list, size_t wsz, size_t msz) {
  std::vector<std::pair<uintptr_t, uintptr_t>> spans;
  for (const Matrix& x : list) {
    const size_t count = (size_t)x.rows * (size_t)x.cols;
    auto add = [&](const void* p, size_t size) {
      if (p && count) spans.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + count * size});
    };
    add(x.w, wsz), add(x.m, msz), add(x.compute, 2);
  }
  std::sort(spans.begin(), spans.end());
  for (size_t i = 1; i < spans.size(); ++i)
    if (spans[i].first < spans[i - 1].second) return true;
  return false;
}

}  // namespace

struct mpadam_orthogonal_state {
  Newton newton;
};
struct mpadam_muon_state {
  Newton newton;
  mpadam_muon_config cfg;
};

extern "C" int32_t mpadam_orthogonal_create(const int64_t* rows, const int64_t* cols, int32_t n, int32_t dtype, int32_t steps,
                                            mpadam_orthogonal_state** out) {
  if (!out) return fail(MPADAM_EINVAL, "out is NULL");
  *out = nullptr;
  if (n < 0) return fail(MPADAM_EINVAL, "n must be >= 0");
  if (n > 0 && (!rows || !cols)) return fail(MPADAM_EINVAL, "rows or cols is NULL");
  if (!real(dtype)) return fail(MPADAM_EINVAL, "dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", dtype);
  if (steps < 1 || steps > 32) return fail(MPADAM_EINVAL, "steps must be in [1, 32]");
  try {
    std::vector<Matrix> list((size_t)n);
    for (int32_t k = 0; k < n; ++k) {
      const int32_t rc = check_side(k, rows[k], cols[k]);
      if (rc) return rc;
      list[k] = {nullptr, nullptr, nullptr, rows[k], cols[k]};
    }
    std::unique_ptr<mpadam_orthogonal_state> s(new mpadam_orthogonal_state());
    s->newton.steps = steps;
    s->newton.kind = {false, dtype == MPADAM_F32, true, dtype == MPADAM_F32, false};
    const int32_t rc = s->newton.build(list, nullptr);
    if (rc) return rc;
    *out = s.release();
  } catch (const std::bad_alloc&) {
    return fail(MPADAM_EALLOC, "host allocation failed");
  }
  return MPADAM_OK;
}

extern "C" int32_t mpadam_orthogonalize(mpadam_orthogonal_state* s, const void* const* x, void* const* out, cudaStream_t stream) {
  if (!s) return fail(MPADAM_EINVAL, "state is NULL");
  Newton& t = s->newton;
  if (t.groups.empty()) return MPADAM_OK;
  const size_t size = t.kind.in_f32 ? 4 : 2;
  int32_t rc = t.check_pointers(x, "x", size);
  if (!rc) rc = t.check_pointers(const_cast<const void* const*>(out), "out", size);
  if (!rc) rc = check_device(t.device);
  if (rc) return rc;
  try {
    rc = t.in.for_launch(&t.args.in, x, t.n, stream);
    if (!rc) rc = t.out.for_launch(&t.args.out, const_cast<const void* const*>(out), t.n, stream);
  } catch (const std::bad_alloc&) {
    return fail(MPADAM_EALLOC, "host allocation failed");
  }
  return rc ? rc : t.run(stream);
}

extern "C" int32_t mpadam_orthogonal_status(mpadam_orthogonal_state* s, int32_t* code) {
  if (!s || !code) return fail(MPADAM_EINVAL, "state or code is NULL");
  return s->newton.status(code);
}

extern "C" int32_t mpadam_orthogonal_destroy(mpadam_orthogonal_state* s) {
  if (!s) return MPADAM_OK;
  cudaDeviceSynchronize();
  delete s;
  return MPADAM_OK;
}

extern "C" int32_t mpadam_muon_create(const mpadam_muon_tensor* tensors, int32_t n, const mpadam_muon_config* cfg,
                                      mpadam_muon_state** out) {
  if (!out) return fail(MPADAM_EINVAL, "out is NULL");
  *out = nullptr;
  if (!cfg) return fail(MPADAM_EINVAL, "config is NULL");
  if (n < 0) return fail(MPADAM_EINVAL, "n must be >= 0");
  if (n > 0 && !tensors) return fail(MPADAM_EINVAL, "tensors is NULL");
  const mpadam_muon_config& c = *cfg;
  if (!real(c.weight_dtype)) return fail(MPADAM_EINVAL, "weight_dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", c.weight_dtype);
  if (!real(c.grad_dtype)) return fail(MPADAM_EINVAL, "grad_dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", c.grad_dtype);
  if (!real(c.momentum_dtype)) return fail(MPADAM_EINVAL, "momentum_dtype must be MPADAM_F32 or MPADAM_BF16 (got %d)", c.momentum_dtype);
  if (c.rounding != MPADAM_ROUND_NEAREST && c.rounding != MPADAM_ROUND_STOCHASTIC)
    return fail(MPADAM_EINVAL, "rounding must be nearest (0) or stochastic (1) (got %d)", c.rounding);
  if (c.scale != MPADAM_SCALE_RMS && c.scale != MPADAM_SCALE_SPECTRAL)
    return fail(MPADAM_EINVAL, "scale must be MPADAM_SCALE_RMS or MPADAM_SCALE_SPECTRAL (got %d)", c.scale);
  if (c.nesterov != 0 && c.nesterov != 1) return fail(MPADAM_EINVAL, "nesterov must be 0 or 1");
  if (c.steps < 1 || c.steps > 32) return fail(MPADAM_EINVAL, "steps must be in [1, 32]");
  if (c.reserved != 0) return fail(MPADAM_EINVAL, "reserved must be 0");
  if (!(c.momentum >= 0.0f && c.momentum < 1.0f)) return fail(MPADAM_EINVAL, "momentum must be in [0, 1)");
  if (!(std::isfinite(c.weight_decay) && c.weight_decay >= 0.0f)) return fail(MPADAM_EINVAL, "weight_decay must be finite and >= 0");
  const size_t wsz = c.weight_dtype == MPADAM_F32 ? 4 : 2, msz = c.momentum_dtype == MPADAM_F32 ? 4 : 2;
  try {
    std::vector<Matrix> list((size_t)n);
    for (int32_t k = 0; k < n; ++k) {
      const mpadam_muon_tensor& t = tensors[k];
      const int32_t rc = check_side(k, t.rows, t.cols);
      if (rc) return rc;
      if (t.compute && c.weight_dtype != MPADAM_F32) return fail(MPADAM_EINVAL, "matrix %d: a compute copy is for binary32 weights", k);
      list[k] = {t.w, t.m, t.compute, t.rows, t.cols};
      if (t.rows == 0 || t.cols == 0) continue;
      if (!t.w || !t.m) return fail(MPADAM_EINVAL, "matrix %d has a NULL pointer", k);
      if (!is_aligned(t.w, wsz) || !is_aligned(t.m, msz) || !is_aligned(t.compute, 2))
        return fail(MPADAM_EINVAL, "matrix %d: a pointer is not aligned to its element size", k);
    }
    if (any_overlap(list, wsz, msz)) return fail(MPADAM_EINVAL, "weights, momentum and compute copies must not overlap");
    std::unique_ptr<mpadam_muon_state> s(new mpadam_muon_state());
    s->cfg = c;
    s->newton.steps = c.steps;
    s->newton.kind = {true, c.grad_dtype == MPADAM_F32, c.momentum_dtype == MPADAM_F32, c.weight_dtype == MPADAM_F32,
                      c.rounding == MPADAM_ROUND_STOCHASTIC && c.weight_dtype == MPADAM_BF16};
    auto rms = [](int64_t r, int64_t k) { return (float)(0.2 * std::sqrt((double)std::max(r, k))); };
    auto spectral = [](int64_t r, int64_t k) { return (float)std::sqrt(std::max(1.0, (double)r / (double)k)); };
    const int32_t rc = c.scale == MPADAM_SCALE_RMS ? s->newton.build(list, +rms) : s->newton.build(list, +spectral);
    if (rc) return rc;
    MuonArgs& a = s->newton.args;
    a.beta = c.momentum;
    a.rest = (float)(1.0 - (double)c.momentum);
    a.nesterov = c.nesterov;
    round_keys(c.seed, a.rk0, a.rk1);
    *out = s.release();
  } catch (const std::bad_alloc&) {
    return fail(MPADAM_EALLOC, "host allocation failed");
  }
  return MPADAM_OK;
}

extern "C" int32_t mpadam_muon_step(mpadam_muon_state* s, const void* const* grads, int64_t step, float lr, const float* grad_scale,
                                    cudaStream_t stream) {
  if (!s) return fail(MPADAM_EINVAL, "state is NULL");
  if (step < 1) return fail(MPADAM_EINVAL, "step must be >= 1 (got %lld)", (long long)step);
  if (!(std::isfinite(lr) && lr >= 0.0f)) return fail(MPADAM_EINVAL, "lr must be finite and >= 0");
  if (!is_aligned(grad_scale, 4)) return fail(MPADAM_EINVAL, "grad_scale misaligned");
  Newton& t = s->newton;
  if (t.groups.empty()) return MPADAM_OK;
  int32_t rc = t.check_pointers(grads, "grads", t.kind.in_f32 ? 4 : 2);
  if (!rc) rc = check_device(t.device);
  if (rc) return rc;
  try {
    rc = t.in.for_launch(&t.args.in, grads, t.n, stream);
  } catch (const std::bad_alloc&) {
    return fail(MPADAM_EALLOC, "host allocation failed");
  }
  if (rc) return rc;
  t.args.grad_scale = grad_scale;
  t.args.step = step;
  t.args.lr = lr;
  t.args.decay = (float)((double)lr * (double)s->cfg.weight_decay);
  return t.run(stream);
}

extern "C" int32_t mpadam_muon_status(mpadam_muon_state* s, int32_t* code) {
  if (!s || !code) return fail(MPADAM_EINVAL, "state or code is NULL");
  return s->newton.status(code);
}

extern "C" int32_t mpadam_muon_destroy(mpadam_muon_state* s) {
  if (!s) return MPADAM_OK;
  cudaDeviceSynchronize();
  delete s;
  return MPADAM_OK;
}
