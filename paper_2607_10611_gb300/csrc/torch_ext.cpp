// torch_ext.cpp -- the Python module _mpadam_torch: what the list operators and
// the 8-bit layer do on torch's side of the C ABI (include/mpadam.h), in C++
// because a short call's time is its host's.  It looks at tensors, allocates
// outputs with torch and calls the library; it holds no arithmetic.
//
// From Python, a step over 98 small tensors took 36 us against 5 on the GPU, the
// norm of 4000 ragged ones 1195 against 91, a linear layer of 1023 x 768 x 2304
// forward and backward 434 against 48.
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/core/AutogradState.h>
#include <c10/core/Event.h>
#include <c10/cuda/CUDACachingAllocator.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/function.h>
#include <torch/csrc/autograd/functions/utils.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/autograd/saved_variable.h>

#include <memory>
#include <string>
#include <vector>

#include "mpadam.h"

namespace {

using at::Tensor;
using torch::autograd::variable_list;

constexpr auto kCodes = at::kFloat8_e4m3fn;
constexpr auto kScales = at::kFloat8_e8m0fnu;

PyObject* g_error = nullptr;  // _native.MPAdamError

// Raises the library's last error as MPAdamError; returns nullptr.
PyObject* raise(int32_t status) {
  PyObject* e = g_error ? PyObject_CallFunction(g_error, "is", (int)status, mpadam_last_error()) : nullptr;
  if (e) {
    PyErr_SetObject(g_error, e);
    Py_DECREF(e);
  } else if (!PyErr_Occurred()) {
    PyErr_SetString(PyExc_RuntimeError, mpadam_last_error());
  }
  return nullptr;
}
// The same from inside C++ calls; the backward pass runs without the interpreter's lock.
void check(int32_t status) {
  if (!status) return;
  TORCH_CHECK(PyGILState_Check(), mpadam_last_error());
  raise(status);
  throw python_error();
}

const Tensor& tensor_of(PyObject* o, const char* what) {
  TORCH_CHECK_VALUE(THPVariable_Check(o), what, " must be a torch tensor");
  return THPVariable_Unpack(o);
}
cudaStream_t current_stream(const Tensor& t) { return c10::cuda::getCurrentCUDAStream(t.get_device()).stream(); }

int32_t type_of(const Tensor& t) { return t.scalar_type() == at::kFloat ? MPADAM_F32 : MPADAM_BF16; }
bool is_real(const Tensor& t) { return t.is_cuda() && (t.scalar_type() == at::kFloat || t.scalar_type() == at::kBFloat16); }
// A matrix whose rows are contiguous and do not overlap.
bool has_rows(const Tensor& t) {
  const int64_t r = t.size(0), c = t.size(1);
  return r == 0 || c == 0 || ((c == 1 || t.stride(1) == 1) && (r == 1 || t.stride(0) >= c));
}

// ---------------------------------------------------------------------------
// Lists of gradients
// ---------------------------------------------------------------------------
// What the gradients of a list have to be.
struct Spec {
  std::vector<int64_t> numel;
  std::vector<int64_t> rows, cols;  // of matrices; else empty
  at::ScalarType type;
  int device;
};
constexpr const char* kSpecName = "mpadam_list_spec";

// list_spec(numels, binary32?, device index) -> capsule
PyObject* list_spec(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 3 && PyList_Check(a[0]), "list_spec(list of sizes, binary32, device)");
  auto s = std::make_unique<Spec>();
  for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[0]); ++i) s->numel.push_back(PyLong_AsLongLong(PyList_GET_ITEM(a[0], i)));
  s->type = PyObject_IsTrue(a[1]) ? at::kFloat : at::kBFloat16;
  s->device = (int)PyLong_AsLong(a[2]);
  if (PyErr_Occurred()) return nullptr;
  return PyCapsule_New(s.release(), kSpecName,
                       [](PyObject* c) { delete static_cast<Spec*>(PyCapsule_GetPointer(c, kSpecName)); });
  END_HANDLE_TH_ERRORS
}

// matrix_spec(shapes, binary32?, device index) -> capsule: shapes are tuples (rows, columns)
PyObject* matrix_spec(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 3 && PyList_Check(a[0]), "matrix_spec(list of shapes, binary32, device)");
  auto s = std::make_unique<Spec>();
  for (Py_ssize_t i = 0; i < PyList_GET_SIZE(a[0]); ++i) {
    long long r, c;
    if (!PyArg_ParseTuple(PyList_GET_ITEM(a[0], i), "LL", &r, &c)) return nullptr;
    s->rows.push_back(r), s->cols.push_back(c), s->numel.push_back(r * c);
  }
  s->type = PyObject_IsTrue(a[1]) ? at::kFloat : at::kBFloat16;
  s->device = (int)PyLong_AsLong(a[2]);
  if (PyErr_Occurred()) return nullptr;
  return PyCapsule_New(s.release(), kSpecName,
                       [](PyObject* c) { delete static_cast<Spec*>(PyCapsule_GetPointer(c, kSpecName)); });
  END_HANDLE_TH_ERRORS
}

// Pointers of a list of gradients that meet the spec.
struct Pointers {
  std::vector<const void*> p;
  Pointers(PyObject* grads, const Spec& s) {
    PyObject* seq = PySequence_Fast(grads, "gradients must be a sequence of tensors");
    if (!seq) throw python_error();
    const std::unique_ptr<PyObject, void (*)(PyObject*)> hold(seq, [](PyObject* o) { Py_DECREF(o); });
    const Py_ssize_t n = PySequence_Fast_GET_SIZE(seq);
    TORCH_CHECK_VALUE((size_t)n == s.numel.size(), n, " gradients for ", s.numel.size(), " tensors");
    p.resize(n ? n : 1);
    PyObject** items = PySequence_Fast_ITEMS(seq);
    const caffe2::TypeMeta type = c10::scalarTypeToTypeMeta(s.type);
    const c10::Device device(c10::DeviceType::CUDA, (c10::DeviceIndex)s.device);
    for (Py_ssize_t i = 0; i < n; ++i) {
      const Tensor& t = tensor_of(items[i], "a gradient");
      const c10::TensorImpl& x = *t.unsafeGetTensorImpl();
      TORCH_CHECK_VALUE(x.dtype() == type && x.numel() == s.numel[i] && x.device() == device && x.is_contiguous(),
                        "gradients must be contiguous ", s.type, " tensors on cuda:", s.device, ", as large as their weights");
      TORCH_CHECK_VALUE(s.rows.empty() || (t.dim() == 2 && t.size(0) == s.rows[i] && t.size(1) == s.cols[i]), "matrix ", i,
                        " of the list must be [", s.rows[i], ", ", s.cols[i], "]");
      p[i] = x.data();
    }
  }
};

// adamw_create(config's address, w, m, v, m scales or None, v scales or None, compute or None) -> state: lists of tensors
// whose types, sizes and devices are checked here; compute's entries may be None.
PyObject* adamw_create(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 7, "adamw_create takes 7 arguments");
  const auto* cfg = static_cast<const mpadam_adamw_config*>(PyLong_AsVoidPtr(a[0]));
  if (PyErr_Occurred()) return nullptr;
  for (int i = 1; i < 7; ++i) TORCH_CHECK_VALUE(PyList_Check(a[i]) || (i > 3 && a[i] == Py_None), "the tensors come in lists");
  const bool low = cfg->state_dtype == MPADAM_E4M3;
  TORCH_CHECK_VALUE(!low || (a[4] != Py_None && a[5] != Py_None), "8-bit moments need m_scales and v_scales");
  TORCH_CHECK_VALUE(low || (a[4] == Py_None && a[5] == Py_None), "binary32 moments have no scales");
  const Py_ssize_t count = PyList_GET_SIZE(a[1]);
  for (int i = 2; i < 7; ++i)
    TORCH_CHECK_VALUE(a[i] == Py_None || PyList_GET_SIZE(a[i]) == count, "one entry per tensor in every list");
  std::vector<mpadam_adamw_tensor> list((size_t)count + 1);
  c10::optional<c10::Device> device;
  auto take = [&](int i, Py_ssize_t k, at::ScalarType type, const char* what) {
    const Tensor& t = tensor_of(PyList_GET_ITEM(a[i], k), what);
    TORCH_CHECK_VALUE(t.scalar_type() == type && t.is_cuda() && t.is_contiguous(), what, ": expected contiguous CUDA tensors of ",
                      type);
    if (!device) device = t.device();
    TORCH_CHECK_VALUE(t.device() == *device, "all tensors of a list must be on one device");
    return t;
  };
  const auto wt = cfg->weight_dtype == MPADAM_F32 ? at::kFloat : at::kBFloat16, st = low ? kCodes : at::kFloat;
  for (Py_ssize_t k = 0; k < count; ++k) {
    mpadam_adamw_tensor& x = list[k];
    const Tensor w = take(1, k, wt, "weights"), m = take(2, k, st, "moments"), v = take(3, k, st, "moments");
    x = {w.data_ptr(), m.data_ptr(), v.data_ptr(), nullptr, nullptr, nullptr, w.numel()};
    TORCH_CHECK_VALUE(m.numel() == x.numel && v.numel() == x.numel, "tensor ", k, ": moments differ in size from the weights");
    if (low) {
      const Tensor ms = take(4, k, kScales, "scales"), vs = take(5, k, kScales, "scales");
      TORCH_CHECK_VALUE(ms.numel() == (x.numel + 127) / 128 && vs.numel() == ms.numel(), "tensor ", k,
                        ": needs one scale per 128 elements");
      x.m_scale = static_cast<uint8_t*>(ms.data_ptr());
      x.v_scale = static_cast<uint8_t*>(vs.data_ptr());
    }
    if (a[6] != Py_None && PyList_GET_ITEM(a[6], k) != Py_None) {
      const Tensor c = take(6, k, at::kBFloat16, "compute copies");
      TORCH_CHECK_VALUE(c.numel() == x.numel, "tensor ", k, ": the compute copy differs in size from the weights");
      x.compute = static_cast<uint16_t*>(c.data_ptr());
    }
  }
  const c10::cuda::OptionalCUDAGuard guard(device);
  mpadam_adamw_state* state = nullptr;
  if (const int32_t rc = mpadam_adamw_create(list.data(), (int32_t)count, cfg, &state)) return raise(rc);
  return PyLong_FromVoidPtr(state);
  END_HANDLE_TH_ERRORS
}

cudaStream_t stream_of(PyObject* o, int device) {
  return o == Py_None ? c10::cuda::getCurrentCUDAStream(device).stream() : reinterpret_cast<cudaStream_t>(PyLong_AsSize_t(o));
}

// A step's arguments (state, spec, grads, t, lr, grad_scale or None, stream or None), handed to `step`.
template <typename F>
PyObject* list_step(PyObject* const* a, F step) {
  void* state = PyLong_AsVoidPtr(a[0]);
  auto* spec = static_cast<Spec*>(PyCapsule_GetPointer(a[1], kSpecName));
  const int64_t t = PyLong_AsLongLong(a[3]);
  const double lr = PyFloat_AsDouble(a[4]);
  if (PyErr_Occurred()) return nullptr;
  const cudaStream_t stream = stream_of(a[6], spec->device);
  if (PyErr_Occurred()) return nullptr;
  const Pointers g(a[2], *spec);
  const float* scale = nullptr;
  if (a[5] != Py_None) {
    const Tensor& x = tensor_of(a[5], "grad_scale");
    TORCH_CHECK_VALUE(x.scalar_type() == at::kFloat && x.is_cuda() && x.get_device() == spec->device && x.numel() >= 1,
                      "grad_scale must be a float32 tensor on cuda:", spec->device);
    scale = x.const_data_ptr<float>();
  }
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)spec->device);
  if (const int32_t rc = step(state, g.p.data(), t, (float)lr, scale, stream)) return raise(rc);
  Py_RETURN_NONE;
}

// adamw_step(state, spec, grads, t, lr, grad_scale or None, stream or None)
PyObject* adamw_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 7, "adamw_step takes 7 arguments");
  return list_step(a, [](void* state, const void* const* g, int64_t t, float lr, const float* scale, cudaStream_t stream) {
    return mpadam_adamw_step(static_cast<mpadam_adamw_state*>(state), g, t, lr, scale, stream);
  });
  END_HANDLE_TH_ERRORS
}

// grad_norm(state, spec, grads, max_norm, out or None, stream or None) -> out
PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 6, "grad_norm takes 6 arguments");
  auto* state = static_cast<mpadam_grad_norm_state*>(PyLong_AsVoidPtr(a[0]));
  auto* spec = static_cast<Spec*>(PyCapsule_GetPointer(a[1], kSpecName));
  const double max_norm = PyFloat_AsDouble(a[3]);
  if (PyErr_Occurred()) return nullptr;
  const cudaStream_t stream = stream_of(a[5], spec->device);
  if (PyErr_Occurred()) return nullptr;
  const Pointers g(a[2], *spec);
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)spec->device);
  Tensor out;
  if (a[4] != Py_None) {
    out = tensor_of(a[4], "out");
    TORCH_CHECK_VALUE(out.scalar_type() == at::kFloat && out.is_cuda() && out.get_device() == spec->device && out.numel() >= 2 &&
                          out.is_contiguous(),
                      "out must be two contiguous float32 elements on cuda:", spec->device);
  } else {
    out = at::empty({2}, at::TensorOptions().dtype(at::kFloat).device(at::kCUDA, (c10::DeviceIndex)spec->device));
  }
  if (const int32_t rc = mpadam_grad_norm(state, g.p.data(), (float)max_norm, out.data_ptr<float>(), stream)) return raise(rc);
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------
// Lists of matrices
// ---------------------------------------------------------------------------
// muon_create(config's address, w, m, compute or None) -> state: lists of matrices whose types, sizes and devices are
// checked here; compute's entries may be None.
PyObject* muon_create(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 4, "muon_create takes 4 arguments");
  const auto* cfg = static_cast<const mpadam_muon_config*>(PyLong_AsVoidPtr(a[0]));
  if (PyErr_Occurred()) return nullptr;
  for (int i = 1; i < 4; ++i) TORCH_CHECK_VALUE(PyList_Check(a[i]) || (i == 3 && a[i] == Py_None), "the matrices come in lists");
  const Py_ssize_t count = PyList_GET_SIZE(a[1]);
  for (int i = 2; i < 4; ++i)
    TORCH_CHECK_VALUE(a[i] == Py_None || PyList_GET_SIZE(a[i]) == count, "one entry per matrix in every list");
  std::vector<mpadam_muon_tensor> list((size_t)count + 1);
  c10::optional<c10::Device> device;
  auto take = [&](int i, Py_ssize_t k, int32_t dtype, const char* what) {
    const auto type = dtype == MPADAM_F32 ? at::kFloat : at::kBFloat16;
    const Tensor& t = tensor_of(PyList_GET_ITEM(a[i], k), what);
    TORCH_CHECK_VALUE(t.scalar_type() == type && t.dim() == 2 && t.is_cuda() && t.is_contiguous(), what,
                      ": expected contiguous CUDA matrices of ", type);
    if (!device) device = t.device();
    TORCH_CHECK_VALUE(t.device() == *device, "all matrices of a list must be on one device");
    return t;
  };
  for (Py_ssize_t k = 0; k < count; ++k) {
    const Tensor w = take(1, k, cfg->weight_dtype, "weights"), m = take(2, k, cfg->momentum_dtype, "momentum");
    TORCH_CHECK_VALUE(m.sizes() == w.sizes(), "matrix ", k, ": the momentum differs in shape from the weights");
    list[k] = {w.data_ptr(), m.data_ptr(), nullptr, w.size(0), w.size(1)};
    if (a[3] != Py_None && PyList_GET_ITEM(a[3], k) != Py_None) {
      const Tensor c = take(3, k, MPADAM_BF16, "compute copies");
      TORCH_CHECK_VALUE(c.sizes() == w.sizes(), "matrix ", k, ": the compute copy differs in shape from the weights");
      list[k].compute = static_cast<uint16_t*>(c.data_ptr());
    }
  }
  const c10::cuda::OptionalCUDAGuard guard(device);
  mpadam_muon_state* state = nullptr;
  if (const int32_t rc = mpadam_muon_create(list.data(), (int32_t)count, cfg, &state)) return raise(rc);
  return PyLong_FromVoidPtr(state);
  END_HANDLE_TH_ERRORS
}

// muon_step(state, spec, grads, t, lr, grad_scale or None, stream or None)
PyObject* muon_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 7, "muon_step takes 7 arguments");
  return list_step(a, [](void* state, const void* const* g, int64_t t, float lr, const float* scale, cudaStream_t stream) {
    return mpadam_muon_step(static_cast<mpadam_muon_state*>(state), g, t, lr, scale, stream);
  });
  END_HANDLE_TH_ERRORS
}

// orthogonalize(state, spec, x, out or None, stream or None) -> list of results
PyObject* orthogonalize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 5, "orthogonalize takes 5 arguments");
  auto* state = static_cast<mpadam_orthogonal_state*>(PyLong_AsVoidPtr(a[0]));
  auto* spec = static_cast<Spec*>(PyCapsule_GetPointer(a[1], kSpecName));
  if (PyErr_Occurred()) return nullptr;
  const cudaStream_t stream = stream_of(a[4], spec->device);
  if (PyErr_Occurred()) return nullptr;
  const Pointers x(a[2], *spec);
  const c10::cuda::CUDAGuard guard((c10::DeviceIndex)spec->device);
  const Py_ssize_t count = (Py_ssize_t)spec->numel.size();
  std::unique_ptr<PyObject, void (*)(PyObject*)> out(nullptr, [](PyObject* o) { Py_XDECREF(o); });
  if (a[3] != Py_None) {
    out.reset(PySequence_List(a[3]));
  } else {
    out.reset(PyList_New(count));
    const auto options = at::TensorOptions().dtype(spec->type).device(at::kCUDA, (c10::DeviceIndex)spec->device);
    for (Py_ssize_t i = 0; out && i < count; ++i) {
      PyObject* t = THPVariable_Wrap(at::empty({spec->rows[i], spec->cols[i]}, options));
      if (!t) throw python_error();
      PyList_SET_ITEM(out.get(), i, t);
    }
  }
  if (!out) throw python_error();
  const Pointers y(out.get(), *spec);
  if (const int32_t rc = mpadam_orthogonalize(state, x.p.data(), const_cast<void* const*>(y.p.data()), stream)) return raise(rc);
  return out.release();
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------
// E4M3 matrices
// ---------------------------------------------------------------------------
struct Matrix {
  Tensor codes, scales;
  int64_t rows() const { return codes.size(0); }
  int64_t cols() const { return codes.size(1); }
  uint8_t* q() const { return static_cast<uint8_t*>(codes.data_ptr()); }
  uint8_t* s() const { return static_cast<uint8_t*>(scales.data_ptr()); }
  // A single row's stride is of no matter, so its codes may have any.
  int64_t ld() const { return rows() > 1 ? codes.stride(0) : (cols() + 15) / 16 * 16; }

  // Where codes and scales lie in one allocation.
  struct Layout {
    int64_t ld, tiles, groups, scales_at, bytes;
    Layout(int64_t rows, int64_t cols)
        : ld((cols + 15) / 16 * 16), tiles((rows + 127) / 128), groups((cols + 511) / 512),
          scales_at((rows * ld + 255) / 256 * 256), bytes(scales_at + tiles * groups * 512) {}
  };
  static Tensor view(const c10::Storage& s, at::ScalarType type, at::IntArrayRef sizes, at::IntArrayRef strides, int64_t offset) {
    Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(s), c10::DispatchKeySet(c10::DispatchKey::CUDA),
                                                        c10::scalarTypeToTypeMeta(type));
    t.unsafeGetTensorImpl()->set_sizes_and_strides(sizes, strides, offset);
    return t;
  }
  // `first`: the byte of the storage that the layout begins at.
  static Matrix over(const c10::Storage& s, int64_t first, int64_t rows, int64_t cols) {
    const Layout l(rows, cols);
    return {view(s, kCodes, {rows, cols}, {l.ld, 1}, first),
            view(s, kScales, {l.tiles, l.groups, 32, 4, 4}, {l.groups * 512, 512, 16, 4, 1}, first + l.scales_at)};
  }
  // On the current device, codes and scales in one allocation and without the dispatcher: 4 us of host as two calls of
  // at::empty and one of narrow.
  static Matrix empty(int64_t rows, int64_t cols) {
    const c10::Storage storage(c10::make_intrusive<c10::StorageImpl>(c10::StorageImpl::use_byte_size_t(), Layout(rows, cols).bytes,
                                                                     c10::cuda::CUDACachingAllocator::get(), false));
    return over(storage, 0, rows, cols);
  }
  // All of what empty() made, as one tensor.
  Tensor bytes() const { return view(codes.storage(), at::kByte, {Layout(rows(), cols()).bytes}, {1}, 0); }
  static Matrix checked(PyObject* c, PyObject* s) {
    Matrix m{tensor_of(c, "codes"), tensor_of(s, "scales")};
    TORCH_CHECK_VALUE(m.codes.scalar_type() == kCodes && m.codes.dim() == 2 && m.codes.is_cuda(),
                      "codes must be a CUDA float8_e4m3fn matrix");
    TORCH_CHECK_VALUE(has_rows(m.codes), "codes must have contiguous rows");
    const int64_t want[5] = {(m.rows() + 127) / 128, (m.cols() + 511) / 512, 32, 4, 4};
    TORCH_CHECK_VALUE(m.scales.scalar_type() == kScales && m.scales.sizes() == at::IntArrayRef(want, 5) &&
                          m.scales.is_contiguous() && m.scales.device() == m.codes.device(),
                      "scales must be a contiguous float8_e8m0fnu tensor of ", at::IntArrayRef(want, 5), " beside the codes");
    return m;
  }
};

// x as it lies and its transpose, where asked for.
void quantize(const Tensor& x, bool square, Matrix* q, Matrix* qt) {
  const int64_t rows = x.size(0), cols = x.size(1);
  if (q) *q = Matrix::empty(rows, cols);
  if (qt) *qt = Matrix::empty(cols, rows);
  check(mpadam_e4m3_quantize(x.const_data_ptr(), type_of(x), rows, cols, rows > 1 ? std::max(x.stride(0), cols) : cols, square,
                             q ? q->q() : nullptr, q ? q->s() : nullptr, q ? q->ld() : 0, qt ? qt->q() : nullptr,
                             qt ? qt->s() : nullptr, qt ? qt->ld() : 0, current_stream(x)));
}

mpadam_e4m3_product product_of(const Matrix& a, const Matrix& b, const Tensor& out, bool accumulate) {
  mpadam_e4m3_product p{};
  p.a = a.q(), p.a_scale = a.s(), p.lda = a.ld();
  p.b = b.q(), p.b_scale = b.s(), p.ldb = b.ld();
  p.d = out.data_ptr();
  p.m = a.rows(), p.n = b.rows(), p.k = a.cols();
  p.ldd = p.m > 1 ? std::max(out.stride(0), p.n) : p.n;
  p.d_dtype = type_of(out);
  p.accumulate = accumulate;
  return p;
}
void multiply(const Matrix& a, const Matrix& b, const Tensor& out, bool accumulate) {
  const mpadam_e4m3_product p = product_of(a, b, out, accumulate);
  check(mpadam_e4m3_matmul(&p, current_stream(out)));
}

Tensor product(const Matrix& a, const Matrix& b, at::ScalarType type) {
  Tensor out = at::empty({a.rows(), b.rows()}, a.codes.options().dtype(type));
  multiply(a, b, out, false);
  return out;
}

// check_matrix(codes, scales)
PyObject* check_matrix(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 2, "check_matrix takes 2 arguments");
  Matrix::checked(a[0], a[1]);
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// quantize(x, square, as it lies?, transposed?) -> (codes, scales or None twice, ...) of both
PyObject* py_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 4, "quantize takes 4 arguments");
  const Tensor& x = tensor_of(a[0], "x");
  TORCH_CHECK_VALUE(x.dim() == 2 && is_real(x), "x must be a CUDA float32 or bfloat16 matrix");
  TORCH_CHECK_VALUE(has_rows(x), "x must have contiguous rows");
  const bool square = PyObject_IsTrue(a[1]), as_is = PyObject_IsTrue(a[2]), turned = PyObject_IsTrue(a[3]);
  const c10::cuda::CUDAGuard guard(x.device());
  Matrix q, qt;
  quantize(x, square, as_is ? &q : nullptr, turned ? &qt : nullptr);
  return Py_BuildValue("(NNNN)", THPVariable_Wrap(q.codes), THPVariable_Wrap(q.scales), THPVariable_Wrap(qt.codes),
                       THPVariable_Wrap(qt.scales));
  END_HANDLE_TH_ERRORS
}

// matmul(a codes, a scales, b codes, b scales, out or None, binary32 result?, accumulate) -> out
PyObject* py_matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 7, "matmul takes 7 arguments");
  const Matrix x = Matrix::checked(a[0], a[1]), y = Matrix::checked(a[2], a[3]);
  const bool accumulate = PyObject_IsTrue(a[6]);
  TORCH_CHECK_VALUE(x.cols() == y.cols(), "inner sizes differ: ", x.cols(), " and ", y.cols());
  TORCH_CHECK_VALUE(x.codes.device() == y.codes.device(), "the operands are on different devices");
  const c10::cuda::CUDAGuard guard(x.codes.device());
  Tensor out;
  if (a[4] != Py_None) {
    out = tensor_of(a[4], "out");
    TORCH_CHECK_VALUE(is_real(out) && out.dim() == 2 && out.size(0) == x.rows() && out.size(1) == y.rows() && has_rows(out) &&
                          out.device() == x.codes.device(),
                      "out must be a float32 or bfloat16 [", x.rows(), ", ", y.rows(), "] with contiguous rows beside the operands");
    multiply(x, y, out, accumulate);
  } else {
    TORCH_CHECK_VALUE(!accumulate, "accumulate needs out");
    out = product(x, y, PyObject_IsTrue(a[5]) ? at::kFloat : at::kBFloat16);
  }
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------
// The linear layer
// ---------------------------------------------------------------------------
// x as a matrix of its last dimension, with contiguous rows.
Tensor rows_of(const Tensor& x) {
  // (a size of -1 would be ambiguous where there are no columns)
  const Tensor m = x.dim() == 2 ? x : x.reshape({c10::multiply_integers(x.sizes().slice(0, x.dim() - 1)), x.size(-1)});
  return has_rows(m) ? m : m.contiguous();
}
Tensor with_shape(const Tensor& y, const Tensor& x) {
  if (x.dim() == 2) return y;
  auto shape = x.sizes().vec();
  shape.back() = y.size(1);
  return y.view(shape);
}

// A matrix that the backward pass takes, kept the way torch keeps tensors: saved-tensor hooks see it, and may hold it
// elsewhere or make it again.
struct SavedMatrix {
  torch::autograd::SavedVariable bytes;
  int64_t rows = 0, cols = 0;
  void save(const Matrix& m) {
    bytes = torch::autograd::SavedVariable(m.bytes(), false);
    rows = m.rows(), cols = m.cols();
  }
  Matrix unpack(const c10::Device& device) const {
    const Tensor b = bytes.unpack();
    TORCH_CHECK(b.scalar_type() == at::kByte && b.device() == device && b.dim() == 1 &&
                    b.numel() == Matrix::Layout(rows, cols).bytes && b.is_contiguous() &&
                    reinterpret_cast<uintptr_t>(b.const_data_ptr()) % 16 == 0,
                "a saved-tensor hook gave the 8-bit linear layer something else back than it was given");
    return Matrix::over(b.storage(), b.storage_offset(), rows, cols);
  }
};

// The layer's node in the graph.  It holds what the backward pass takes as members: as a torch::autograd::Function, with a
// context that keeps them by name, forward and backward of a small layer took 198 us of host, so 160 (torch's own
// linear: 207).  What that class does besides is done here: saved tensors' hooks, the refusal of tangents and of second
// passes, and only the gradients that are asked for.
struct LinearBackward : torch::autograd::Node {
  SavedMatrix qt, qwt;  // x's transpose, w's
  Tensor grad_w;
  std::vector<int64_t> x_shape;
  at::ScalarType x_type, w_type;
  bool need_x, need_w, released = false;

  variable_list apply(variable_list&& grads) override {
    TORCH_CHECK(!at::GradMode::is_enabled(), "the 8-bit linear layer is differentiable once: no create_graph");
    TORCH_CHECK(!released, "backward through the same 8-bit linear layer a second time: give retain_graph=True the first time");
    const Tensor& dy = grads[0];
    if (!dy.defined()) return {Tensor(), Tensor()};
    // What this pass asks for may be less than what could be had (torch.autograd.grad, inputs=): grad_w is then left alone.
    const bool want_x = need_x && task_should_compute_output(0), want_w = need_w && task_should_compute_output(1);
    const c10::cuda::CUDAGuard guard(dy.device());
    Matrix q, qdt;
    quantize(rows_of(dy), false, want_x ? &q : nullptr, want_w ? &qdt : nullptr);
    Tensor dx, dw;
    if (want_x) {
      dx = product(q, qwt.unpack(dy.device()), x_type);
      if (x_shape.size() != 2) dx = dx.view(x_shape);
    }
    if (want_w) {
      const Matrix x = qt.unpack(dy.device());
      if (grad_w.defined()) {
        multiply(qdt, x, grad_w, true);
        // Torch orders streams by the gradients that nodes pass on, and this one passes none: the stream that w's would have
        // gone to, for which the caller of backward() waits, is made to wait here.
        const c10::Stream here = c10::cuda::getCurrentCUDAStream(dy.get_device()).unwrap();
        const auto there = next_edge(1).function->stream();
        if (there && *there != here) {
          c10::Event done(c10::DeviceType::CUDA);
          done.record(here);
          done.block(*there);
        }
      } else {
        dw = product(qdt, x, w_type);
      }
    }
    return {dx, dw};
  }
  void release_variables() override {
    qt.bytes.reset_data();
    qwt.bytes.reset_data();
    grad_w = Tensor();
    released = true;
  }
  std::string name() const override { return "E4M3LinearBackward"; }
};

// A tangent would be lost, which forward mode takes as a derivative of zero.
void refuse_tangent(const Tensor& t, const char* what, const char* by = "the 8-bit linear layer") {
  TORCH_CHECK(!c10::AutogradState::get_tls_state().get_fw_grad_mode() || !t._fw_grad(0).defined(), what,
              " has a tangent: ", by, " has no forward-mode derivative");
}
void check_activations(const Tensor& x) {
  TORCH_CHECK_VALUE(x.dim() >= 1 && is_real(x), "x must be a CUDA float32 or bfloat16 tensor");
  refuse_tangent(x, "x");
}

// linear(x, w, grad_w or None) -> y
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 3, "linear takes 3 arguments");
  const Tensor &x = tensor_of(a[0], "x"), &w = tensor_of(a[1], "w");
  check_activations(x);
  TORCH_CHECK_VALUE(w.dim() == 2 && is_real(w) && w.device() == x.device(), "w must be a float32 or bfloat16 matrix beside x");
  TORCH_CHECK_VALUE(w.size(1) == x.size(-1), "inner sizes differ: ", x.size(-1), " and ", w.size(1));
  refuse_tangent(w, "w");
  c10::optional<Tensor> grad_w;
  if (a[2] != Py_None) {
    grad_w = tensor_of(a[2], "grad_w");
    TORCH_CHECK_VALUE(grad_w->scalar_type() == at::kFloat && grad_w->sizes() == w.sizes() && grad_w->device() == x.device() &&
                          has_rows(*grad_w),
                      "grad_w must be a float32 tensor of w's shape beside it");
  }
  const bool on = at::GradMode::is_enabled(), need_x = on && x.requires_grad(), need_w = on && w.requires_grad();
  TORCH_CHECK_VALUE(!on || !grad_w || need_w, "grad_w would never be added to: w requires no gradient");
  const c10::cuda::CUDAGuard guard(x.device());
  Matrix q, qt, qw, qwt;
  Tensor y;
  {
    const at::AutoDispatchBelowADInplaceOrView below;  // what follows is the layer's own: no graph of its parts
    quantize(rows_of(x), false, &q, need_w ? &qt : nullptr);
    quantize(rows_of(w), true, &qw, need_x ? &qwt : nullptr);
    y = with_shape(product(q, qw, x.scalar_type()), x);
  }
  if (need_x || need_w) {
    const std::shared_ptr<LinearBackward> node(new LinearBackward(), torch::autograd::deleteNode);
    if (need_w) node->qt.save(qt);
    if (need_x) node->qwt.save(qwt);
    if (grad_w) node->grad_w = *grad_w;
    node->x_shape = x.sizes().vec();
    node->x_type = x.scalar_type(), node->w_type = w.scalar_type();
    node->need_x = need_x, node->need_w = need_w;
    node->set_next_edges(torch::autograd::collect_next_edges(x, w));
    torch::autograd::set_history(y, node);
  }
  return THPVariable_Wrap(y);
  END_HANDLE_TH_ERRORS
}

// linear_held(x, codes, scales) -> y
PyObject* linear_held(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 3, "linear_held takes 3 arguments");
  const Tensor& x = tensor_of(a[0], "x");
  check_activations(x);
  const Matrix w = Matrix::checked(a[1], a[2]);
  TORCH_CHECK_VALUE(w.codes.device() == x.device(), "the weight is on another device than x");
  TORCH_CHECK_VALUE(w.cols() == x.size(-1), "inner sizes differ: ", x.size(-1), " and ", w.cols());
  TORCH_CHECK_VALUE(!(at::GradMode::is_enabled() && x.requires_grad()),
                    "a quantised weight passes no gradient: give linear() the weight itself");
  const c10::cuda::CUDAGuard guard(x.device());
  const Tensor m = rows_of(x);
  const Matrix q = Matrix::empty(m.size(0), m.size(1));
  const Tensor y = at::empty({q.rows(), w.rows()}, m.options());
  const mpadam_e4m3_product p = product_of(q, w, y, false);
  check(mpadam_e4m3_quantize_matmul(m.const_data_ptr(), type_of(m), q.rows() > 1 ? std::max(m.stride(0), q.cols()) : q.cols(), &p,
                                    current_stream(m)));
  return THPVariable_Wrap(with_shape(y, x));
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------
// Layer normalisation
// ---------------------------------------------------------------------------
int64_t row_stride(const Tensor& m) { return m.size(0) > 1 ? std::max(m.stride(0), m.size(1)) : m.size(1); }
const void* pointer(const Tensor& t) { return t.defined() ? t.const_data_ptr() : nullptr; }

// The norm's node in the graph, of the same make as the linear layer's.  x and w are kept as inputs (torch then refuses a
// backward pass after one of them was written to), the rows' means and 1 / sigmas as one tensor.
struct LayerNormBackward : torch::autograd::Node {
  torch::autograd::SavedVariable x, w, stats;
  at::ScalarType w_type;
  bool has_w, has_b, need_x, need_w, need_b, released = false;

  variable_list apply(variable_list&& grads) override {
    TORCH_CHECK(!at::GradMode::is_enabled(), "layer_norm is differentiable once: no create_graph");
    TORCH_CHECK(!released, "backward through the same layer_norm a second time: give retain_graph=True the first time");
    const Tensor& dy = grads[0];
    if (!dy.defined()) return {Tensor(), Tensor(), Tensor()};
    const bool want_x = need_x && task_should_compute_output(0), want_w = need_w && task_should_compute_output(1),
               want_b = need_b && task_should_compute_output(2);
    if (!want_x && !want_w && !want_b) return {Tensor(), Tensor(), Tensor()};
    const c10::cuda::CUDAGuard guard(dy.device());
    const Tensor in = x.unpack(), weight = has_w ? w.unpack() : Tensor(), st = stats.unpack();
    const Tensor mx = rows_of(in), md = rows_of(dy);
    const int64_t rows = mx.size(0), cols = mx.size(1);
    TORCH_CHECK(in.device() == dy.device() && in.sizes() == dy.sizes() && in.scalar_type() == dy.scalar_type() && st.dim() == 2 &&
                    st.size(0) == 2 && st.size(1) == rows && st.scalar_type() == at::kFloat && st.is_contiguous() &&
                    st.device() == dy.device() &&
                    (!has_w || (weight.scalar_type() == w_type && weight.numel() == cols && weight.device() == dy.device())),
                "a saved-tensor hook gave layer_norm something else back than it was given");
    const Tensor mw = has_w ? weight.contiguous() : Tensor();
    Tensor dx, dw, db, work;
    mpadam_layer_norm_grad p{};
    p.x = mx.const_data_ptr(), p.ldx = row_stride(mx);
    p.dy = md.const_data_ptr(), p.lddy = row_stride(md);
    p.w = pointer(mw);
    p.mean = st.const_data_ptr<float>(), p.rstd = p.mean + rows;
    p.rows = rows, p.cols = cols;
    p.x_dtype = type_of(mx);
    p.w_dtype = has_w || has_b ? (w_type == at::kFloat ? MPADAM_F32 : MPADAM_BF16) : MPADAM_F32;
    if (want_x) {
      dx = at::empty(in.sizes(), in.options());
      p.dx = dx.data_ptr(), p.lddx = cols;
    }
    const auto vector = md.options().dtype(w_type);
    if (want_w) dw = at::empty({cols}, vector), p.dw = dw.data_ptr();
    if (want_b) db = at::empty({cols}, vector), p.db = db.data_ptr();
    if (want_w || want_b) {
      check(mpadam_layer_norm_workspace(rows, cols, &p.workspace_bytes));
      work = at::empty({p.workspace_bytes}, md.options().dtype(at::kByte));
      p.workspace = work.data_ptr();
    }
    check(mpadam_layer_norm_backward(&p, current_stream(md)));
    return {dx, dw, db};
  }
  void release_variables() override {
    x.reset_data();
    w.reset_data();
    stats.reset_data();
    released = true;
  }
  std::string name() const override { return "LayerNormRowsBackward"; }
};

// layer_norm(x, w or None, b or None, eps) -> y
PyObject* layer_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 4, "layer_norm takes 4 arguments");
  const Tensor& x = tensor_of(a[0], "x");
  TORCH_CHECK_VALUE(x.dim() >= 1 && is_real(x), "x must be a CUDA float32 or bfloat16 tensor");
  const double eps = PyFloat_AsDouble(a[3]);
  if (PyErr_Occurred()) return nullptr;
  refuse_tangent(x, "x", "layer_norm");
  const int64_t cols = x.size(-1);
  Tensor w, b;
  auto vector = [&](PyObject* o, const char* what) {
    const Tensor& v = tensor_of(o, what);
    TORCH_CHECK_VALUE(v.dim() == 1 && v.size(0) == cols && v.device() == x.device() &&
                          (v.scalar_type() == at::kFloat || v.scalar_type() == x.scalar_type()),
                      what, " must be a tensor of ", cols, " elements beside x, float32 or of x's type");
    refuse_tangent(v, what, "layer_norm");
    return v;
  };
  if (a[1] != Py_None) w = vector(a[1], "weight");
  if (a[2] != Py_None) b = vector(a[2], "bias");
  TORCH_CHECK_VALUE(!w.defined() || !b.defined() || w.scalar_type() == b.scalar_type(), "weight and bias differ in their type");
  const auto w_type = w.defined() ? w.scalar_type() : b.defined() ? b.scalar_type() : at::kFloat;
  const bool on = at::GradMode::is_enabled(), need_x = on && x.requires_grad(),
             need_w = on && w.defined() && w.requires_grad(), need_b = on && b.defined() && b.requires_grad();
  const bool need = need_x || need_w || need_b;
  const c10::cuda::CUDAGuard guard(x.device());
  Tensor y, stats;
  {
    const at::AutoDispatchBelowADInplaceOrView below;
    const Tensor m = rows_of(x), mw = w.defined() ? w.contiguous() : w, mb = b.defined() ? b.contiguous() : b;
    y = at::empty(x.sizes(), x.options());
    mpadam_layer_norm p{};
    if (need) {
      stats = at::empty({2, m.size(0)}, x.options().dtype(at::kFloat));
      p.mean = stats.data_ptr<float>(), p.rstd = p.mean + m.size(0);
    }
    p.x = m.const_data_ptr(), p.ldx = row_stride(m);
    p.w = pointer(mw), p.b = pointer(mb);
    p.y = y.data_ptr(), p.ldy = cols;
    p.rows = m.size(0), p.cols = cols;
    p.x_dtype = type_of(m), p.w_dtype = w_type == at::kFloat ? MPADAM_F32 : MPADAM_BF16;
    p.eps = (float)eps;
    check(mpadam_layer_norm_forward(&p, current_stream(m)));
  }
  if (need) {
    const std::shared_ptr<LayerNormBackward> node(new LayerNormBackward(), torch::autograd::deleteNode);
    node->x = torch::autograd::SavedVariable(x, false);
    if (w.defined()) node->w = torch::autograd::SavedVariable(w, false);
    node->stats = torch::autograd::SavedVariable(stats, false);
    node->w_type = w_type;
    node->has_w = w.defined(), node->has_b = b.defined();
    node->need_x = need_x, node->need_w = need_w, node->need_b = need_b;
    node->set_next_edges(torch::autograd::collect_next_edges(x, w, b));
    torch::autograd::set_history(y, node);
  }
  return THPVariable_Wrap(y);
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------------------
// Weights in NVFP4
// ---------------------------------------------------------------------------
// The matrix that codes, scales, a scale and a shape make up.
mpadam_nvfp4_matrix nvfp4_of(PyObject* c, PyObject* s, PyObject* scale, PyObject* rows, PyObject* cols) {
  const Tensor &codes = tensor_of(c, "codes"), &scales = tensor_of(s, "scales");
  mpadam_nvfp4_matrix w{};
  w.rows = PyLong_AsLongLong(rows), w.cols = PyLong_AsLongLong(cols);
  w.global_scale = (float)PyFloat_AsDouble(scale);
  if (PyErr_Occurred()) throw python_error();
  TORCH_CHECK_VALUE(w.rows >= 0 && w.cols >= 0 && w.rows <= INT32_MAX && w.cols <= INT32_MAX, "rows and columns must be in [0, 2^31)");
  const int64_t numel = w.rows * w.cols;
  TORCH_CHECK_VALUE(codes.scalar_type() == at::kByte && codes.is_cuda() && codes.is_contiguous() && codes.numel() == (numel + 1) / 2,
                    "codes must be a contiguous CUDA uint8 tensor of ", (numel + 1) / 2, " bytes, two codes each");
  TORCH_CHECK_VALUE((scales.scalar_type() == at::kByte || scales.scalar_type() == kCodes) && scales.device() == codes.device() &&
                        scales.is_contiguous() && scales.numel() == (numel + 15) / 16,
                    "scales must be a contiguous tensor of ", (numel + 15) / 16, " E4M3 codes (uint8 or float8_e4m3fn) beside the codes");
  TORCH_CHECK_VALUE(w.global_scale > 0.0f && w.global_scale <= 3.402823466e38f, "global_scale must be a finite binary32 above 0");
  w.codes = static_cast<const uint8_t*>(codes.const_data_ptr());
  w.scales = static_cast<const uint8_t*>(scales.const_data_ptr());
  return w;
}

// check_nvfp4(codes, scales, global scale, rows, cols)
PyObject* check_nvfp4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 5, "check_nvfp4 takes 5 arguments");
  nvfp4_of(a[0], a[1], a[2], a[3], a[4]);
  Py_RETURN_NONE;
  END_HANDLE_TH_ERRORS
}

// nvfp4_linear(x, codes, scales, global scale, rows, cols) -> y
PyObject* nvfp4_linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_VALUE(n == 6, "nvfp4_linear takes 6 arguments");
  const Tensor& x = tensor_of(a[0], "x");
  TORCH_CHECK_VALUE(x.dim() >= 1 && is_real(x), "x must be a CUDA float32 or bfloat16 tensor");
  refuse_tangent(x, "x", "a product with an NVFP4 weight");
  const mpadam_nvfp4_matrix w = nvfp4_of(a[1], a[2], a[3], a[4], a[5]);
  TORCH_CHECK_VALUE(tensor_of(a[1], "codes").device() == x.device(), "the weight is on another device than x");
  TORCH_CHECK_VALUE(w.cols == x.size(-1), "inner sizes differ: ", x.size(-1), " and ", w.cols);
  TORCH_CHECK_VALUE(!(at::GradMode::is_enabled() && x.requires_grad()), "an NVFP4 weight passes no gradient");
  const c10::cuda::CUDAGuard guard(x.device());
  const Tensor m = rows_of(x);
  const Tensor y = at::empty({m.size(0), w.rows}, m.options());
  check(mpadam_nvfp4_linear(m.const_data_ptr(), type_of(m), m.size(0), row_stride(m), &w, y.data_ptr(), w.rows, current_stream(m)));
  return THPVariable_Wrap(with_shape(y, x));
  END_HANDLE_TH_ERRORS
}

PyObject* set_error(PyObject*, PyObject* cls) {
  Py_INCREF(cls);
  Py_XSETREF(g_error, cls);
  Py_RETURN_NONE;
}

#define MPADAM_FAST(f) reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)), METH_FASTCALL, nullptr
PyMethodDef kMethods[] = {{"list_spec", MPADAM_FAST(list_spec)},
                          {"matrix_spec", MPADAM_FAST(matrix_spec)},
                          {"adamw_create", MPADAM_FAST(adamw_create)},
                          {"adamw_step", MPADAM_FAST(adamw_step)},
                          {"grad_norm", MPADAM_FAST(grad_norm)},
                          {"muon_create", MPADAM_FAST(muon_create)},
                          {"muon_step", MPADAM_FAST(muon_step)},
                          {"orthogonalize", MPADAM_FAST(orthogonalize)},
                          {"check_matrix", MPADAM_FAST(check_matrix)},
                          {"quantize", MPADAM_FAST(py_quantize)},
                          {"matmul", MPADAM_FAST(py_matmul)},
                          {"linear", MPADAM_FAST(linear)},
                          {"linear_held", MPADAM_FAST(linear_held)},
                          {"layer_norm", MPADAM_FAST(layer_norm)},
                          {"check_nvfp4", MPADAM_FAST(check_nvfp4)},
                          {"nvfp4_linear", MPADAM_FAST(nvfp4_linear)},
                          {"set_error", set_error, METH_O, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_mpadam_torch", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mpadam_torch() { return PyModule_Create(&kModule); }
