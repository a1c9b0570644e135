// Argument marshalling of the entry points that a program calls once or more for every layer (routing with and without the
// normalisation or from logits, forward, backward, those of 4-bit and of 8-bit floats), for binding.py: the checks and addresses of up to thirty tensors and the call itself.  In
// Python these are 0.2 us a tensor and 0.1 us an argument (0.6 where its shape and dtype are checked), 7 us of a call that launches two
// kernels.  Nothing is kept from one call
// for the next but the addresses of the library's functions.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <dlfcn.h>
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <exception>
#include <string>
#include <type_traits>

#include "btx_moe.h"

namespace {

struct Library {
  decltype(&btx_moe_route_workspace_bytes) route_bytes;
  decltype(&btx_moe_route) route;
  decltype(&btx_moe_norm_route) norm_route;
  decltype(&btx_moe_ff_forward_workspace_bytes) forward_bytes;
  decltype(&btx_moe_ff_forward) forward;
  decltype(&btx_moe_ff_backward_workspace_bytes) backward_bytes;
  decltype(&btx_moe_ff_backward) backward;
  decltype(&btx_moe_group_route_workspace_bytes) group_route_bytes;
  decltype(&btx_moe_group_route) group_route;
  decltype(&btx_moe_group_route_backward) group_route_backward;
  decltype(&btx_mx4_scale_pitch) mx4_pitch;
  decltype(&btx_mx4_quantize) mx4_quantize;
  decltype(&btx_mx4_dequantize) mx4_dequantize;
  decltype(&btx_moe_ff_forward_mx4_workspace_bytes) forward_mx4_bytes;
  decltype(&btx_moe_ff_forward_mx4) forward_mx4;
  decltype(&btx_fp8_code_pitch) fp8_pitch;
  decltype(&btx_fp8_scale_pitch) fp8_scale_pitch;
  decltype(&btx_fp8_quantize) fp8_quantize;
  decltype(&btx_fp8_dequantize) fp8_dequantize;
  decltype(&btx_rmsnorm_fp8) rmsnorm_fp8;
  decltype(&btx_fp8_matmul_workspace_bytes) matmul_bytes;
  decltype(&btx_fp8_matmul) matmul;
  decltype(&btx_moe_ff_forward_fp8_workspace_bytes) forward_fp8_bytes;
  decltype(&btx_moe_ff_forward_fp8) forward_fp8;
} lib{};

struct PyError {};                       // a Python exception has been set
[[noreturn]] void fail(PyObject* type, const char* what) {
  PyErr_SetString(type, what);
  throw PyError{};
}
void require(bool ok, const char* what) {
  if (!ok) fail(PyExc_AssertionError, what);
}

const at::Tensor& tensor(PyObject* o) {
  if (!THPVariable_Check(o)) fail(PyExc_TypeError, "a tensor is expected");
  return THPVariable_Unpack(o);
}
// a size or an option as the library takes it
int size32(int64_t n) {
  if (n != (int)n) fail(PyExc_ValueError, "sizes and options have 32 bits");
  return (int)n;
}
// stacked expert matrices: each [rows, cols] matrix contiguous, the experts any distance apart
bool is_stacked(const at::Tensor& w) {
  return w.dim() == 3 && w.stride(2) == 1 && w.stride(1) == w.size(2) && w.stride(0) >= w.size(1) * w.size(2);
}
int64_t stacked(const at::Tensor& w) {
  require(is_stacked(w), "stacked expert matrices only");
  return w.stride(0);
}
// device address (None: NULL)
void* address(PyObject* o, bool or_stacked = false) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  require(t.is_cuda() && (t.is_contiguous() || (or_stacked && is_stacked(t))), "device-resident contiguous tensors only");
  return t.data_ptr();
}
template <typename T> T* address_of(PyObject* o) { return static_cast<T*>(address(o)); }
int dtype_code(const at::Tensor& t) {
  if (t.scalar_type() == at::kFloat) return BTX_F32;
  if (t.scalar_type() == at::kBFloat16) return BTX_BF16;
  fail(PyExc_TypeError, "unsupported dtype");
}
// address() of a tensor of this dtype and shape
template <typename T> T* typed(PyObject* o, at::ScalarType type, at::IntArrayRef shape, const std::string& what) {
  if (o == Py_None) return nullptr;
  const at::Tensor& t = tensor(o);
  if (t.scalar_type() != type || t.sizes() != shape) {
    std::string text = what + " is " + (type == at::kInt ? "int32" : type == at::kFloat ? "float32" : type == at::kByte ? "uint8" : "bfloat16") + " (";
    for (const int64_t n : shape) text += std::to_string(n) + ", ";
    if (!shape.empty()) text.resize(text.size() - 2);
    fail(PyExc_ValueError, (text + ")").c_str());
  }
  return address_of<T>(o);
}
const at::Tensor& matrix(PyObject* o) {
  const at::Tensor& t = tensor(o);
  if (t.dim() != 2) fail(PyExc_ValueError, "a matrix is expected");
  return t;
}
// Shapes and strides of the experts that x goes through.  The library takes one expert stride for W1 and W3, and one dtype
struct Experts {
  int64_t T, d, E, f, s13, s2;
  Experts(const at::Tensor& x, const at::Tensor& W1, const at::Tensor& W3, const at::Tensor& W2)
      : T(x.size(0)), d(x.size(1)), E(0), f(0), s13(stacked(W1)), s2(stacked(W2)) {
    E = W1.size(0);
    f = W1.size(2);
    for (const int64_t n : {T, d, E, f}) size32(n);
    require(W1.size(1) == d && W3.sizes() == W1.sizes() && W2.size(0) == E && W2.size(1) == f && W2.size(2) == d &&
                W1.scalar_type() == x.scalar_type() && W3.scalar_type() == x.scalar_type() && W2.scalar_type() == x.scalar_type(),
            "W1, W3 [E, d, f] and W2 [E, f, d] of x's dtype");
    require(E == 1 || (is_stacked(W3) && W3.stride(0) == s13), "W3 is stacked like W1");
  }
};
int64_t integer(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw PyError{};
  return v;
}
int int32(PyObject* o) { return size32(integer(o)); }
float real(PyObject* o) {
  const double v = PyFloat_AsDouble(o);
  if (v == -1.0 && PyErr_Occurred()) throw PyError{};
  return (float)v;
}
// out: attributes of a Routing
struct RoutingPtrs {
  void* at[10];
  int k;
  RoutingPtrs(PyObject* r, const char* const* names, int n) : k(0) {
    for (int i = 0; i < n; ++i) {
      PyObject* o = PyObject_GetAttrString(r, names[i]);
      if (!o) throw PyError{};
      try {
        at[i] = address(o);
        if (i == 0) k = size32(matrix(o).size(1));       // topk_idx
      } catch (...) {
        Py_DECREF(o);
        throw;
      }
      Py_DECREF(o);                                      // the Routing holds on to it
    }
  }
};

// an attribute; the object holds on to it, too
struct Attr {
  PyObject* o;
  Attr(PyObject* of, const char* name) : o(PyObject_GetAttrString(of, name)) {
    if (!o) throw PyError{};
  }
  ~Attr() { Py_DECREF(o); }
  Attr(const Attr&) = delete;
  Attr& operator=(const Attr&) = delete;
  operator PyObject*() const { return o; }
};
// codes [.., n, K/2] and scales of an Mx4
struct Mx4Ptrs {
  uint8_t *codes, *scales;
  Mx4Ptrs(PyObject* q, at::IntArrayRef batch, int64_t n, int64_t K, const std::string& what) {
    const Attr c(q, "codes"), s(q, "scales"), k(q, "K");
    if (integer(k) != K) fail(PyExc_ValueError, (what + ".K is " + std::to_string(K)).c_str());
    at::DimVector shape(batch.begin(), batch.end());
    shape.append({n, K / 2});
    codes = typed<uint8_t>(c, at::kByte, shape, what + ".codes");
    shape.back() = lib.mx4_pitch(K);
    scales = typed<uint8_t>(s, at::kByte, shape, what + ".scales");
  }
};

// Tensors of a call on one device, that of `first`
struct Place {
  int64_t device;
  explicit Place(PyObject* first) : device(tensor(first).is_cuda() ? tensor(first).get_device() : -1) {}
  template <typename T> T* operator()(PyObject* o, at::ScalarType type, at::IntArrayRef shape, const std::string& what) const {
    T* const p = typed<T>(o, type, shape, what);
    if (o != Py_None && tensor(o).get_device() != device) fail(PyExc_ValueError, (what + " is on another device").c_str());
    return p;
  }
};
// codes [.., n, K padded] and scales of an Fp8
struct Fp8Ptrs {
  uint8_t *codes, *scales;
  Fp8Ptrs(const Place& at, PyObject* q, at::IntArrayRef batch, int64_t n, int64_t K, const std::string& what) {
    const Attr c(q, "codes"), s(q, "scales"), k(q, "K");
    if (integer(k) != K) fail(PyExc_ValueError, (what + ".K is " + std::to_string(K)).c_str());
    at::DimVector shape(batch.begin(), batch.end());
    shape.append({n, lib.fp8_pitch(K)});
    codes = at.operator()<uint8_t>(c, at::kByte, shape, what + ".codes");
    shape.back() = lib.fp8_scale_pitch(K);
    scales = at.operator()<uint8_t>(s, at::kByte, shape, what + ".scales");
  }
};

template <typename Call> PyObject* called(Call call) {
  int status;
  Py_BEGIN_ALLOW_THREADS
  status = call();
  Py_END_ALLOW_THREADS
  return PyLong_FromLong(status);
}
// The call with this workspace, or, where it is too small or there is none, minus the bytes that one has to have
template <typename Call> PyObject* with_workspace(PyObject* workspace, size_t bytes, Call call, const Place* place = nullptr) {
  if (workspace != Py_None) {
    const at::Tensor& w = tensor(workspace);
    if (place && w.get_device() != place->device) fail(PyExc_ValueError, "workspace is on another device");
    const size_t has = (size_t)w.numel() * w.element_size();
    if (has >= bytes) {
      void* const at = address(workspace);
      int status;
      Py_BEGIN_ALLOW_THREADS
      status = call(at, has);
      Py_END_ALLOW_THREADS
      return PyLong_FromLong(status);
    }
  }
  return PyLong_FromLongLong(-(long long)std::max<size_t>(bytes, 256));
}

// arguments by position; Python exceptions and C++ ones end here
template <typename Body> PyObject* guarded(Py_ssize_t n, Py_ssize_t expected, Body body) {
  try {
    if (!lib.route) fail(PyExc_RuntimeError, "the library is not loaded");
    if (n != expected) fail(PyExc_TypeError, "wrong number of arguments");
    return body();
  } catch (const PyError&) {
  } catch (const std::exception& e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  return nullptr;
}

const char* const kRouting[10] = {"topk_idx", "gates", "probs", "counts", "offsets", "perm", "inv_pos", "gate_sum", "prob_sum", "lb_loss"};

// x, W_router, b_router, U, k, route_mode, lb_mode, lb_alpha, tau, capacity_factor, routing, workspace, stream
PyObject* route(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 13, [&] {
    const at::Tensor &x = matrix(a[0]), &W = matrix(a[1]);
    const int T = size32(x.size(0)), d = size32(x.size(1)), E = size32(W.size(1)), k = int32(a[4]);
    require(W.size(0) == d && W.scalar_type() == at::kFloat, "W_router is [d, E] fp32");
    const int dt = dtype_code(x), mode = int32(a[5]), lb_mode = int32(a[6]);
    const float alpha = real(a[7]), tau = real(a[8]), cf = real(a[9]);
    const RoutingPtrs r(a[10], kRouting, 10);
    const void* const xp = address(a[0]);
    const float *Wp = address_of<float>(a[1]), *bp = address_of<float>(a[2]), *Up = address_of<float>(a[3]);
    void* const stream = reinterpret_cast<void*>(integer(a[12]));
    return with_workspace(a[11], lib.route_bytes(T, d, E, k), [&](void* ws, size_t bytes) {
      return lib.route(xp, dt, Wp, bp, Up, T, d, E, k, mode, lb_mode, alpha, tau, cf, (int32_t*)r.at[0], (float*)r.at[1], (float*)r.at[2],
                       (int32_t*)r.at[3], (int32_t*)r.at[4], (int32_t*)r.at[5], (int32_t*)r.at[6], (float*)r.at[7], (float*)r.at[8],
                       (float*)r.at[9], ws, bytes, stream);
    });
  });
}

// h, gain, eps, xn, rstd, and route()'s from W_router on
PyObject* norm_route(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 17, [&] {
    const at::Tensor &h = matrix(a[0]), &gain = tensor(a[1]), &W = matrix(a[5]);
    const int T = size32(h.size(0)), d = size32(h.size(1)), E = size32(W.size(1)), k = int32(a[8]);
    require(W.size(0) == d && W.scalar_type() == at::kFloat, "W_router is [d, E] fp32");
    require(gain.dim() == 1 && gain.size(0) == d && gain.scalar_type() == at::kFloat, "gain is [d] fp32");
    const int dt = dtype_code(h), mode = int32(a[9]), lb_mode = int32(a[10]);
    const float eps = real(a[2]), alpha = real(a[11]), tau = real(a[12]), cf = real(a[13]);
    const RoutingPtrs r(a[14], kRouting, 10);
    const void* const hp = address(a[0]);
    void* const xn = address(a[3]);
    float* const rstd = address_of<float>(a[4]);
    const float *gp = address_of<float>(a[1]), *Wp = address_of<float>(a[5]), *bp = address_of<float>(a[6]), *Up = address_of<float>(a[7]);
    void* const stream = reinterpret_cast<void*>(integer(a[16]));
    return with_workspace(a[15], lib.route_bytes(T, d, E, k), [&](void* ws, size_t bytes) {
      return lib.norm_route(hp, dt, gp, eps, xn, rstd, Wp, bp, Up, T, d, E, k, mode, lb_mode, alpha, tau, cf, (int32_t*)r.at[0],
                            (float*)r.at[1], (float*)r.at[2], (int32_t*)r.at[3], (int32_t*)r.at[4], (int32_t*)r.at[5], (int32_t*)r.at[6],
                            (float*)r.at[7], (float*)r.at[8], (float*)r.at[9], ws, bytes, stream);
    });
  });
}

// x, W1, W3, W2, routing, residual, out, h1, h3, workspace, stream
PyObject* forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 11, [&] {
    const at::Tensor &x = matrix(a[0]), &W1 = tensor(a[1]), &W3 = tensor(a[2]), &W2 = tensor(a[3]);
    const Experts w(x, W1, W3, W2);
    static const char* const names[] = {"topk_idx", "gates", "offsets", "perm", "inv_pos"};
    const RoutingPtrs r(a[4], names, 5);
    const int dt = dtype_code(x), k = r.k;
    const void *xp = address(a[0]), *w1 = address(a[1], true), *w3 = address(a[2], true), *w2 = address(a[3], true), *res = address(a[5]);
    void *out = address(a[6]), *h1 = address(a[7]), *h3 = address(a[8]);
    void* const stream = reinterpret_cast<void*>(integer(a[10]));
    return with_workspace(a[9], lib.forward_bytes((int)w.T, (int)w.d, (int)w.f, (int)w.E, k, dt), [&](void* ws, size_t bytes) {
      return lib.forward(xp, w1, w3, w2, dt, w.s13, w.s2, (int)w.T, (int)w.d, (int)w.f, (int)w.E, k, (const float*)r.at[1], (const int32_t*)r.at[2],
                         (const int32_t*)r.at[3], (const int32_t*)r.at[4], res, out, h1, h3, ws, bytes, stream);
    });
  });
}

// dY, x, W_router, W1, W3, W2, routing, h1, h3, route_mode, lb_mode, lb_alpha, lb_grad_scale, flags, noise, tau, dX, dW_router, db_router,
// dW1, dW3, dW2, weight gradients in fp32, workspace, stream
PyObject* backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 25, [&] {
    const at::Tensor &x = matrix(a[1]), &W1 = tensor(a[3]), &W3 = tensor(a[4]), &W2 = tensor(a[5]);
    const Experts w(x, W1, W3, W2);
    const bool dw_f32 = PyObject_IsTrue(a[22]) == 1;
    for (int i = 0; i < 3; ++i) {
      if (a[19 + i] == Py_None) continue;
      const at::Tensor &dW = tensor(a[19 + i]), &W = tensor(a[3 + i]);
      require(dW.sizes() == W.sizes() && stacked(dW) == stacked(W), "dW is stacked like W");
      require(dW.scalar_type() == (dw_f32 ? at::kFloat : at::kBFloat16), "dW is of dW_dtype");
    }
    static const char* const names[] = {"topk_idx", "gates", "probs", "offsets", "perm", "inv_pos", "gate_sum", "prob_sum", "counts"};
    const RoutingPtrs r(a[6], names, 9);
    const int dt = dtype_code(x), k = r.k, mode = int32(a[9]), lb_mode = int32(a[10]), dw_dt = dw_f32 ? BTX_F32 : BTX_BF16;
    const float alpha = real(a[11]), scale = real(a[12]), tau = real(a[15]);
    const unsigned flags = (unsigned)int32(a[13]);
    const void *dY = address(a[0]), *xp = address(a[1]), *w1 = address(a[3], true), *w3 = address(a[4], true), *w2 = address(a[5], true);
    const void *h1 = address(a[7]), *h3 = address(a[8]);
    const float *Wr = address_of<float>(a[2]), *noise = address_of<float>(a[14]);
    void *dX = address(a[16]), *dW1 = address(a[19], true), *dW3 = address(a[20], true), *dW2 = address(a[21], true);
    float *dWr = address_of<float>(a[17]), *dbr = address_of<float>(a[18]);
    void* const stream = reinterpret_cast<void*>(integer(a[24]));
    return with_workspace(a[23], lib.backward_bytes((int)w.T, (int)w.d, (int)w.f, (int)w.E, k, dt), [&](void* ws, size_t bytes) {
      return lib.backward(dY, xp, Wr, w1, w3, w2, dt, w.s13, w.s2, (int)w.T, (int)w.d, (int)w.f, (int)w.E, k, mode, lb_mode, alpha, scale, flags, noise,
                          tau, (const int32_t*)r.at[0], (const float*)r.at[1], (const float*)r.at[2], (const int32_t*)r.at[3],
                          (const int32_t*)r.at[4], (const int32_t*)r.at[5], (const float*)r.at[6], (const float*)r.at[7],
                          (const int32_t*)r.at[8], h1, h3, dX, dWr, dbr, dW1, dW3, dW2, dw_dt, ws, bytes, stream);
    });
  });
}

// logits, k, score_fn, bias, n_groups, topk_groups, group_score, renorm, scale, routing, workspace, stream
PyObject* group_route(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 12, [&] {
    const at::Tensor& logits = matrix(a[0]);
    const int T = size32(logits.size(0)), E = size32(logits.size(1));
    const int k = int32(a[1]), score_fn = int32(a[2]), groups = int32(a[4]), keep = int32(a[5]), group_score = int32(a[6]), renorm = int32(a[7]);
    const float scale = real(a[8]);
    const int dt = dtype_code(logits);
    const void* const l = address(a[0]);
    const float* const bias = typed<float>(a[3], at::kFloat, {E}, "bias");
    const Attr o_idx(a[9], "topk_idx"), o_gates(a[9], "gates"), o_scores(a[9], "scores"), o_counts(a[9], "counts"), o_offsets(a[9], "offsets"),
        o_perm(a[9], "perm"), o_inv(a[9], "inv_pos");
    int32_t* const idx = typed<int32_t>(o_idx, at::kInt, {T, k}, "topk_idx");
    float *const gates = typed<float>(o_gates, at::kFloat, {T, k}, "gates"), *const scores = typed<float>(o_scores, at::kFloat, {T, E}, "scores");
    int32_t *const counts = typed<int32_t>(o_counts, at::kInt, {E}, "counts"), *const offsets = typed<int32_t>(o_offsets, at::kInt, {E + (int64_t)1}, "offsets");
    int32_t *const perm = typed<int32_t>(o_perm, at::kInt, {(int64_t)T * k}, "perm"), *const inv = typed<int32_t>(o_inv, at::kInt, {T, k}, "inv_pos");
    void* const stream = reinterpret_cast<void*>(integer(a[11]));
    const auto call = [&](void* ws, size_t bytes) {
      return lib.group_route(l, dt, bias, T, E, k, score_fn, groups, keep, group_score, renorm, scale, idx, gates, scores, counts, offsets,
                             perm, inv, ws, bytes, stream);
    };
    const size_t bytes = lib.group_route_bytes(T, E, k);
    if (!bytes) return called([&] { return call(nullptr, 0); });
    return with_workspace(a[10], bytes, call);
  });
}

// logits, routing, dgates, score_fn, renorm, scale, dscores, dlogits, workspace (none), stream
PyObject* group_route_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    const at::Tensor& logits = matrix(a[0]);
    const int T = size32(logits.size(0)), E = size32(logits.size(1));
    const int dt = dtype_code(logits), score_fn = int32(a[3]), renorm = int32(a[4]);
    const float scale = real(a[5]);
    const Attr o_idx(a[1], "topk_idx");
    const int k = size32(matrix(o_idx).size(1));
    const void* const l = address(a[0]);
    const int32_t* const idx = typed<int32_t>(o_idx, at::kInt, {T, k}, "topk_idx");
    const float *const dgates = typed<float>(a[2], at::kFloat, {T, k}, "dgates"), *const dscores = typed<float>(a[6], at::kFloat, {T, E}, "dscores");
    void* const out = typed<void>(a[7], logits.scalar_type(), {T, E}, "dlogits");
    void* const stream = reinterpret_cast<void*>(integer(a[9]));
    return called([&] {
      return lib.group_route_backward(l, dt, idx, dgates, dscores, T, E, k, score_fn, renorm, scale, out, stream);
    });
  });
}

// x, axis (of the library), out, workspace (none), stream
PyObject* mx4_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const at::Tensor& x = tensor(a[0]);
    if (x.dim() < 2) fail(PyExc_ValueError, "a matrix or a stack of them is expected");
    const int axis = int32(a[1]), dt = dtype_code(x);
    const at::IntArrayRef batch = x.sizes().slice(0, x.dim() - 2);
    const int64_t rows = x.size(-2), cols = x.size(-1), K = axis ? cols : rows;
    const Mx4Ptrs q(a[2], batch, axis ? rows : cols, K, "out");
    const void* const from = address(a[0]);
    void* const stream = reinterpret_cast<void*>(integer(a[4]));
    return called([&] { return lib.mx4_quantize(from, dt, c10::multiply_integers(batch), rows, cols, axis, q.codes, q.scales, stream); });
  });
}

// q, axis, out, workspace (none), stream
PyObject* mx4_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const at::Tensor& out = tensor(a[2]);
    if (out.dim() < 2) fail(PyExc_ValueError, "a matrix or a stack of them is expected");
    const int axis = int32(a[1]), dt = dtype_code(out);
    const at::IntArrayRef batch = out.sizes().slice(0, out.dim() - 2);
    const int64_t rows = out.size(-2), cols = out.size(-1);
    const Mx4Ptrs q(a[0], batch, axis ? rows : cols, axis ? cols : rows, "q");
    void* const to = address(a[2]);
    void* const stream = reinterpret_cast<void*>(integer(a[4]));
    return called([&] { return lib.mx4_dequantize(q.codes, q.scales, dt, c10::multiply_integers(batch), rows, cols, axis, to, stream); });
  });
}

// x, W1, W3, W2, routing, residual, out, workspace, stream
PyObject* forward_mx4(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    const at::Tensor& x = matrix(a[0]);
    const int T = size32(x.size(0)), d = size32(x.size(1));
    const Attr w1_codes(a[1], "codes"), w2_K(a[3], "K"), o_idx(a[4], "topk_idx");
    const int E = tensor(w1_codes).dim() ? size32(tensor(w1_codes).size(0)) : 0, f = int32(w2_K), k = size32(matrix(o_idx).size(1));
    const Mx4Ptrs W1(a[1], {E}, f, d, "W1"), W3(a[2], {E}, f, d, "W3"), W2(a[3], {E}, d, f, "W2");
    const Attr o_gates(a[4], "gates"), o_offsets(a[4], "offsets"), o_perm(a[4], "perm"), o_inv(a[4], "inv_pos");
    const void *const from = typed<void>(a[0], at::kBFloat16, {T, d}, "x"), *const res = typed<void>(a[5], at::kBFloat16, {T, d}, "residual");
    void* const out = typed<void>(a[6], at::kBFloat16, {T, d}, "out");
    const float* const gates = typed<float>(o_gates, at::kFloat, {T, k}, "gates");
    const int32_t *const offsets = typed<int32_t>(o_offsets, at::kInt, {E + (int64_t)1}, "offsets"),
                  *const perm = typed<int32_t>(o_perm, at::kInt, {(int64_t)T * k}, "perm"),
                  *const inv = typed<int32_t>(o_inv, at::kInt, {T, k}, "inv_pos");
    void* const stream = reinterpret_cast<void*>(integer(a[8]));
    return with_workspace(a[7], lib.forward_mx4_bytes(T, d, f, E, k), [&](void* ws, size_t bytes) {
      return lib.forward_mx4(from, W1.codes, W1.scales, W3.codes, W3.scales, W2.codes, W2.scales, T, d, f, E, k, gates,
                             offsets, perm, inv, res, out, ws, bytes, stream);
    });
  });
}

// x, axis (of the library), block_rows, out, workspace (none), stream
PyObject* fp8_quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&] {
    const at::Tensor& x = tensor(a[0]);
    if (x.dim() < 2) fail(PyExc_ValueError, "a matrix or a stack of them is expected");
    const int axis = int32(a[1]), block_rows = int32(a[2]), dt = dtype_code(x);
    const at::IntArrayRef batch = x.sizes().slice(0, x.dim() - 2);
    const int64_t rows = x.size(-2), cols = x.size(-1);
    const Place at(a[0]);
    const Fp8Ptrs q(at, a[3], batch, axis ? rows : cols, axis ? cols : rows, "out");
    const void* const from = address(a[0]);
    void* const stream = reinterpret_cast<void*>(integer(a[5]));
    return called([&] { return lib.fp8_quantize(from, dt, c10::multiply_integers(batch), rows, cols, axis, block_rows, q.codes, q.scales, stream); });
  });
}

// q, axis, out, workspace (none), stream
PyObject* fp8_dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 5, [&] {
    const at::Tensor& out = tensor(a[2]);
    if (out.dim() < 2) fail(PyExc_ValueError, "a matrix or a stack of them is expected");
    const int axis = int32(a[1]), dt = dtype_code(out);
    const at::IntArrayRef batch = out.sizes().slice(0, out.dim() - 2);
    const int64_t rows = out.size(-2), cols = out.size(-1);
    const Place at(a[2]);
    const Fp8Ptrs q(at, a[0], batch, axis ? rows : cols, axis ? cols : rows, "q");
    void* const to = address(a[2]);
    void* const stream = reinterpret_cast<void*>(integer(a[4]));
    return called([&] { return lib.fp8_dequantize(q.codes, q.scales, dt, c10::multiply_integers(batch), rows, cols, axis, to, stream); });
  });
}

// h, gain, eps, residual, sum, xn, rstd, out, workspace (none), stream
PyObject* rmsnorm_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 10, [&] {
    const at::Tensor& h = matrix(a[0]);
    const int T = size32(h.size(0)), d = size32(h.size(1)), dt = dtype_code(h);
    const at::ScalarType type = h.scalar_type();
    const float eps = real(a[2]);
    const Place at(a[0]);
    const void* const from = address(a[0]);
    const float* const gain = at.operator()<float>(a[1], at::kFloat, {d}, "gain");
    const void* const res = at.operator()<void>(a[3], type, {T, d}, "residual");
    void *const sum = at.operator()<void>(a[4], type, {T, d}, "sum"), *const xn = at.operator()<void>(a[5], type, {T, d}, "xn");
    float* const rstd = at.operator()<float>(a[6], at::kFloat, {T}, "rstd");
    const Fp8Ptrs q(at, a[7], {}, T, d, "out");
    void* const stream = reinterpret_cast<void*>(integer(a[9]));
    return called([&] { return lib.rmsnorm_fp8(from, res, dt, gain, eps, T, d, sum, xn, rstd, q.codes, q.scales, stream); });
  });
}

// a, b, residual, out, workspace, stream
PyObject* fp8_matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 6, [&] {
    const at::Tensor& out = matrix(a[3]);
    const Attr a_K(a[0], "K");
    const int M = size32(out.size(0)), N = size32(out.size(1)), K = int32(a_K), dt = dtype_code(out);
    const Place at(a[3]);
    const Fp8Ptrs A(at, a[0], {}, M, K, "a"), B(at, a[1], {}, N, K, "b");
    const void* const res = at.operator()<void>(a[2], out.scalar_type(), {M, N}, "residual");
    void* const to = address(a[3]);
    void* const stream = reinterpret_cast<void*>(integer(a[5]));
    const auto call = [&](void* ws, size_t bytes) {
      return lib.matmul(A.codes, A.scales, B.codes, B.scales, M, N, K, res, to, dt, ws, bytes, stream);
    };
    const size_t bytes = lib.matmul_bytes(M, N, K);
    if (!bytes) return called([&] { return call(nullptr, 0); });
    return with_workspace(a[4], bytes, call, &at);
  });
}

// x, W1, W3, W2, routing, residual, out, workspace, stream
PyObject* forward_fp8(PyObject*, PyObject* const* a, Py_ssize_t n) {
  return guarded(n, 9, [&] {
    const Attr x_codes(a[0], "codes"), x_K(a[0], "K"), w1_codes(a[1], "codes"), w2_K(a[3], "K"), o_idx(a[4], "topk_idx");
    const int T = size32(matrix(x_codes).size(0)), d = int32(x_K);
    const int E = tensor(w1_codes).dim() ? size32(tensor(w1_codes).size(0)) : 0, f = int32(w2_K), k = size32(matrix(o_idx).size(1));
    const Place at(x_codes);
    const Fp8Ptrs x(at, a[0], {}, T, d, "x"), W1(at, a[1], {E}, f, d, "W1"), W3(at, a[2], {E}, f, d, "W3"), W2(at, a[3], {E}, d, f, "W2");
    const Attr o_gates(a[4], "gates"), o_offsets(a[4], "offsets"), o_perm(a[4], "perm"), o_inv(a[4], "inv_pos");
    const void* const res = at.operator()<void>(a[5], at::kBFloat16, {T, d}, "residual");
    void* const out = at.operator()<void>(a[6], at::kBFloat16, {T, d}, "out");
    const float* const gates = at.operator()<float>(o_gates, at::kFloat, {T, k}, "gates");
    const int32_t *const offsets = at.operator()<int32_t>(o_offsets, at::kInt, {E + (int64_t)1}, "offsets"),
                  *const perm = at.operator()<int32_t>(o_perm, at::kInt, {(int64_t)T * k}, "perm"),
                  *const inv = at.operator()<int32_t>(o_inv, at::kInt, {T, k}, "inv_pos");
    void* const stream = reinterpret_cast<void*>(integer(a[8]));
    return with_workspace(a[7], lib.forward_fp8_bytes(T, d, f, E, k), [&](void* ws, size_t bytes) {
      return lib.forward_fp8(x.codes, x.scales, W1.codes, W1.scales, W3.codes, W3.scales, W2.codes, W2.scales, T, d, f, E, k, gates, offsets, perm,
                             inv, res, out, ws, bytes, stream);
    }, &at);
  });
}

// path of the library, which is loaded already
PyObject* bind(PyObject*, PyObject* path) {
  const char* p = PyUnicode_AsUTF8(path);
  if (!p) return nullptr;
  void* const handle = dlopen(p, RTLD_NOW | RTLD_NOLOAD);
  Library l{};
  auto find = [&](auto& to, const char* name) {
    to = handle ? reinterpret_cast<std::remove_reference_t<decltype(to)>>(dlsym(handle, name)) : nullptr;
    return to != nullptr;
  };
  if (!find(l.route_bytes, "btx_moe_route_workspace_bytes") || !find(l.route, "btx_moe_route") || !find(l.norm_route, "btx_moe_norm_route") ||
      !find(l.forward_bytes, "btx_moe_ff_forward_workspace_bytes") || !find(l.forward, "btx_moe_ff_forward") ||
      !find(l.backward_bytes, "btx_moe_ff_backward_workspace_bytes") || !find(l.backward, "btx_moe_ff_backward") ||
      !find(l.group_route_bytes, "btx_moe_group_route_workspace_bytes") || !find(l.group_route, "btx_moe_group_route") ||
      !find(l.group_route_backward, "btx_moe_group_route_backward") || !find(l.mx4_pitch, "btx_mx4_scale_pitch") ||
      !find(l.mx4_quantize, "btx_mx4_quantize") || !find(l.mx4_dequantize, "btx_mx4_dequantize") ||
      !find(l.forward_mx4_bytes, "btx_moe_ff_forward_mx4_workspace_bytes") || !find(l.forward_mx4, "btx_moe_ff_forward_mx4") ||
      !find(l.fp8_pitch, "btx_fp8_code_pitch") || !find(l.fp8_scale_pitch, "btx_fp8_scale_pitch") || !find(l.fp8_quantize, "btx_fp8_quantize") ||
      !find(l.fp8_dequantize, "btx_fp8_dequantize") || !find(l.rmsnorm_fp8, "btx_rmsnorm_fp8") ||
      !find(l.matmul_bytes, "btx_fp8_matmul_workspace_bytes") || !find(l.matmul, "btx_fp8_matmul") ||
      !find(l.forward_fp8_bytes, "btx_moe_ff_forward_fp8_workspace_bytes") || !find(l.forward_fp8, "btx_moe_ff_forward_fp8")) {
    PyErr_Format(PyExc_RuntimeError, "%s does not have the library's entry points", p);
    return nullptr;
  }
  lib = l;
  Py_RETURN_NONE;
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_O, nullptr}, FAST(route), FAST(norm_route), FAST(forward), FAST(backward), FAST(group_route),
                         FAST(group_route_backward), FAST(mx4_quantize), FAST(mx4_dequantize), FAST(forward_mx4), FAST(fp8_quantize), FAST(fp8_dequantize),
                         FAST(rmsnorm_fp8), FAST(fp8_matmul), FAST(forward_fp8), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
