// The calls around the linears of a block for Python (module `_node`; binding.py gives them their names, defaults and results): few-token
// products, 8-bit activation checkpoints, SwiGLU, layer norm. Each checks what the library cannot see of an address (type, shape, strides,
// device), allocates from torch's caching allocator what the caller has not brought, and makes the library call on the current stream of the
// tensors' device, whichever device is current.
//
// As with NVFP4Linear's node, what it replaces is host time, which is all of the time of a call on a few tokens: through ctypes a product, a norm
// or a SwiGLU of a few tokens took 12.5 to 13.3 us from Python, this way 4.5 to 5.5.
#include "torch_common.h"

#include <ATen/MemoryOverlap.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>

#include <pybind11/pybind11.h>

using nvfp4_torch::matrix;
using nvfp4_torch::raise_status;
using nvfp4_torch::up;

namespace {

enum Save : int64_t { kNothing = 0, kInput = 1, kCkpt8 = 2 };

// ---- arguments -----------------------------------------------------------------------------------------------------------------------
using Args = PyObject* const*;

const at::Tensor& tensor(PyObject* o, const char* where, const char* name) {
  TORCH_CHECK_TYPE(THPVariable_Check(o), where, ": ", name, " is not a tensor");
  return THPVariable_Unpack(o);
}
bool given(PyObject* o) { return o != Py_None; }
int64_t whole(PyObject* o) {
  const long long v = PyLong_AsLongLong(o);
  if (v == -1 && PyErr_Occurred()) throw python_error();
  return v;
}
void count(Py_ssize_t n, Py_ssize_t want, const char* where) { TORCH_CHECK_TYPE(n == want, where, ": ", n, " arguments instead of ", want); }

int32_t code_of(at::ScalarType t) { return t == at::kFloat ? NVFP4_DT_F32 : NVFP4_DT_BF16; }
at::ScalarType type_of(int64_t code, const char* where) {
  if (code != NVFP4_DT_BF16 && code != NVFP4_DT_F32) raise_status(NVFP4_ERR_ENUM, where);
  return code == NVFP4_DT_F32 ? at::kFloat : at::kBFloat16;
}
bool either(at::ScalarType t) { return t == at::kBFloat16 || t == at::kFloat; }

// Leading dimension of a matrix argument of the given type (or of either, with no type) and shape (a negative size: any).
int64_t rows_of(const at::Tensor& t, const char* where, const char* name, c10::optional<at::ScalarType> type, int64_t rows, int64_t cols, c10::Device dev) {
  TORCH_CHECK(type ? t.scalar_type() == *type : either(t.scalar_type()), where, ": ", name, " is ", t.scalar_type(), ", not ",
              type ? c10::toString(*type) : "BFloat16 or Float");
  TORCH_CHECK(t.dim() == 2 && (rows < 0 || t.size(0) == rows) && (cols < 0 || t.size(1) == cols), where, ": ", name, " has shape ", t.sizes(),
              rows < 0 ? "" : c10::str(", not [", rows, ", ", cols, "]"));
  TORCH_CHECK(t.is_cuda() && t.device() == dev, where, ": ", name, " is on ", t.device(), ", not on ", dev.is_cuda() ? c10::str(dev) : "a CUDA device");
  TORCH_CHECK(t.stride(1) == 1 || t.size(1) <= 1, where, ": ", name, " has columns at a stride of ", t.stride(1));
  return t.size(0) > 1 ? t.stride(0) : up(t.size(1), 8);  // (a single row's stride says nothing)
}
void* vector(const at::Tensor& t, const char* where, const char* name, at::ScalarType type, int64_t n, c10::Device dev) {
  TORCH_CHECK(t.scalar_type() == type && t.dim() == 1 && t.size(0) == n && t.device() == dev && t.is_cuda() && (n <= 1 || t.stride(0) == 1), where, ": ", name, " is ",
              t.scalar_type(), " ", t.sizes(), " on ", t.device(), ", not a contiguous ", type, " vector of ", n, " on ", dev);
  return t.data_ptr();
}

void* bytes(const at::Tensor& t, const char* where, const char* name, int64_t at_least, c10::Device dev, at::ScalarType type = at::kByte) {
  TORCH_CHECK(t.scalar_type() == type, where, ": ", name, " is ", t.scalar_type(), ", not ", type);
  TORCH_CHECK(t.device() == dev && t.is_cuda() && t.is_contiguous(), where, ": ", name, " is on ", t.device(), ", not contiguous on ", dev);
  TORCH_CHECK((int64_t)t.nbytes() >= at_least, where, ": ", name, " has ", t.nbytes(), " bytes, too small for ", at_least);
  return t.data_ptr();
}

// A result that other threads still read or write something else through: refused as far as that is seen (not between interleaved views).
void apart(const at::Tensor& a, const at::Tensor& b, const char* where, const char* name, const char* other) {
  const at::MemOverlapStatus s = at::get_overlap_status(a, b);
  TORCH_CHECK(s != at::MemOverlapStatus::Full && s != at::MemOverlapStatus::Partial && (a.numel() == 0 || a.data_ptr() != b.data_ptr()), where, ": ", name, " and ", other,
              " share memory");
}

// A checkpoint's buffer: the codes, then the scales.
int64_t ckpt8_bytes(int64_t R, int64_t K) {
  const int64_t ld = nvfp4_ckpt8_ld(K);
  return R * (ld + ld / 32);
}
nvfp4_ckpt8 ckpt8(const at::Tensor& buf, const char* where, int64_t R, int64_t K, c10::Device dev) {
  TORCH_CHECK(R >= 0 && K >= 0 && R <= ((int64_t)1 << 38) && K <= ((int64_t)1 << 24), where, ": a checkpoint of shape [", R, ", ", K, "]");  // (their product fits)
  TORCH_CHECK(buf.is_cuda() && buf.device() == dev, where, ": a checkpoint on ", buf.device(), ", not on ", dev.is_cuda() ? c10::str(dev) : "a CUDA device");
  TORCH_CHECK(buf.scalar_type() == at::kByte && buf.is_contiguous() && buf.numel() == ckpt8_bytes(R, K), where,
              ": no checkpoint for a matrix [", R, ", ", K, "] on ", dev, ": ", buf.scalar_type(), " ", buf.sizes(), " on ", buf.device());
  uint8_t* p = static_cast<uint8_t*>(buf.data_ptr());
  return {p, p + R * nvfp4_ckpt8_ld(K), R, K};
}
at::Tensor new_ckpt8(int64_t R, int64_t K, const at::TensorOptions& opt) { return at::empty({ckpt8_bytes(R, K)}, opt.dtype(at::kByte)); }

// ---- results -------------------------------------------------------------------------------------------------------------------------
PyObject* wrap(const at::Tensor& t) {
  if (t.defined()) return THPVariable_Wrap(t);
  Py_RETURN_NONE;
}
template <typename... T>
PyObject* tuple_of(const T&... t) {
  PyObject* r = PyTuple_New(sizeof...(T));
  if (!r) throw python_error();
  Py_ssize_t i = 0;
  (PyTuple_SET_ITEM(r, i++, wrap(t)), ...);
  return r;
}
void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }
// The library call, without Python's lock: a launch waits where the device's queue is full.
template <typename F>
void enqueue(const char* where, F&& call) {
  nvfp4_status s;
  {
    pybind11::gil_scoped_release no_gil;
    s = call();
  }
  if (s != NVFP4_OK) raise_status(s, where);
}
// The tensors' device is the current one while a call lasts. (A device of another kind is refused by the checks.)
struct Guard {
  c10::cuda::OptionalCUDAGuard g;
  explicit Guard(c10::Device dev) {
    if (dev.is_cuda()) g.set_device(dev);
  }
};

// ---- the calls -----------------------------------------------------------------------------------------------------------------------
// gemv(X, codes, sf, gscale, R, K, gs_mode, sf_layout, dtype code, bias, outlier columns, kept columns, W_out, out, dev_status)
PyObject* gemv(PyObject*, Args a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const char* where = "nvfp4_gemv";
  count(n, 15, where);
  const at::Tensor& X = tensor(a[0], where, "X");
  const c10::Device dev = X.device();
  const int64_t ldx = rows_of(X, where, "X", at::kBFloat16, -1, -1, dev), M = X.size(0), D = X.size(1);
  const Guard guard(dev);
  nvfp4_operand W{};
  W.R = whole(a[4]);
  W.K = whole(a[5]);
  W.gs_mode = (int32_t)whole(a[6]);
  W.sf_layout = (int32_t)whole(a[7]);
  const at::ScalarType type = type_of(whole(a[8]), where);
  const bool sized = W.R > 0 && W.K > 0 && W.gs_mode >= 0 && W.gs_mode <= 2 && W.sf_layout >= 0 && W.sf_layout <= 1;  // (else the library refuses, or has nothing to do)
  W.codes = static_cast<uint8_t*>(bytes(tensor(a[1], where, "codes"), where, "codes", sized ? (int64_t)nvfp4_operand_codes_bytes(W.R, W.K) : 0, dev));
  W.sf = static_cast<uint8_t*>(bytes(tensor(a[2], where, "scales"), where, "scales", sized ? (int64_t)nvfp4_operand_sf_bytes(W.R, W.K, W.sf_layout) : 0, dev));
  W.gscale = static_cast<float*>(bytes(tensor(a[3], where, "global scales"), where, "global scales", sized ? 4 * (int64_t)nvfp4_operand_gscale_count(W.R, W.K, W.gs_mode) : 0, dev, at::kFloat));
  const void* bias = given(a[9]) ? vector(tensor(a[9], where, "bias"), where, "bias", at::kBFloat16, W.R, dev) : nullptr;
  int64_t n_out = 0;
  const int32_t *outl = nullptr, *keep = nullptr;
  const void* W_out = nullptr;
  if (given(a[10])) {
    const at::Tensor& o = tensor(a[10], where, "outlier columns");
    n_out = o.numel();
    if (n_out > 0) {
      outl = static_cast<const int32_t*>(vector(o, where, "outlier columns", at::kInt, n_out, dev));
      keep = static_cast<const int32_t*>(vector(tensor(a[11], where, "kept columns"), where, "kept columns", at::kInt, W.K, dev));
      const at::Tensor& w = tensor(a[12], where, "W_out");
      const int64_t Kh = nvfp4_outlier_pad(n_out);
      TORCH_CHECK(rows_of(w, where, "W_out", at::kBFloat16, W.R, Kh, dev) == Kh, where, ": W_out is not contiguous");
      W_out = w.data_ptr();
    }
  }
  int32_t* status = given(a[14]) ? static_cast<int32_t*>(bytes(tensor(a[14], where, "dev_status"), where, "dev_status", 4, dev, at::kInt)) : nullptr;
  TORCH_CHECK(W.R >= 0, where, ": ", W.R, " weight rows");
  at::Tensor Y = given(a[13]) ? tensor(a[13], where, "out") : matrix(M, W.R, X.options().dtype(type));
  const int64_t ldy = rows_of(Y, where, "out", type, M, W.R, dev);
  if (given(a[13])) apart(Y, X, where, "out", "X");
  const size_t need = nvfp4_gemv_workspace_bytes(M, D, n_out);
  const at::Tensor ws = need ? at::empty({(int64_t)need}, X.options().dtype(at::kByte)) : at::Tensor();
  enqueue(where, [&] { return nvfp4_gemv(X.data_ptr(), ldx, M, D, &W, keep, outl, n_out, W_out, bias, Y.data_ptr(), code_of(type), ldy, status, need ? ws.data_ptr() : nullptr, need,
                   current_stream()); });
  return wrap(Y);
  END_HANDLE_TH_ERRORS
}

// ckpt8_pack(X, buffer)
PyObject* ckpt8_pack(PyObject*, Args a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const char* where = "nvfp4_ckpt8_pack";
  count(n, 2, where);
  const at::Tensor& X = tensor(a[0], where, "X");
  const c10::Device dev = X.device();
  const int64_t ldx = rows_of(X, where, "X", c10::nullopt, -1, -1, dev), R = X.size(0), K = X.size(1);
  const Guard guard(dev);
  at::Tensor buf = given(a[1]) ? tensor(a[1], where, "the checkpoint") : new_ckpt8(R, K, X.options());
  const nvfp4_ckpt8 c = ckpt8(buf, where, R, K, dev);
  enqueue(where, [&] { return nvfp4_ckpt8_pack(X.data_ptr(), code_of(X.scalar_type()), ldx, R, K, &c, current_stream()); });
  return wrap(buf);
  END_HANDLE_TH_ERRORS
}

// ckpt8_unpack(buffer, R, K, dtype code, out)
PyObject* ckpt8_unpack(PyObject*, Args a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const char* where = "nvfp4_ckpt8_unpack";
  count(n, 5, where);
  const at::Tensor& buf = tensor(a[0], where, "the checkpoint");
  const c10::Device dev = buf.device();
  const int64_t R = whole(a[1]), K = whole(a[2]);
  const nvfp4_ckpt8 c = ckpt8(buf, where, R, K, dev);
  const at::ScalarType type = type_of(whole(a[3]), where);
  const Guard guard(dev);
  at::Tensor X = given(a[4]) ? tensor(a[4], where, "out") : matrix(R, K, buf.options().dtype(type));
  const int64_t ld = rows_of(X, where, "out", type, R, K, dev);
  enqueue(where, [&] { return nvfp4_ckpt8_unpack(&c, X.data_ptr(), code_of(type), ld, current_stream()); });
  return wrap(X);
  END_HANDLE_TH_ERRORS
}

void check_save(int64_t save, const char* where) {
  if (save < kNothing || save > kCkpt8) raise_status(NVFP4_ERR_ENUM, where);
}

// swiglu_fwd(G, U, save, out) -> (H, checkpoint of G, of U)
PyObject* swiglu_fwd(PyObject*, Args a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const char* where = "nvfp4_swiglu_fwd";
  count(n, 4, where);
  const at::Tensor &G = tensor(a[0], where, "G"), &U = tensor(a[1], where, "U");
  const c10::Device dev = G.device();
  const int64_t ldg = rows_of(G, where, "G", at::kBFloat16, -1, -1, dev), T = G.size(0), D = G.size(1);
  const int64_t ldu = rows_of(U, where, "U", at::kBFloat16, T, D, dev), save = whole(a[2]);
  check_save(save, where);
  const Guard guard(dev);
  at::Tensor H = given(a[3]) ? tensor(a[3], where, "out") : matrix(T, D, G.options()), g8, u8;
  const int64_t ldh = rows_of(H, where, "out", at::kBFloat16, T, D, dev);
  nvfp4_ckpt8 cg, cu;
  if (save == kCkpt8) {
    cg = ckpt8(g8 = new_ckpt8(T, D, G.options()), where, T, D, dev);
    cu = ckpt8(u8 = new_ckpt8(T, D, G.options()), where, T, D, dev);
  }
  enqueue(where, [&] { return nvfp4_swiglu_fwd(G.data_ptr(), ldg, U.data_ptr(), ldu, T, D, H.data_ptr(), ldh, save == kCkpt8 ? &cg : nullptr, save == kCkpt8 ? &cu : nullptr, current_stream()); });
  return tuple_of(H, g8, u8);
  END_HANDLE_TH_ERRORS
}

// swiglu_bwd(dH, T, D, G, U, checkpoint of G, of U, dG, dU) -> (dG, dU)
PyObject* swiglu_bwd(PyObject*, Args a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const char* where = "nvfp4_swiglu_bwd";
  count(n, 9, where);
  const at::Tensor& dH = tensor(a[0], where, "dH");
  const c10::Device dev = dH.device();
  const int64_t T = whole(a[1]), D = whole(a[2]), lddh = rows_of(dH, where, "dH", at::kBFloat16, T, D, dev);
  const Guard guard(dev);
  const void *G = nullptr, *U = nullptr;
  int64_t ldg = 0, ldu = 0;
  nvfp4_ckpt8 cg, cu;
  const bool packed = given(a[5]);
  if (packed) {
    cg = ckpt8(tensor(a[5], where, "the checkpoint of G"), where, T, D, dev);
    cu = ckpt8(tensor(a[6], where, "the checkpoint of U"), where, T, D, dev);
  } else {
    const at::Tensor &g = tensor(a[3], where, "G"), &u = tensor(a[4], where, "U");
    ldg = rows_of(g, where, "G", at::kBFloat16, T, D, dev);
    ldu = rows_of(u, where, "U", at::kBFloat16, T, D, dev);
    G = g.data_ptr();
    U = u.data_ptr();
  }
  at::Tensor dG = given(a[7]) ? tensor(a[7], where, "dG") : matrix(T, D, dH.options()), dU = given(a[8]) ? tensor(a[8], where, "dU") : matrix(T, D, dH.options());
  const int64_t lddg = rows_of(dG, where, "dG", at::kBFloat16, T, D, dev), lddu = rows_of(dU, where, "dU", at::kBFloat16, T, D, dev);
  if (given(a[7]) || given(a[8])) apart(dG, dU, where, "dG", "dU");
  enqueue(where, [&] { return nvfp4_swiglu_bwd(dH.data_ptr(), lddh, G, ldg, U, ldu, packed ? &cg : nullptr, packed ? &cu : nullptr, T, D, dG.data_ptr(), lddg, dU.data_ptr(), lddu, current_stream()); });
  return tuple_of(dG, dU);
  END_HANDLE_TH_ERRORS
}

// layernorm_fwd(X, gamma, beta, eps, save, out) -> (Y, stats, checkpoint of X)
PyObject* layernorm_fwd(PyObject*, Args a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const char* where = "nvfp4_layernorm_fwd";
  count(n, 6, where);
  const at::Tensor &X = tensor(a[0], where, "X"), &gamma = tensor(a[1], where, "gamma");
  const c10::Device dev = X.device();
  const int64_t ldx = rows_of(X, where, "X", c10::nullopt, -1, -1, dev), T = X.size(0), D = X.size(1), save = whole(a[4]);
  const at::ScalarType type = gamma.scalar_type();
  TORCH_CHECK(either(type), where, ": gamma is ", type, ", not BFloat16 or Float");
  const void* pg = vector(gamma, where, "gamma", type, D, dev);
  const void* pb = given(a[2]) ? vector(tensor(a[2], where, "beta"), where, "beta", type, D, dev) : nullptr;
  const double eps = PyFloat_AsDouble(a[3]);
  if (eps == -1.0 && PyErr_Occurred()) throw python_error();
  check_save(save, where);
  const Guard guard(dev);
  at::Tensor Y = given(a[5]) ? tensor(a[5], where, "out") : matrix(T, D, X.options().dtype(at::kBFloat16)), stats, x8;
  const int64_t ldy = rows_of(Y, where, "out", at::kBFloat16, T, D, dev);
  if (save != kNothing) stats = at::empty({T, 2}, X.options().dtype(at::kFloat));
  nvfp4_ckpt8 c;
  if (save == kCkpt8) c = ckpt8(x8 = new_ckpt8(T, D, X.options()), where, T, D, dev);
  enqueue(where, [&] { return nvfp4_layernorm_fwd(X.data_ptr(), code_of(X.scalar_type()), ldx, T, D, pg, pb, code_of(type), (float)eps, Y.data_ptr(), ldy,
                            stats.defined() ? static_cast<float*>(stats.data_ptr()) : nullptr, save == kCkpt8 ? &c : nullptr, current_stream()); });
  return tuple_of(Y, stats, x8);
  END_HANDLE_TH_ERRORS
}

// layernorm_bwd(dY, T, D, dtype code of X, X, checkpoint, stats, gamma, with beta, dX, dtype code of the parameters' gradients, workspace)
// -> (dX, dgamma, dbeta)
PyObject* layernorm_bwd(PyObject*, Args a, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  const char* where = "nvfp4_layernorm_bwd";
  count(n, 12, where);
  const at::Tensor &dY = tensor(a[0], where, "dY"), &stats = tensor(a[6], where, "stats"), &gamma = tensor(a[7], where, "gamma");
  const c10::Device dev = dY.device();
  const int64_t T = whole(a[1]), D = whole(a[2]), lddy = rows_of(dY, where, "dY", at::kBFloat16, T, D, dev);
  const at::ScalarType x_type = type_of(whole(a[3]), where), p_type = gamma.scalar_type();
  TORCH_CHECK(either(p_type), where, ": gamma is ", p_type, ", not BFloat16 or Float");
  const void* pg = vector(gamma, where, "gamma", p_type, D, dev);
  const Guard guard(dev);
  const bool packed = given(a[5]);
  nvfp4_ckpt8 c;
  const void* X = nullptr;
  int64_t ldx = 0;
  if (packed) {
    c = ckpt8(tensor(a[5], where, "the checkpoint"), where, T, D, dev);
  } else {
    const at::Tensor& x = tensor(a[4], where, "X");
    ldx = rows_of(x, where, "X", x_type, T, D, dev);
    X = x.data_ptr();
  }
  rows_of(stats, where, "stats", at::kFloat, T, 2, dev);
  TORCH_CHECK(stats.is_contiguous(), where, ": stats is not contiguous");
  at::Tensor dX = given(a[9]) ? tensor(a[9], where, "dX") : matrix(T, D, dY.options().dtype(x_type));
  const int64_t lddx = rows_of(dX, where, "dX", x_type, T, D, dev);
  const at::ScalarType d_type = given(a[10]) ? type_of(whole(a[10]), where) : p_type;
  const bool beta = PyObject_IsTrue(a[8]) == 1;
  at::Tensor dgamma = at::empty({D}, dY.options().dtype(d_type)), dbeta = beta ? at::empty({D}, dY.options().dtype(d_type)) : at::Tensor();
  const int64_t need = (int64_t)nvfp4_layernorm_bwd_workspace_bytes(T, D);
  const at::Tensor ws = given(a[11]) ? tensor(a[11], where, "the workspace") : at::empty({need}, dY.options().dtype(at::kByte));
  void* pw = bytes(ws, where, "the workspace", 0, dev);
  enqueue(where, [&] { return nvfp4_layernorm_bwd(dY.data_ptr(), lddy, X, code_of(x_type), ldx, packed ? &c : nullptr, T, D, pg, code_of(p_type), static_cast<const float*>(stats.data_ptr()),
                            dX.data_ptr(), lddx, dgamma.data_ptr(), beta ? dbeta.data_ptr() : nullptr, code_of(d_type), pw, ws.nbytes(), current_stream()); });
  return tuple_of(dX, dgamma, dbeta);
  END_HANDLE_TH_ERRORS
}

}  // namespace

PyMethodDef nvfp4_torch::block_methods[] = {
    {"gemv", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(gemv)), METH_FASTCALL, nullptr},
    {"ckpt8_pack", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(ckpt8_pack)), METH_FASTCALL, nullptr},
    {"ckpt8_unpack", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(ckpt8_unpack)), METH_FASTCALL, nullptr},
    {"swiglu_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(swiglu_fwd)), METH_FASTCALL, nullptr},
    {"swiglu_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(swiglu_bwd)), METH_FASTCALL, nullptr},
    {"layernorm_fwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(layernorm_fwd)), METH_FASTCALL, nullptr},
    {"layernorm_bwd", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(layernorm_bwd)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
