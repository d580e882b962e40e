// The calls on 8-bit matrices for torch tensors: checks of arguments, new tensors for the results, the current stream.  A
// Python extension, because these calls often take less time on the GPU than their arguments take in Python (silu(gate) * up
// of one token: 6.5 us a call through ctypes, 4.8 so, of which the launch is 3).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/hip/EmptyTensor.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <limits>
#include <string>

#include "../../include/xorenc.h"

namespace {

using at::ScalarType;
using at::Tensor;
using at::TensorBase;

constexpr int64_t kBlock = XORENC_FP8_BLOCK, kMostInt = std::numeric_limits<int32_t>::max();

int64_t round_up(int64_t n, int64_t d) { return (n + d - 1) / d * d; }
int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }

struct Refused {  // becomes a ValueError
  std::string why;
};
struct Raised {};  // a Python error is set

// The current GPU and its stream.
struct Place {
  c10::DeviceIndex gpu = c10::hip::current_device();
  void *stream() const { return c10::hip::getCurrentHIPStream(gpu).stream(); }
  bool has(const TensorBase &t) const { return t.is_cuda() && t.get_device() == gpu; }
  // Each with memory of its own: results are saved, freed and handed to other streams one by one.  (Several in one allocation would take
  // 0.4 us less each, but torch saves no two types of one storage.)
  TensorBase fresh(at::IntArrayRef sizes, at::IntArrayRef strides, ScalarType type) const {
    return at::detail::empty_strided_cuda(sizes, strides, type, c10::Device(c10::kCUDA, gpu));
  }
};

const Tensor &tensor(PyObject *o, const char *what) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s must be a tensor", what);
    throw Raised();
  }
  return THPVariable_Unpack(o);
}

int32_t int_of(int64_t n, const char *what) {
  if (n > kMostInt || n < -kMostInt) throw Refused{std::string(what) + " is beyond 32 bits"};
  return (int32_t)n;
}
int32_t int_of(PyObject *o, const char *what) {
  int over = 0;
  const long long n = PyLong_AsLongLongAndOverflow(o, &over);
  if (n == -1 && !over && PyErr_Occurred()) throw Raised();
  return int_of(over ? (int64_t)kMostInt + 1 : (int64_t)n, what);
}

bool is_x_type(ScalarType t) { return t == ScalarType::BFloat16 || t == ScalarType::Float; }
int32_t x_type(const TensorBase &t, const char *what) {
  if (!is_x_type(t.scalar_type())) throw Refused{std::string(what) + " must be float32 or bfloat16"};
  return t.scalar_type() == ScalarType::BFloat16 ? XORENC_X_BF16 : XORENC_X_F32;
}

// Checks a row-major matrix (or stack of matrices) on the current GPU; its leading dimension.
int64_t rows_of(const TensorBase &t, int64_t dims, const char *what, const Place &here) {
  if (t.dim() != dims) throw Refused{std::string(what) + " must have " + std::to_string(dims) + " dimensions"};
  if (!here.has(t) || t.layout() != at::kStrided) throw Refused{std::string(what) + " is not on the current GPU"};
  const int64_t cols = t.size(dims - 1);
  if (cols == 0) throw Refused{std::string(what) + " has no columns"};
  int_of(cols, what);
  if (t.stride(dims - 1) != 1 && cols != 1) throw Refused{std::string("the columns of ") + what + " must be contiguous"};
  return t.size(dims - 2) > 1 ? t.stride(dims - 2) : round_up(cols, 16);
}

int64_t values_of(const TensorBase &t, int64_t dims, const char *what, const Place &here) {
  if (t.scalar_type() != ScalarType::Float8_e4m3fn) throw Refused{std::string(what) + " must be float8_e4m3fn"};
  return rows_of(t, dims, what, here);
}

const float *scales_of(const TensorBase &t, at::IntArrayRef shape, const char *what, const Place &here) {
  if (t.scalar_type() != ScalarType::Float || !here.has(t) || t.layout() != at::kStrided || t.sizes() != shape) {
    std::string s;
    for (int64_t n : shape) s += (s.empty() ? "" : ", ") + std::to_string(n);
    throw Refused{std::string(what) + " must be float32 of shape (" + s + ") on the current GPU"};
  }
  return static_cast<const float *>(t.data_ptr());
}

const uint8_t *bytes(const TensorBase &t) { return static_cast<const uint8_t *>(t.data_ptr()); }

// A new 8-bit matrix of activations: rows on 16-byte boundaries, scales block column by block column.
struct NewRows {
  int64_t ld, rows;
  TensorBase Q, S;
  NewRows(int64_t rows_, int64_t cols, const Place &here)
      : ld(round_up(cols, 16)), rows(rows_), Q(here.fresh({rows, cols}, {ld, 1}, ScalarType::Float8_e4m3fn)),
        S(here.fresh({rows, blocks_of(cols)}, {1, step()}, ScalarType::Float)) {}
  int64_t step() const { return rows ? rows : 1; }
  uint8_t *q() const { return static_cast<uint8_t *>(Q.data_ptr()); }
  float *s() const { return static_cast<float *>(S.data_ptr()); }
};

template <class F>
void call(const char *entry, F f) {
  int32_t rc;
  Py_BEGIN_ALLOW_THREADS
  rc = f();
  Py_END_ALLOW_THREADS
  if (rc == XORENC_OK) return;
  PyObject *const module = PyImport_ImportModule("paper_1905_10138_amd.binding");
  PyObject *const type = module ? PyObject_GetAttrString(module, "XorencError") : nullptr;
  PyObject *const error = type ? PyObject_CallFunction(type, "is", (int)rc, entry) : nullptr;
  if (error) PyErr_SetObject(type, error);
  Py_XDECREF(error);
  Py_XDECREF(type);
  Py_XDECREF(module);
  throw Raised();
}

PyObject *result(std::initializer_list<TensorBase> tensors) {  // None in the place of an undefined one
  PyObject *const out = PyTuple_New((Py_ssize_t)tensors.size());
  if (!out) throw Raised();
  Py_ssize_t i = 0;
  for (const TensorBase &t : tensors) {
    PyObject *o = Py_None;
    if (t.defined())
      o = THPVariable_Wrap(t);
    else
      Py_INCREF(o);
    if (!o) {
      Py_DECREF(out);
      throw Raised();
    }
    PyTuple_SET_ITEM(out, i++, o);
  }
  return out;
}

// (X, block_rows) -> (Q, S)
PyObject *quant(PyObject *const *args) {
  const Place here;
  const Tensor &X = tensor(args[0], "X");
  const int32_t block_rows = int_of(args[1], "block_rows");
  const int64_t dims = X.dim();
  if (dims != 2 && dims != 3) throw Refused{"X must be a matrix or a stack of matrices"};
  const int64_t ldx = rows_of(X, dims, "X", here), rows = X.size(dims - 2), cols = X.size(dims - 1), blocks = blocks_of(cols);
  const int32_t type = x_type(X, "X");
  if (dims == 2 && block_rows == 1) {
    const NewRows out(rows, cols, here);
    call("xorenc_quant_fp8", [&] {
      return xorenc_quant_fp8(X.data_ptr(), type, ldx, 0, 1, rows, (int32_t)cols, 1, out.q(), out.ld, 0, out.s(), 1, out.step(), 0, here.stream());
    });
    return result({out.Q, out.S});
  }
  const int64_t n = dims == 2 ? 1 : X.size(0), ldq = round_up(cols, 16), s_rows = block_rows == 1 ? rows : blocks_of(rows);
  TensorBase Q, S;
  if (dims == 2) {
    Q = here.fresh({rows, cols}, {ldq, 1}, ScalarType::Float8_e4m3fn);
    S = here.fresh({s_rows, blocks}, {blocks, 1}, ScalarType::Float);
  } else {
    Q = here.fresh({n, rows, cols}, {rows * ldq, ldq, 1}, ScalarType::Float8_e4m3fn);
    S = here.fresh({n, s_rows, blocks}, {s_rows * blocks, blocks, 1}, ScalarType::Float);
  }
  const int32_t matrices = int_of(n, "the number of matrices");
  call("xorenc_quant_fp8", [&] {
    return xorenc_quant_fp8(X.data_ptr(), type, ldx, dims == 2 ? 0 : X.stride(0), matrices, rows, (int32_t)cols, block_rows,
                            static_cast<uint8_t *>(Q.data_ptr()), ldq, dims == 2 ? 0 : rows * ldq, static_cast<float *>(S.data_ptr()), blocks, 1,
                            dims == 2 ? 0 : s_rows * blocks, here.stream());
  });
  return result({Q, S});
}

// (X, weight, residual, eps, total, normed) -> (Q, S, t, y)
PyObject *norm(PyObject *const *args) {
  const Place here;
  const Tensor &X = tensor(args[0], "X"), &weight = tensor(args[1], "weight");
  const int64_t ldx = rows_of(X, 2, "X", here), rows = X.size(0), cols = X.size(1);
  const int32_t type = x_type(X, "X"), w_type = x_type(weight, "weight");
  if (weight.dim() != 1 || weight.size(0) != cols || (cols > 1 && weight.stride(0) != 1) || !here.has(weight))
    throw Refused{"weight must be (features,), contiguous, on the current GPU"};
  const double eps = PyFloat_AsDouble(args[3]);
  if (eps == -1.0 && PyErr_Occurred()) throw Raised();
  auto like_x = [&](const Tensor &t, const char *what) {
    const int64_t ld = rows_of(t, 2, what, here);
    if (t.sizes() != X.sizes() || t.scalar_type() != X.scalar_type()) throw Refused{std::string(what) + " must have the shape and type of X"};
    return ld;
  };
  const void *residual = nullptr;
  TensorBase total, y;
  int64_t ldr = 0, ldt = cols, y_row = cols, y_col = 1;
  if (args[2] != Py_None) {
    const Tensor &r = tensor(args[2], "residual");
    ldr = like_x(r, "residual");
    residual = r.data_ptr();
  }
  if (args[4] != Py_None) {
    const Tensor &t = tensor(args[4], "total");
    ldt = like_x(t, "total");
    total = t;
  }
  if (args[5] != Py_True && args[5] != Py_False) {
    const Tensor &t = tensor(args[5], "normed");
    if (t.sizes() != X.sizes() || t.scalar_type() != X.scalar_type() || !here.has(t) || t.layout() != at::kStrided)
      throw Refused{"normed must have the shape and type of X, on the current GPU"};
    y = t;
    y_row = t.stride(0);
    y_col = cols == 1 ? 1 : t.stride(1);
  }
  const NewRows out(rows, cols, here);
  if (residual && !total.defined()) total = here.fresh({rows, cols}, {cols, 1}, X.scalar_type());
  if (args[5] == Py_True) y = here.fresh({rows, cols}, {cols, 1}, X.scalar_type());
  call("xorenc_add_rmsnorm_fp8", [&] {
    return xorenc_add_rmsnorm_fp8(X.data_ptr(), type, ldx, residual, ldr, weight.data_ptr(), w_type, rows, (int32_t)cols, (float)eps,
                                  total.defined() ? total.data_ptr() : nullptr, ldt, y.defined() ? y.data_ptr() : nullptr, y_row, y_col, out.q(),
                                  out.ld, out.s(), 1, out.step(), here.stream());
  });
  return result({out.Q, out.S, total, y});
}

// (X) -> (Q, S)
PyObject *gate(PyObject *const *args) {
  const Place here;
  const Tensor &X = tensor(args[0], "X");
  const int64_t ldx = rows_of(X, 2, "X", here), rows = X.size(0), cols = X.size(1) / 2;
  const int32_t type = x_type(X, "X");
  if (X.size(1) % 2) throw Refused{"X must have as many gates as ups"};
  const NewRows out(rows, cols, here);
  const uint8_t *const gates = bytes(X);
  call("xorenc_silu_mul_fp8", [&] {
    return xorenc_silu_mul_fp8(gates, gates + cols * (type == XORENC_X_BF16 ? 2 : 4), type, ldx, rows, (int32_t)cols, out.q(), out.ld, out.s(), 1,
                               out.step(), here.stream());
  });
  return result({out.Q, out.S});
}

// (A, SA, W, SW, out_dtype, Y) -> Y
PyObject *matmul(PyObject *const *args) {
  const Place here;
  const Tensor &A = tensor(args[0], "A"), &SA = tensor(args[1], "SA"), &W = tensor(args[2], "W"), &SW = tensor(args[3], "SW");
  const int64_t lda = values_of(A, 2, "A", here), ldw = values_of(W, 2, "W", here), M = A.size(0), N = W.size(0), K = A.size(1), blocks = blocks_of(K);
  if (W.size(1) != K) throw Refused{"A and W must have as many columns"};
  const float *const sa = scales_of(SA, {M, blocks}, "SA", here), *const sw = scales_of(SW, {blocks_of(N), blocks}, "SW", here);
  if (blocks > 1 && SW.stride(1) != 1) throw Refused{"the columns of SW must be contiguous"};
  if (args[4] != Py_None && !THPDtype_Check(args[4])) throw Refused{"out_dtype must be a torch type"};
  const ScalarType asked = args[4] == Py_None ? ScalarType::Undefined : reinterpret_cast<THPDtype *>(args[4])->scalar_type;
  TensorBase Y;
  int64_t ldy = N;
  if (args[5] == Py_None) {
    if (asked != ScalarType::Undefined && !is_x_type(asked)) throw Refused{"Y must be float32 or bfloat16"};
    Y = here.fresh({M, N}, {N, 1}, asked == ScalarType::Undefined ? ScalarType::BFloat16 : asked);
  } else {
    Y = tensor(args[5], "Y");
    ldy = rows_of(Y, 2, "Y", here);
    if (Y.size(0) != M || Y.size(1) != N || (asked != ScalarType::Undefined && asked != Y.scalar_type()))
      throw Refused{"Y must be (tokens, outputs) of the type asked for"};
  }
  const int32_t type = x_type(Y, "Y"), m = int_of(M, "the number of tokens"), n = int_of(N, "the number of outputs");
  call("xorenc_matmul_fp8", [&] {
    return xorenc_matmul_fp8(bytes(A), lda, sa, SA.stride(0), blocks > 1 ? SA.stride(1) : 0, bytes(W), ldw, sw, N > kBlock ? SW.stride(0) : blocks, m,
                             n, (int32_t)K, Y.data_ptr(), type, ldy, here.stream());
  });
  if (args[5] == Py_None) return THPVariable_Wrap(Y);
  Py_INCREF(args[5]);
  return args[5];
}

// (X, router, W13, S13, W2, S2, picks, renormalise, Y) -> Y
PyObject *moe(PyObject *const *args) {
  const Place here;
  const Tensor &X = tensor(args[0], "X"), &router = tensor(args[1], "router"), &W13 = tensor(args[2], "W13"), &S13 = tensor(args[3], "S13"),
               &W2 = tensor(args[4], "W2"), &S2 = tensor(args[5], "S2");
  const int32_t type = x_type(X, "X"), picks = int_of(args[6], "picks");
  const int renormalise = PyObject_IsTrue(args[7]);
  if (renormalise < 0) throw Raised();
  xorenc_moe L = {};
  L.struct_size = sizeof(L);
  const int64_t ldx = rows_of(X, 2, "X", here);
  L.ld_router = rows_of(router, 2, "router", here);
  L.ld_w13 = values_of(W13, 3, "W13", here);
  L.ld_w2 = values_of(W2, 3, "W2", here);
  const int64_t T = X.size(0), H = X.size(1), E = W2.size(0), I = W2.size(2), hb = blocks_of(H), ib = blocks_of(I);
  if (router.scalar_type() != X.scalar_type() || router.size(0) != E || router.size(1) != H)
    throw Refused{"router must be (experts, hidden) of the type of X"};
  if (W2.size(1) != H || W13.size(0) != E || W13.size(1) != 2 * I || W13.size(2) != H)
    throw Refused{"W13 must be (experts, 2 inner, hidden) and W2 (experts, hidden, inner)"};
  L.S13 = scales_of(S13, {E, blocks_of(2 * I), hb}, "S13", here);
  L.S2 = scales_of(S2, {E, hb, ib}, "S2", here);
  if ((hb > 1 && S13.stride(2) != 1) || (ib > 1 && S2.stride(2) != 1)) throw Refused{"the columns of S13 and S2 must be contiguous"};
  L.experts = int_of(E, "the number of experts");
  L.hidden = (int32_t)H;
  L.inner = (int32_t)I;
  L.router = router.data_ptr();
  L.W13 = bytes(W13);
  L.W2 = bytes(W2);
  L.w13_stride = E > 1 ? W13.stride(0) : 0;
  L.w2_stride = E > 1 ? W2.stride(0) : 0;
  L.ld_s13 = 2 * I > kBlock ? S13.stride(1) : hb;
  L.s13_stride = S13.stride(0);
  L.ld_s2 = H > kBlock ? S2.stride(1) : ib;
  L.s2_stride = S2.stride(0);
  TensorBase Y;
  int64_t ldy = H, need = 0;
  if (args[8] == Py_None) {
    Y = here.fresh({T, H}, {H, 1}, X.scalar_type());
  } else {
    Y = tensor(args[8], "Y");
    ldy = rows_of(Y, 2, "Y", here);
    if (Y.sizes() != X.sizes() || Y.scalar_type() != X.scalar_type()) throw Refused{"Y must have the shape and type of X"};
  }
  const int32_t tokens = int_of(T, "the number of tokens");
  call("xorenc_moe_workspace", [&] { return xorenc_moe_workspace(tokens, L.hidden, L.inner, L.experts, picks, type, &need); });
  const TensorBase workspace = here.fresh({need / 4 + 1}, {1}, ScalarType::Float);
  call("xorenc_moe_fp8", [&] {
    return xorenc_moe_fp8(&L, X.data_ptr(), type, ldx, tokens, picks, renormalise, Y.data_ptr(), ldy, workspace.data_ptr(), need, here.stream());
  });
  if (args[8] == Py_None) return THPVariable_Wrap(Y);
  Py_INCREF(args[8]);
  return args[8];
}

#include "xorenc_torch_experts.h"

template <PyObject *(*F)(PyObject *const *), int N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
  HANDLE_TH_ERRORS
  if (n != N) {
    PyErr_Format(PyExc_TypeError, "%d arguments expected", N);
    return nullptr;
  }
  try {
    return F(args);
  } catch (const Refused &r) {
    PyErr_SetString(PyExc_ValueError, r.why.c_str());
  } catch (const Raised &) {
  }
  return nullptr;
  END_HANDLE_TH_ERRORS
}

template <PyObject *(*F)(PyObject *const *), int N>
PyMethodDef method(const char *name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(&entry<F, N>)), METH_FASTCALL, nullptr};
}

PyMethodDef methods[] = {method<quant, 2>("quant"),   method<norm, 6>("norm"), method<gate, 1>("gate"),
                         method<matmul, 6>("matmul"), method<moe, 9>("moe"),   method<pick, 3>("pick"),
                         method<sort, 2>("sort"),     method<gather, 5>("gather"), method<combine, 6>("combine"),
                         method<combine_grad, 6>("combine_grad"), method<linear, 9>("linear"), method<experts, 10>("experts"),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_fp8", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__fp8() { return PyModule_Create(&module); }
