// The entry points of bnn.h that a program calls once per layer, taken straight from torch tensors.
//
// A layer on a few thousand values is a launch of 2.4 us, and checking and converting its tensors through Python's attribute
// calls (about 50 ns each, 20 to 30 of them) was 1.6 to 2 us beside it.  Here it is 0.2: one call from the binding with the
// tensors themselves.  Each function returns the status of the call (the
// two of gradients their tensors, where the call went through), or None for anything but the plain case (tensors of
// the binding's types on the GPU, given outputs, integers, pairs of integers); the binding's own code then takes the call,
// and raises what it raises.  bind(): addresses of the library's functions, in the order of `names`.  built_for: the torch and the
// Python of whose objects this file's accessors know the layout; the binding uses it with no other.
#include <torch/csrc/autograd/python_variable.h>

#include <algorithm>
#include <cstring>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <c10/hip/HIPStream.h>

#include "bnn.h"

namespace {

struct Library {
  decltype(&bnn_xnor_gemm) gemm;
  decltype(&bnn_xnor_gemm_epilogue) epilogue;
  decltype(&bnn_encode) encode;
  decltype(&bnn_conv2d) conv2d;
  decltype(&bnn_conv2d_packed) conv2d_packed;
  decltype(&bnn_im2col_packed) im2col;
  decltype(&bnn_conv2d_f32_sign) f32_sign;
  decltype(&bnn_conv2d_f32) f32;
  decltype(&bnn_maxpool2x2) maxpool;
  decltype(&bnn_fc_f32) fc;
  decltype(&bnn_quant_rows_i8) quant;
  decltype(&bnn_linear_i8) linear;
  decltype(&bnn_norm_gate) norm;
  decltype(&bnn_norm_gate_backward) norm_backward;
  decltype(&bnn_gated_ff) gated;
  decltype(&bnn_gated_ff_i8) gated_i8;
  decltype(&bnn_gated_ff_backward) gated_backward;
  decltype(&bnn_norm_gate_backward_workspace_bytes) norm_workspace;
  decltype(&bnn_gated_ff_backward_workspace_bytes) gated_workspace;
  decltype(&bnn_quant_blocks_f8) quant_blocks;
  decltype(&bnn_quant_columns_f8) quant_columns;
  decltype(&bnn_linear_f8) linear_f8;
  decltype(&bnn_expert_linear_f8) expert_linear;
  decltype(&bnn_expert_linear_f8_dw) expert_linear_dw;
  decltype(&bnn_expert_rows) expert_rows;
  decltype(&bnn_expert_sort_workspace_bytes) sort_workspace;
  decltype(&bnn_expert_sort) sort;
  decltype(&bnn_expert_gather) gather;
  decltype(&bnn_expert_combine) combine;
  decltype(&bnn_expert_combine_backward) combine_backward;
  decltype(&bnn_gated_act) gated_act;
  decltype(&bnn_gated_act_f8) gated_act_f8;
  decltype(&bnn_gated_act_backward) gated_act_backward;
};
constexpr const char *names[] = {"bnn_xnor_gemm", "bnn_xnor_gemm_epilogue", "bnn_encode", "bnn_conv2d", "bnn_conv2d_packed",
                                 "bnn_im2col_packed", "bnn_conv2d_f32_sign", "bnn_conv2d_f32", "bnn_maxpool2x2", "bnn_fc_f32", "bnn_quant_rows_i8", "bnn_linear_i8",
                                 "bnn_norm_gate", "bnn_norm_gate_backward", "bnn_gated_ff", "bnn_gated_ff_i8", "bnn_gated_ff_backward",
                                 "bnn_norm_gate_backward_workspace_bytes", "bnn_gated_ff_backward_workspace_bytes",
                                 "bnn_quant_blocks_f8", "bnn_quant_columns_f8", "bnn_linear_f8", "bnn_expert_linear_f8", "bnn_expert_linear_f8_dw",
                                 "bnn_expert_rows", "bnn_expert_sort_workspace_bytes", "bnn_expert_sort", "bnn_expert_gather", "bnn_expert_combine",
                                 "bnn_expert_combine_backward", "bnn_gated_act", "bnn_gated_act_f8", "bnn_gated_act_backward"};
Library lib = {};

struct Other {};  // not the plain case

// The arguments of a call, taken in order.
class Args {
 public:
  Args(PyObject *const *a, Py_ssize_t n, Py_ssize_t want) : a_(a) {
    // subclasses and modes may give a tensor's attributes another meaning
    if (n != want || !lib.gemm || at::impl::torch_function_mode_enabled()) throw Other();
  }
  const at::Tensor &tensor() {
    PyObject *o = *a_++;
    if (!THPVariable_CheckExact(o)) throw Other();
    return THPVariable_Unpack(o);
  }
  const at::Tensor &tensor(at::ScalarType type) {
    const at::Tensor &t = tensor();
    if (!t.is_cuda() || t.scalar_type() != type) throw Other();
    return t;
  }
  const at::Tensor &tensor(at::ScalarType type, int64_t dim) {
    const at::Tensor &t = tensor(type);
    if (t.dim() != dim) throw Other();
    return t;
  }
  void *pointer() {  // of any tensor, or None
    if (*a_ == Py_None) {
      ++a_;
      return nullptr;
    }
    return tensor().data_ptr();
  }
  const at::Tensor *tensor_or_none() {
    if (*a_ == Py_None) {
      ++a_;
      return nullptr;
    }
    return &tensor();
  }
  float real() {
    PyObject *o = *a_++;
    if (!PyFloat_CheckExact(o)) throw Other();
    return (float)PyFloat_AS_DOUBLE(o);
  }
  int64_t integer() { return integer(*a_++); }
  int small() { return as_int(integer()); }
  void pair(int (&v)[2]) {
    PyObject *o = *a_++;
    if (!PyTuple_CheckExact(o) || PyTuple_GET_SIZE(o) != 2) throw Other();
    for (int i = 0; i < 2; ++i) v[i] = as_int(integer(PyTuple_GET_ITEM(o, i)));
  }

 private:
  static int64_t integer(PyObject *o) {
    if (!PyLong_CheckExact(o)) throw Other();
    int overflow;
    const long long v = PyLong_AsLongLongAndOverflow(o, &overflow);
    if (overflow) throw Other();
    return v;
  }
  static int as_int(int64_t v) {
    if (v != (int)v) throw Other();
    return (int)v;
  }
  PyObject *const *a_;
};

int size(const at::Tensor &t, int64_t d) {
  const int64_t n = t.size(d);
  if (n != (int)n) throw Other();
  return (int)n;
}

float *f32(void *p) { return static_cast<float *>(p); }
int32_t *i32(void *p) { return static_cast<int32_t *>(p); }
uint64_t *u64(const at::Tensor &t) { return static_cast<uint64_t *>(t.data_ptr()); }
// rows of a matrix: one row may have any stride
int64_t row_stride(const at::Tensor &t, int64_t least) { return t.size(0) > 1 ? t.stride(0) : least; }

// Other threads run meanwhile; held again also where the call throws.
struct Released {
  PyThreadState *state = PyEval_SaveThread();
  ~Released() { PyEval_RestoreThread(state); }
};

template <class Call>
PyObject *launch(const Call &call) {
  void *const stream = c10::hip::getCurrentHIPStream().stream();
  bnn_status st;
  {
    Released released;
    st = call(stream);
  }
  return PyLong_FromLong((long)st);
}

// body(args) -> PyObject *; whatever it throws: not the plain case (tensors without storage throw c10::Error).
template <class Body>
PyObject *guarded(PyObject *const *a, Py_ssize_t n, Py_ssize_t want, const Body &body) {
  try {
    Args args(a, n, want);
    return body(args);
  } catch (...) {
    Py_RETURN_NONE;
  }
}

using at::kFloat;
using at::kInt;
using at::kLong;

PyObject *gemm(PyObject *, PyObject *const *a, Py_ssize_t n) {  // A, B, K, C
  return guarded(a, n, 4, [](Args &v) {
    const at::Tensor &A = v.tensor(kLong, 2), &B = v.tensor(kLong, 2);
    const int64_t K = v.integer();
    const at::Tensor &C = v.tensor(kInt, 2);
    const int64_t M = A.size(0), N = B.size(0), lda = row_stride(A, std::max<int64_t>(A.size(1), 1)),
                  ldb = row_stride(B, std::max<int64_t>(B.size(1), 1)), ldc = M > 1 ? C.stride(0) : std::max<int64_t>(N, 1);
    const uint64_t *const pa = u64(A), *const pb = u64(B);
    int32_t *const pc = i32(C.data_ptr());
    return launch([&](void *s) { return lib.gemm(pa, lda, pb, ldb, pc, ldc, M, N, K, s); });
  });
}

PyObject *epilogue(PyObject *, PyObject *const *a, Py_ssize_t n) {  // A, B, K, scale, bias, axis, Y
  return guarded(a, n, 7, [](Args &v) {
    const at::Tensor &A = v.tensor(kLong, 2), &B = v.tensor(kLong, 2);
    const int64_t K = v.integer();
    const float *const sc = f32(v.pointer()), *const bi = f32(v.pointer());
    const int axis = v.small();
    const at::Tensor &Y = v.tensor(kFloat, 2);
    const int64_t M = A.size(0), N = B.size(0), lda = row_stride(A, std::max<int64_t>(A.size(1), 1)),
                  ldb = row_stride(B, std::max<int64_t>(B.size(1), 1)), ld = std::max<int64_t>(N, 1);
    if (Y.size(0) != M || Y.size(1) != N || !Y.is_contiguous()) throw Other();
    const uint64_t *const pa = u64(A), *const pb = u64(B);
    float *const py = f32(Y.data_ptr());
    return launch([&](void *s) { return lib.epilogue(pa, lda, pb, ldb, M, N, K, nullptr, ld, py, ld, sc, bi, (bnn_ch_axis)axis, s); });
  });
}

PyObject *encode(PyObject *, PyObject *const *a, Py_ssize_t n) {  // src, dst
  return guarded(a, n, 2, [](Args &v) {
    const at::Tensor &src = v.tensor(kFloat, 2), &dst = v.tensor(kLong, 2);
    if (src.stride(1) != 1 || dst.stride(1) != 1) throw Other();
    const int64_t rows = src.size(0), K = src.size(1), Kw = K / 64 + (K % 64 != 0);
    const int64_t ls = rows > 1 ? src.stride(0) : std::max(K, src.stride(0)), ld = rows > 1 ? dst.stride(0) : std::max(Kw, dst.stride(0));
    const float *const ps = f32(src.data_ptr());
    uint64_t *const pd = u64(dst);
    return launch([&](void *s) { return lib.encode(ps, rows, K, ls, pd, ld, s); });
  });
}

PyObject *conv2d(PyObject *, PyObject *const *a, Py_ssize_t n) {  // x, w, D, kH, kW, stride, pad, out_i32, out_f32, scale, bias, workspace
  return guarded(a, n, 12, [](Args &v) {
    const at::Tensor &x = v.tensor(kFloat, 4), &w = v.tensor(kLong);
    const int D = v.small(), kH = v.small(), kW = v.small();
    int st[2], pd[2];
    v.pair(st);
    v.pair(pd);
    int32_t *const oi = i32(v.pointer());
    float *const of = f32(v.pointer());
    const float *const sc = f32(v.pointer()), *const bi = f32(v.pointer());
    const at::Tensor &ws = v.tensor();
    if (!x.is_contiguous() || !w.is_contiguous()) throw Other();
    const int N = size(x, 0), C = size(x, 1), H = size(x, 2), W = size(x, 3);
    const float *const px = f32(x.data_ptr());
    const uint64_t *const pw = u64(w);
    void *const pws = ws.data_ptr();
    const size_t nws = (size_t)ws.numel();
    return launch([&](void *s) {
      return lib.conv2d(px, pw, N, C, H, W, D, kH, kW, st[0], st[1], pd[0], pd[1], oi, of, sc, bi, pws, nws, s);
    });
  });
}

PyObject *conv2d_packed(PyObject *, PyObject *const *a, Py_ssize_t n) {  // xp, w, C, D, kH, kW, stride, pad, pool, i32, f32, packed, scale, bias
  return guarded(a, n, 14, [](Args &v) {
    const at::Tensor &x = v.tensor(kLong, 4), &w = v.tensor(kLong);
    const int C = v.small(), D = v.small(), kH = v.small(), kW = v.small();
    int st[2], pd[2];
    v.pair(st);
    v.pair(pd);
    const int pool = v.small();
    int32_t *const oi = i32(v.pointer());
    float *const of = f32(v.pointer());
    uint64_t *const op = static_cast<uint64_t *>(v.pointer());
    const float *const sc = f32(v.pointer()), *const bi = f32(v.pointer());
    if (!x.is_contiguous() || !w.is_contiguous() || C <= 0 || x.size(3) != ((int64_t)C + 63) / 64) throw Other();
    const int N = size(x, 0), H = size(x, 1), W = size(x, 2);
    const uint64_t *const px = u64(x), *const pw = u64(w);
    return launch([&](void *s) {
      return lib.conv2d_packed(px, pw, N, C, H, W, D, kH, kW, st[0], st[1], pd[0], pd[1], pool, oi, of, op, sc, bi, s);
    });
  });
}

PyObject *im2col(PyObject *, PyObject *const *a, Py_ssize_t n) {  // x, kH, kW, stride, pad, cols, workspace
  return guarded(a, n, 7, [](Args &v) {
    const at::Tensor &x = v.tensor(kFloat, 4);
    const int kH = v.small(), kW = v.small();
    int st[2], pd[2];
    v.pair(st);
    v.pair(pd);
    const at::Tensor &cols = v.tensor(kLong), &ws = v.tensor();
    if (!x.is_contiguous() || !cols.is_contiguous()) throw Other();
    const int N = size(x, 0), C = size(x, 1), H = size(x, 2), W = size(x, 3);
    // what the binding requires of cols, where its own arithmetic is plain
    if (kH <= 0 || kW <= 0 || st[0] <= 0 || st[1] <= 0 || pd[0] < 0 || pd[1] < 0) throw Other();
    const int64_t h = (int64_t)H + 2 * (int64_t)pd[0] - kH, w = (int64_t)W + 2 * (int64_t)pd[1] - kW;
    if (h < 0 || w < 0 || (double)N * (h / st[0] + 1) * (w / st[1] + 1) * kH * kW * (C / 64 + 1) > 1e15) throw Other();
    if (cols.numel() != N * (h / st[0] + 1) * (w / st[1] + 1) * kH * kW * (((int64_t)C + 63) / 64)) throw Other();
    const float *const px = f32(x.data_ptr());
    uint64_t *const pc = u64(cols);
    void *const pws = ws.data_ptr();
    const size_t nws = (size_t)ws.numel();
    return launch([&](void *s) { return lib.im2col(px, N, C, H, W, kH, kW, st[0], st[1], pd[0], pd[1], pc, pws, nws, s); });
  });
}

// x, w, scale, bias, stride, pad, out
template <class Out>
PyObject *first_layer(Args &v, bnn_status (*call)(const float *, const float *, int, int, int, int, int, int, int, int, int, int,
                                                  int, const float *, const float *, Out *, void *)) {
  const at::Tensor &x = v.tensor(kFloat, 4), &w = v.tensor(kFloat, 4);
  const float *const sc = f32(v.pointer()), *const bi = f32(v.pointer());
  int st[2], pd[2];
  v.pair(st);
  v.pair(pd);
  Out *const out = static_cast<Out *>(v.tensor().data_ptr());
  const int N = size(x, 0), C = size(x, 1), H = size(x, 2), W = size(x, 3), D = size(w, 0), kH = size(w, 2), kW = size(w, 3);
  const float *const px = f32(x.data_ptr()), *const pw = f32(w.data_ptr());
  return launch([&](void *s) { return call(px, pw, N, C, H, W, D, kH, kW, st[0], st[1], pd[0], pd[1], sc, bi, out, s); });
}

PyObject *f32_sign(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 7, [](Args &v) { return first_layer(v, lib.f32_sign); });
}

PyObject *conv2d_f32(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 7, [](Args &v) { return first_layer(v, lib.f32); });
}

PyObject *maxpool(PyObject *, PyObject *const *a, Py_ssize_t n) {  // in, out_i32, out_f32, scale, bias
  return guarded(a, n, 5, [](Args &v) {
    const at::Tensor &t = v.tensor(kInt, 4);
    int32_t *const oi = i32(v.pointer());
    float *const of = f32(v.pointer());
    const float *const sc = f32(v.pointer()), *const bi = f32(v.pointer());
    if (!t.is_contiguous()) throw Other();
    const int N = size(t, 0), D = size(t, 1), H = size(t, 2), W = size(t, 3);
    const int32_t *const p = i32(t.data_ptr());
    return launch([&](void *s) { return lib.maxpool(p, N, D, H, W, oi, of, sc, bi, s); });
  });
}

PyObject *fc(PyObject *, PyObject *const *a, Py_ssize_t n) {  // x, w, bias, sign_input, out
  return guarded(a, n, 5, [](Args &v) {
    const at::Tensor &x = v.tensor(kFloat, 2), &w = v.tensor(kFloat, 2);
    const float *const bi = f32(v.pointer());
    const int sign = v.small();
    float *const out = f32(v.tensor().data_ptr());
    const int64_t M = x.size(0), K = x.size(1), N = w.size(0);
    const float *const px = f32(x.data_ptr()), *const pw = f32(w.data_ptr());
    return launch([&](void *s) { return lib.fc(px, pw, bi, M, K, N, sign, out, s); });
  });
}

// ---- 8-bit and gated layers: matrices with rows of consecutive values, of given sizes and types, as the binding's checks ask ----
struct Matrix {
  char *p = nullptr;
  int64_t ld = 0, rows = 0, cols = 0;
};
Matrix matrix(const at::Tensor &t, at::ScalarType type) {
  if (!t.is_cuda() || t.scalar_type() != type || t.dim() != 2) throw Other();
  Matrix m;
  m.rows = t.size(0), m.cols = t.size(1);
  if (m.cols > 1 && t.stride(1) != 1) throw Other();
  m.ld = m.rows > 1 ? t.stride(0) : std::max(m.cols, t.stride(0));
  m.p = static_cast<char *>(t.data_ptr());
  return m;
}
Matrix matrix(const at::Tensor &t, at::ScalarType type, int64_t rows, int64_t cols) {
  const Matrix m = matrix(t, type);
  if (m.rows != rows || m.cols != cols) throw Other();
  return m;
}
Matrix matrix(const at::Tensor *t, at::ScalarType type, int64_t rows, int64_t cols) {
  return t ? matrix(*t, type, rows, cols) : Matrix();
}
float *vector(const at::Tensor *t, int64_t n) {
  if (!t) return nullptr;
  if (!t->is_cuda() || t->scalar_type() != kFloat || t->dim() != 1 || t->size(0) != n || (n > 1 && t->stride(0) != 1)) throw Other();
  return f32(t->data_ptr());
}
void *workspace(const at::Tensor &t, size_t &bytes) {
  if (!t.is_cuda() || !t.is_contiguous()) throw Other();
  bytes = (size_t)t.numel() * t.element_size();
  return t.data_ptr();
}
int float_type(at::ScalarType t) {
  if (t == kFloat) return BNN_F32;
  if (t == at::kBFloat16) return BNN_BF16;
  if (t == at::kHalf) return BNN_F16;
  throw Other();
}
int8_t *i8(const Matrix &m) { return reinterpret_cast<int8_t *>(m.p); }
using at::kChar;

PyObject *quant_rows(PyObject *, PyObject *const *a, Py_ssize_t n) {  // x, q, scale
  return guarded(a, n, 3, [](Args &v) {
    const at::Tensor &t = v.tensor();
    const int type = float_type(t.scalar_type());
    const Matrix x = matrix(t, t.scalar_type()), q = matrix(v.tensor(), kChar, x.rows, x.cols);
    float *const scale = vector(&v.tensor(), x.rows);
    return launch([&](void *s) { return lib.quant(x.p, type, x.rows, x.cols, x.ld, i8(q), q.ld, scale, s); });
  });
}

PyObject *linear_i8(PyObject *, PyObject *const *args, Py_ssize_t n) {  // a, a_scale, b, b_scale, bias, out
  return guarded(args, n, 6, [](Args &v) {
    const Matrix a = matrix(v.tensor(), kChar);
    const float *const sa = vector(&v.tensor(), a.rows);
    const Matrix b = matrix(v.tensor(), kChar);
    const float *const sb = vector(&v.tensor(), b.rows), *const bias = vector(v.tensor_or_none(), b.rows);
    const at::Tensor &out = v.tensor();
    const Matrix y = matrix(out, out.scalar_type(), a.rows, b.rows);
    if (b.cols != a.cols) throw Other();
    const int type = float_type(out.scalar_type());
    return launch([&](void *s) { return lib.linear(i8(a), a.ld, sa, i8(b), b.ld, sb, bias, a.rows, b.rows, a.cols, y.p, type, y.ld, s); });
  });
}

// b, r, gate, gate_rows, res_scale, w_post, bias_post, w_pre, bias_pre, post, pre, eps
bnn_norm_gate_in norm_in(Args &v, at::ScalarType &type, at::ScalarType &r_type) {
  const at::Tensor *const b = v.tensor_or_none();
  const at::Tensor &r = v.tensor();
  const at::Tensor *const gate = v.tensor_or_none();
  const int64_t gate_rows = v.integer();
  r_type = r.scalar_type();
  type = b ? b->scalar_type() : r_type;
  const Matrix mr = matrix(r, r_type), mb = matrix(b, type, mr.rows, mr.cols);
  if (gate && gate_rows < 1) throw Other();
  const Matrix mg = matrix(gate, type, gate ? (mr.rows - 1) / gate_rows + 1 : 0, mr.cols);
  if (mr.rows < 1 || mr.cols > (1 << 30)) throw Other();
  bnn_norm_gate_in in = {};
  in.rows = mr.rows, in.D = (int)mr.cols;
  in.type = float_type(type), in.r_type = float_type(r_type);
  in.b = mb.p, in.b_ld = mb.ld, in.r = mr.p, in.r_ld = mr.ld, in.gate = mg.p, in.gate_ld = mg.ld, in.gate_rows = gate ? gate_rows : 0;
  const float **const vectors[] = {&in.res_scale, &in.w_post, &in.bias_post, &in.w_pre, &in.bias_pre};
  for (const float **to : vectors) *to = vector(v.tensor_or_none(), mr.cols);
  in.post = v.small(), in.pre = v.small();
  in.eps = v.real();
  return in;
}

PyObject *norm_gate(PyObject *, PyObject *const *a, Py_ssize_t n) {  // norm_in's, r_out, n_out, q_out, q_scale
  return guarded(a, n, 16, [](Args &v) {
    at::ScalarType type, r_type;
    const bnn_norm_gate_in in = norm_in(v, type, r_type);
    const Matrix r = matrix(v.tensor_or_none(), r_type, in.rows, in.D), out = matrix(v.tensor_or_none(), type, in.rows, in.D),
                 q = matrix(v.tensor_or_none(), kChar, in.rows, in.D);
    float *const scale = vector(v.tensor_or_none(), in.rows);
    return launch([&](void *s) { return lib.norm(&in, r.p, r.ld, out.p, out.ld, i8(q), q.ld, scale, s); });
  });
}

// norm_in's, dn, dr_out, dr, db, dgate, dres_scale, dw_post, dbias_post, dw_pre, dbias_pre, workspace
PyObject *norm_gate_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 23, [](Args &v) {
    at::ScalarType type, r_type;
    const bnn_norm_gate_in in = norm_in(v, type, r_type);
    const Matrix dn = matrix(v.tensor_or_none(), type, in.rows, in.D), dro = matrix(v.tensor_or_none(), r_type, in.rows, in.D),
                 dr = matrix(v.tensor(), r_type, in.rows, in.D), db = matrix(v.tensor_or_none(), type, in.rows, in.D),
                 dg = matrix(v.tensor_or_none(), type, in.gate ? (in.rows - 1) / in.gate_rows + 1 : 0, in.D);
    float *sums[5];
    for (float *&p : sums) p = vector(v.tensor_or_none(), in.D);
    size_t nws;
    void *const pws = workspace(v.tensor(), nws);
    return launch([&](void *s) {
      return lib.norm_backward(&in, dn.p, dn.ld, dro.p, dro.ld, dr.p, dr.ld, db.p, db.ld, dg.p, dg.ld, sums[0], sums[1], sums[2], sums[3],
                               sums[4], pws, nws, s);
    });
  });
}

// Room for a call of its own, and its results: eight tensors made one by one from Python are 14 us, here 5.
at::Tensor room(size_t bytes, const at::Tensor &on) {
  return at::empty({(int64_t)std::max<size_t>(bytes, 16)}, on.options().dtype(at::kByte));
}
at::Tensor like(const at::Tensor &t) { return at::empty(t.sizes(), t.options(), at::MemoryFormat::Contiguous); }

// The tensors of a call that went through, None for those that are not there; else its status.
template <size_t N>
PyObject *results(PyObject *status, const at::Tensor (&made)[N]) {
  if (!status || PyLong_AsLong(status) != BNN_OK) return status;
  Py_DECREF(status);
  PyObject *const all = PyTuple_New(N);
  if (!all) return nullptr;
  for (size_t i = 0; i < N; ++i) {
    PyObject *const o = made[i].defined() ? THPVariable_Wrap(made[i]) : Py_NewRef(Py_None);
    if (!o) {
      Py_DECREF(all);
      return nullptr;
    }
    PyTuple_SET_ITEM(all, i, o);
  }
  return all;
}

// norm_in's, dn, dr_out -> dr, db, dgate, dres_scale, dw_post, dbias_post, dw_pre, dbias_pre
PyObject *norm_gate_gradients(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 14, [&](Args &v) {
    at::ScalarType type, r_type;
    const bnn_norm_gate_in in = norm_in(v, type, r_type);
    const Matrix dn = matrix(v.tensor_or_none(), type, in.rows, in.D), dro = matrix(v.tensor_or_none(), r_type, in.rows, in.D);
    constexpr int of[] = {1, 0, 2, 4, 5, 6, 7, 8};  // whose gradient each is
    at::Tensor made[8];
    void *p[8];
    for (int i = 0; i < 8; ++i) {
      if (a[of[i]] != Py_None) made[i] = like(THPVariable_Unpack(a[of[i]]));
      p[i] = made[i].defined() ? made[i].data_ptr() : nullptr;
    }
    const size_t bytes = lib.norm_workspace(in.rows, in.D, in.gate_rows);
    const at::Tensor ws = room(bytes, made[0]);
    return results(launch([&](void *s) {
      return lib.norm_backward(&in, dn.p, dn.ld, dro.p, dro.ld, p[0], in.D, p[1], in.D, p[2], in.D, f32(p[3]), f32(p[4]), f32(p[5]), f32(p[6]),
                               f32(p[7]), ws.data_ptr(), bytes, s);
    }), made);
  });
}

float *saved_of(const at::Tensor *t, int64_t T, int64_t F) {
  if (!t) return nullptr;
  if (!t->is_cuda() || t->scalar_type() != kFloat || t->dim() != 3 || t->size(0) != 2 || t->size(1) != T || t->size(2) != F || !t->is_contiguous())
    throw Other();
  return f32(t->data_ptr());
}

PyObject *gated_ff(PyObject *, PyObject *const *a, Py_ssize_t n) {  // x, wg, wu, act, out, saved
  return guarded(a, n, 6, [](Args &v) {
    const at::Tensor &t = v.tensor();
    const at::ScalarType type = t.scalar_type();
    const Matrix x = matrix(t, type), wg = matrix(v.tensor(), type);
    if (wg.cols != x.cols) throw Other();
    const Matrix wu = matrix(v.tensor(), type, wg.rows, x.cols);
    const int act = v.small();
    const Matrix h = matrix(v.tensor(), type, x.rows, wg.rows);
    float *const saved = saved_of(v.tensor_or_none(), x.rows, wg.rows);
    const int code = float_type(type);
    return launch([&](void *s) { return lib.gated(x.p, x.ld, wg.p, wg.ld, wu.p, wu.ld, code, x.rows, x.cols, wg.rows, act, h.p, h.ld, saved, s); });
  });
}

PyObject *gated_ff_i8(PyObject *, PyObject *const *a, Py_ssize_t n) {  // x, x_scale, wg, wg_scale, wu, wu_scale, act, out
  return guarded(a, n, 8, [](Args &v) {
    const Matrix x = matrix(v.tensor(), kChar);
    const float *const sx = vector(&v.tensor(), x.rows);
    const Matrix wg = matrix(v.tensor(), kChar);
    const float *const sg = vector(&v.tensor(), wg.rows);
    if (wg.cols != x.cols) throw Other();
    const Matrix wu = matrix(v.tensor(), kChar, wg.rows, x.cols);
    const float *const su = vector(&v.tensor(), wg.rows);
    const int act = v.small();
    const at::Tensor &out = v.tensor();
    const Matrix h = matrix(out, out.scalar_type(), x.rows, wg.rows);
    const int code = float_type(out.scalar_type());
    return launch([&](void *s) {
      return lib.gated_i8(i8(x), x.ld, sx, i8(wg), wg.ld, sg, i8(wu), wu.ld, su, x.rows, x.cols, wg.rows, act, h.p, code, h.ld, s);
    });
  });
}

PyObject *gated_ff_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {  // x, wg, wu, saved, dh, dx, dwg, dwu, workspace
  return guarded(a, n, 9, [](Args &v) {
    const at::Tensor &t = v.tensor();
    const at::ScalarType type = t.scalar_type();
    const Matrix x = matrix(t, type), wg = matrix(v.tensor(), type);
    if (wg.cols != x.cols) throw Other();
    const int64_t T = x.rows, D = x.cols, F = wg.rows;
    const Matrix wu = matrix(v.tensor(), type, F, D);
    const float *const saved = saved_of(&v.tensor(), T, F);
    const Matrix dh = matrix(v.tensor(), type, T, F), dx = matrix(v.tensor(), type, T, D), dwg = matrix(v.tensor(), type, F, D),
                 dwu = matrix(v.tensor(), type, F, D);
    size_t nws;
    void *const pws = workspace(v.tensor(), nws);
    const int code = float_type(type);
    return launch([&](void *s) {
      return lib.gated_backward(x.p, x.ld, wg.p, wg.ld, wu.p, wu.ld, code, T, D, F, saved, dh.p, dh.ld, dx.p, dx.ld, dwg.p, dwg.ld, dwu.p,
                                dwu.ld, pws, nws, s);
    });
  });
}

PyObject *gated_ff_gradients(PyObject *, PyObject *const *a, Py_ssize_t n) {  // x, wg, wu, saved, dh -> dx, dwg, dwu
  return guarded(a, n, 5, [](Args &v) {
    const at::Tensor &tx = v.tensor(), &tg = v.tensor(), &tu = v.tensor();
    const at::ScalarType type = tx.scalar_type();
    const Matrix x = matrix(tx, type), wg = matrix(tg, type);
    if (wg.cols != x.cols) throw Other();
    const int64_t T = x.rows, D = x.cols, F = wg.rows;
    const Matrix wu = matrix(tu, type, F, D);
    const float *const saved = saved_of(&v.tensor(), T, F);
    const Matrix dh = matrix(v.tensor(), type, T, F);
    const int code = float_type(type);
    const at::Tensor made[3] = {like(tx), like(tg), like(tu)};
    const size_t bytes = lib.gated_workspace(T, D, F);
    const at::Tensor ws = room(bytes, tx);
    void *const p[3] = {made[0].data_ptr(), made[1].data_ptr(), made[2].data_ptr()};
    return results(launch([&](void *s) {
      return lib.gated_backward(x.p, x.ld, wg.p, wg.ld, wu.p, wu.ld, code, T, D, F, saved, dh.p, dh.ld, p[0], D, p[1], D, p[2], D,
                                ws.data_ptr(), bytes, s);
    }), made);
  });
}

// ---- 8-bit floating point and experts: outputs are made here where they are not given (None); what comes back are the tensors ----
const at::Tensor &present(const at::Tensor &t, at::ScalarType type) {  // on the device whose stream the call goes to
  if (!t.is_cuda() || t.scalar_type() != type || t.get_device() != c10::hip::getCurrentHIPStream().device_index()) throw Other();
  return t;
}
Matrix present_matrix(const at::Tensor &t, at::ScalarType type) { return matrix(present(t, type), type); }
Matrix present_matrix(const at::Tensor &t, at::ScalarType type, int64_t rows, int64_t cols) {
  return matrix(present(t, type), type, rows, cols);
}
template <class T>
T *whole(const at::Tensor *t, at::ScalarType type, std::initializer_list<int64_t> shape) {
  if (!t) return nullptr;
  if (present(*t, type).sizes() != at::IntArrayRef(shape) || !t->is_contiguous()) throw Other();
  return static_cast<T *>(t->data_ptr());
}
// Rows with `row` elements of room each, [rows, cols] or for experts [experts, rows, cols], as the binding checks them.
struct Padded {
  uint8_t *p;
  int64_t ld, between;
};
Padded padded(const at::Tensor &t, int64_t experts, int64_t rows, int64_t cols, int64_t row, int64_t quantum) {
  const int64_t d = t.dim();
  if (d != (experts < 0 ? 2 : 3) || t.size(d - 2) != rows || t.size(d - 1) != cols || (experts >= 0 && t.size(0) != experts)) throw Other();
  if (cols > 1 && t.stride(d - 1) != 1) throw Other();
  Padded m;
  m.ld = rows > 1 ? t.stride(d - 2) : std::max((row + quantum - 1) / quantum * quantum, t.stride(d - 2) / quantum * quantum);
  m.between = experts > 1 ? t.stride(0) : rows * m.ld;
  if (m.ld < row) throw Other();
  if (t.numel() > 0) {
    const double last = (double)t.storage_offset() + (double)(std::max<int64_t>(experts, 1) - 1) * m.between + (double)(rows - 1) * m.ld + row;
    if (last * t.element_size() > (double)t.storage().nbytes()) throw Other();
  }
  m.p = static_cast<uint8_t *>(t.data_ptr());
  return m;
}
int64_t blocks_of(int64_t K) { return (K + 127) / 128; }
constexpr at::ScalarType kF8 = at::kFloat8_e4m3fn, kE8 = at::kFloat8_e8m0fnu;
Padded f8_values(const at::Tensor &t, int64_t experts, int64_t rows, int64_t K) {
  return padded(present(t, kF8), experts, rows, K, blocks_of(K) * 128, 16);
}
Padded f8_scales(const at::Tensor &t, int64_t experts, int64_t rows, int64_t K) {
  return padded(present(t, kE8), experts, rows, blocks_of(K), (blocks_of(K) + 3) / 4 * 4, 4);
}
struct Weight {
  Padded q, s;
  int wide, per;
};
Weight f8_weight(const at::Tensor &q, const at::Tensor &s, int64_t experts, int64_t N, int64_t K) {
  Weight w;
  w.q = f8_values(q, experts, N, K);
  w.wide = s.scalar_type() == kFloat;
  if (s.dim() != q.dim()) throw Other();
  w.per = s.size(s.dim() - 2) == N && !w.wide && N > 1 ? 1 : 128;
  const int64_t rows = w.per == 1 ? N : blocks_of(N);
  w.s = w.wide ? padded(present(s, kFloat), experts, rows, blocks_of(K), blocks_of(K), 1) : f8_scales(s, experts, rows, K);
  return w;
}
at::Tensor made_f8(const at::Tensor *t, int64_t rows, int64_t K, const at::Tensor &on) {
  return t ? *t : at::empty({rows, blocks_of(K) * 128}, on.options().dtype(kF8)).narrow(1, 0, K);
}
at::Tensor made_scales(const at::Tensor *t, int64_t rows, int64_t K, const at::Tensor &on) {
  return t ? *t : at::empty({rows, (blocks_of(K) + 3) / 4 * 4}, on.options().dtype(kE8)).narrow(1, 0, blocks_of(K));
}
at::Tensor made(const at::Tensor *t, at::IntArrayRef sizes, at::ScalarType type, const at::Tensor &on) {
  return t ? *t : at::empty(sizes, on.options().dtype(type));
}
int product_type(const at::Tensor &out, Args &v) {  // with the next argument, a choice of sums
  return float_type(out.scalar_type()) | v.small();
}
PyObject *result(PyObject *status, const at::Tensor &t) {
  if (!status || PyLong_AsLong(status) != BNN_OK) return status;
  Py_DECREF(status);
  return THPVariable_Wrap(t);
}

// x, q, scale, rows, k, columns -> q, scale
PyObject *quant_f8(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 6, [](Args &v) {
    const at::Tensor &t = v.tensor(), *const gq = v.tensor_or_none(), *const gs = v.tensor_or_none(), *const gr = v.tensor_or_none();
    const int64_t k = v.integer();
    const bool columns = v.integer() != 0;
    const int type = float_type(t.scalar_type());
    const Matrix x = present_matrix(t, t.scalar_type());
    if (gr && gr->dim() != 1) throw Other();
    const int64_t S = gr ? gr->size(0) : x.rows, out_rows = columns ? x.cols : S, K = columns ? S : x.cols;
    const int32_t *const rows = gr ? whole<int32_t>(gr, kInt, {S}) : nullptr;
    const at::Tensor out[2] = {made_f8(gq, out_rows, K, t), made_scales(gs, out_rows, K, t)};
    const Padded q = f8_values(out[0], -1, out_rows, K), s = f8_scales(out[1], -1, out_rows, K);
    return results(launch([&](void *stream) {
      return (columns ? lib.quant_columns : lib.quant_blocks)(x.p, type, x.rows, x.ld, rows, k, S, x.cols, q.p, q.ld, s.p, s.ld, stream);
    }), out);
  });
}

PyObject *linear_f8(PyObject *, PyObject *const *args, Py_ssize_t n) {  // a, a_scale, b, b_scale, bias, out, sums -> status
  return guarded(args, n, 7, [](Args &v) {
    const at::Tensor &ta = v.tensor(), &tsa = v.tensor(), &tb = v.tensor(), &tsb = v.tensor();
    if (ta.dim() != 2 || tb.dim() != 2) throw Other();
    const int64_t M = ta.size(0), K = ta.size(1), N = tb.size(0);
    const Padded a = f8_values(ta, -1, M, K), sa = f8_scales(tsa, -1, M, K);
    const Weight b = f8_weight(tb, tsb, -1, N, K);
    const at::Tensor *const tbias = v.tensor_or_none();
    if (tbias) present(*tbias, kFloat);
    const float *const bias = vector(tbias, N);
    const at::Tensor &out = v.tensor();
    const int code = product_type(out, v);
    const Matrix y = present_matrix(out, out.scalar_type(), M, N);
    return launch([&](void *s) {
      return lib.linear_f8(a.p, a.ld, sa.p, sa.ld, b.q.p, b.q.ld, b.s.p, b.wide, b.s.ld, b.per, bias, M, N, K, y.p, code, y.ld, s);
    });
  });
}

PyObject *expert_linear_f8(PyObject *, PyObject *const *args, Py_ssize_t n) {  // a, a_scale, offsets, b, b_scale, out, sums -> status
  return guarded(args, n, 7, [](Args &v) {
    const at::Tensor &ta = v.tensor(), &tsa = v.tensor(), &to = v.tensor(), &tb = v.tensor(), &tsb = v.tensor(), &out = v.tensor();
    if (ta.dim() != 2 || tb.dim() != 3) throw Other();
    const int64_t S = ta.size(0), K = ta.size(1), E = tb.size(0), N = tb.size(1);
    const Padded a = f8_values(ta, -1, S, K), sa = f8_scales(tsa, -1, S, K);
    const Weight b = f8_weight(tb, tsb, E, N, K);
    const int32_t *const offsets = whole<int32_t>(&to, kInt, {E + 1});
    const int code = product_type(out, v);
    const Matrix y = present_matrix(out, out.scalar_type(), S, N);
    return launch([&](void *s) {
      return lib.expert_linear(a.p, a.ld, sa.p, sa.ld, offsets, E, b.q.p, b.q.ld, b.q.between, b.s.p, b.wide, b.s.ld, b.s.between, b.per, S, N,
                               K, y.p, code, y.ld, s);
    });
  });
}

PyObject *expert_linear_f8_dw(PyObject *, PyObject *const *args, Py_ssize_t n) {  // a, a_scale, b, b_scale, offsets, out, sums -> status
  return guarded(args, n, 7, [](Args &v) {
    const at::Tensor &ta = v.tensor(), &tsa = v.tensor(), &tb = v.tensor(), &tsb = v.tensor(), &to = v.tensor(), &out = v.tensor();
    if (ta.dim() != 2 || tb.dim() != 2 || to.dim() != 1 || to.size(0) < 1) throw Other();
    const int64_t N = ta.size(0), S = ta.size(1), K = tb.size(0), E = to.size(0) - 1;
    const Padded a = f8_values(ta, -1, N, S), sa = f8_scales(tsa, -1, N, S), b = f8_values(tb, -1, K, S), sb = f8_scales(tsb, -1, K, S);
    const int32_t *const offsets = whole<int32_t>(&to, kInt, {E + 1});
    const int code = product_type(out, v);
    const Padded dw = padded(present(out, out.scalar_type()), E, N, K, K, 1);
    return launch([&](void *s) {
      return lib.expert_linear_dw(a.p, a.ld, sa.p, sa.ld, b.p, b.ld, sb.p, sb.ld, offsets, E, N, K, S, dw.p, code, dw.ld, dw.between, s);
    });
  });
}

// experts, E, align, offsets, rows, places, workspace -> offsets, rows, places
PyObject *expert_sort(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 7, [](Args &v) {
    const at::Tensor &t = v.tensor();
    const int64_t E = v.integer(), align = v.integer();
    const at::Tensor *const go = v.tensor_or_none(), *const gr = v.tensor_or_none(), *const gp = v.tensor_or_none(), *const gw = v.tensor_or_none();
    if ((t.scalar_type() != kInt && t.scalar_type() != kLong) || t.dim() != 2 || !t.is_contiguous() || E < 1) throw Other();
    present(t, t.scalar_type());
    const int64_t T = t.size(0), k = t.size(1);
    const at::Tensor out[3] = {made(go, {E + 1}, kInt, t), made(gr, {gr ? 0 : lib.expert_rows(T, k, E, align)}, kInt, t), made(gp, {T, k}, kInt, t)};
    if (out[1].dim() != 1) throw Other();
    const int64_t S = out[1].size(0);
    int32_t *const offsets = whole<int32_t>(&out[0], kInt, {E + 1}), *const rows = whole<int32_t>(&out[1], kInt, {S}),
            *const places = whole<int32_t>(&out[2], kInt, {T, k});
    size_t bytes = lib.sort_workspace(T, k, E);
    at::Tensor room_for;
    void *ws = nullptr;
    if (gw) ws = workspace(present(*gw, gw->scalar_type()), bytes);
    else if (bytes) room_for = room(bytes, t), ws = room_for.data_ptr();
    return results(launch([&](void *s) {
      return lib.sort(t.data_ptr(), t.scalar_type() == kLong ? 8 : 4, T, k, E, align, S, offsets, rows, places, ws, bytes, s);
    }), out);
  });
}

PyObject *expert_gather(PyObject *, PyObject *const *a, Py_ssize_t n) {  // x, rows, k, out -> out
  return guarded(a, n, 4, [](Args &v) {
    const at::Tensor &t = v.tensor(), &tr = v.tensor();
    const int64_t k = v.integer();
    const at::ScalarType type = t.scalar_type();
    const Matrix x = present_matrix(t, type);
    if (tr.dim() != 1) throw Other();
    const int64_t S = tr.size(0);
    const int32_t *const rows = whole<int32_t>(&tr, kInt, {S});
    const int code = float_type(type);
    const at::Tensor out = made(v.tensor_or_none(), {S, x.cols}, type, t);
    const Matrix y = present_matrix(out, type, S, x.cols);
    return result(launch([&](void *s) { return lib.gather(x.p, code, x.rows, x.ld, rows, k, S, x.cols, y.p, y.ld, s); }), out);
  });
}

PyObject *expert_combine(PyObject *, PyObject *const *a, Py_ssize_t n) {  // ys, places, weights, out -> out
  return guarded(a, n, 4, [](Args &v) {
    const at::Tensor &t = v.tensor(), &tp = v.tensor(), *const tw = v.tensor_or_none();
    const at::ScalarType type = t.scalar_type();
    const Matrix ys = present_matrix(t, type);
    if (tp.dim() != 2) throw Other();
    const int64_t T = tp.size(0), k = tp.size(1);
    const int32_t *const places = whole<int32_t>(&tp, kInt, {T, k});
    const float *const weights = whole<float>(tw, kFloat, {T, k});
    const int code = float_type(type);
    const at::Tensor out = made(v.tensor_or_none(), {T, ys.cols}, type, t);
    const Matrix y = present_matrix(out, type, T, ys.cols);
    return result(launch([&](void *s) { return lib.combine(ys.p, code, ys.rows, ys.ld, places, weights, T, k, ys.cols, y.p, y.ld, s); }), out);
  });
}

// ys, rows, places, weights, dout, dys, dweights -> dys, dweights
PyObject *expert_combine_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
  return guarded(a, n, 7, [](Args &v) {
    const at::Tensor &t = v.tensor(), &tr = v.tensor(), &tp = v.tensor(), *const tw = v.tensor_or_none(), &td = v.tensor();
    const at::ScalarType type = t.scalar_type();
    const Matrix ys = present_matrix(t, type);
    if (tp.dim() != 2) throw Other();
    const int64_t T = tp.size(0), k = tp.size(1), S = ys.rows, D = ys.cols;
    const int32_t *const rows = whole<int32_t>(&tr, kInt, {S}), *const places = whole<int32_t>(&tp, kInt, {T, k});
    const float *const weights = whole<float>(tw, kFloat, {T, k});
    const Matrix dout = present_matrix(td, type, T, D);
    const int code = float_type(type);
    const at::Tensor *const gy = v.tensor_or_none(), *const gw = v.tensor_or_none();
    const at::Tensor out[2] = {made(gy, {S, D}, type, t), made(gw, {T, k}, kFloat, t)};
    const Matrix dys = present_matrix(out[0], type, S, D);
    float *const dweights = whole<float>(&out[1], kFloat, {T, k});
    return results(launch([&](void *s) {
      return lib.combine_backward(ys.p, code, S, ys.ld, rows, places, weights, dout.p, dout.ld, T, k, D, dys.p, dys.ld, dweights, s);
    }), out);
  });
}

struct Gated {
  Matrix gu;
  int64_t S, F;
  int code;
  at::ScalarType type;
};
Gated gated_of(const at::Tensor &t) {
  Gated g;
  g.type = t.scalar_type(), g.code = float_type(g.type), g.gu = present_matrix(t, g.type);
  if (g.gu.cols % 2) throw Other();
  g.S = g.gu.rows, g.F = g.gu.cols / 2;
  return g;
}
PyObject *gated_act(PyObject *, PyObject *const *a, Py_ssize_t n) {  // gu, act, out, live -> out
  return guarded(a, n, 4, [](Args &v) {
    const at::Tensor &t = v.tensor();
    const Gated g = gated_of(t);
    const int act = v.small();
    const at::Tensor out = made(v.tensor_or_none(), {g.S, g.F}, g.type, t);
    const int32_t *const live = whole<int32_t>(v.tensor_or_none(), kInt, {1});
    const Matrix h = present_matrix(out, g.type, g.S, g.F);
    return result(launch([&](void *s) { return lib.gated_act(g.gu.p, g.code, g.S, g.gu.ld, g.F, act, live, h.p, h.ld, s); }), out);
  });
}
PyObject *gated_act_f8(PyObject *, PyObject *const *a, Py_ssize_t n) {  // gu, act, q, scale, live -> q, scale
  return guarded(a, n, 5, [](Args &v) {
    const at::Tensor &t = v.tensor();
    const Gated g = gated_of(t);
    const int act = v.small();
    const at::Tensor *const gq = v.tensor_or_none(), *const gs = v.tensor_or_none();
    const int32_t *const live = whole<int32_t>(v.tensor_or_none(), kInt, {1});
    const at::Tensor out[2] = {made_f8(gq, g.S, g.F, t), made_scales(gs, g.S, g.F, t)};
    const Padded q = f8_values(out[0], -1, g.S, g.F), sc = f8_scales(out[1], -1, g.S, g.F);
    return results(launch([&](void *s) { return lib.gated_act_f8(g.gu.p, g.code, g.S, g.gu.ld, g.F, act, live, q.p, q.ld, sc.p, sc.ld, s); }), out);
  });
}
PyObject *gated_act_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {  // gu, dh, act, out, live -> out
  return guarded(a, n, 5, [](Args &v) {
    const at::Tensor &t = v.tensor(), &td = v.tensor();
    const Gated g = gated_of(t);
    const int act = v.small();
    const Matrix dh = present_matrix(td, g.type, g.S, g.F);
    const at::Tensor out = made(v.tensor_or_none(), {g.S, 2 * g.F}, g.type, t);
    const int32_t *const live = whole<int32_t>(v.tensor_or_none(), kInt, {1});
    const Matrix dgu = present_matrix(out, g.type, g.S, 2 * g.F);
    return result(launch([&](void *s) {
      return lib.gated_act_backward(g.gu.p, g.code, g.S, g.gu.ld, g.F, act, live, dh.p, dh.ld, dgu.p, dgu.ld, s);
    }), out);
  });
}

PyObject *bind(PyObject *, PyObject *const *a, Py_ssize_t n) {
  constexpr Py_ssize_t want = sizeof(Library) / sizeof(void *);
  static_assert(want == sizeof(names) / sizeof(names[0]), "an address for every name");
  void *p[want];
  if (n != want) {
    PyErr_SetString(PyExc_TypeError, "one address per name");
    return nullptr;
  }
  for (Py_ssize_t i = 0; i < want; ++i) {
    p[i] = PyLong_AsVoidPtr(a[i]);
    if (!p[i]) {
      if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "an address");
      return nullptr;
    }
  }
  memcpy(&lib, p, sizeof lib);
  Py_RETURN_NONE;
}

#define BNN_METHOD(f) {#f, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)(void)>(f)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {BNN_METHOD(bind), BNN_METHOD(gemm), BNN_METHOD(epilogue), BNN_METHOD(encode), BNN_METHOD(conv2d),
                         BNN_METHOD(conv2d_packed), BNN_METHOD(im2col), BNN_METHOD(f32_sign), BNN_METHOD(conv2d_f32),
                         BNN_METHOD(maxpool), BNN_METHOD(fc), BNN_METHOD(quant_rows), BNN_METHOD(linear_i8),
                         BNN_METHOD(norm_gate), BNN_METHOD(norm_gate_backward), BNN_METHOD(norm_gate_gradients), BNN_METHOD(gated_ff), BNN_METHOD(gated_ff_i8),
                         BNN_METHOD(gated_ff_backward), BNN_METHOD(gated_ff_gradients), BNN_METHOD(quant_f8), BNN_METHOD(linear_f8),
                         BNN_METHOD(expert_linear_f8), BNN_METHOD(expert_linear_f8_dw), BNN_METHOD(expert_sort), BNN_METHOD(expert_gather),
                         BNN_METHOD(expert_combine), BNN_METHOD(expert_combine_backward), BNN_METHOD(gated_act), BNN_METHOD(gated_act_f8),
                         BNN_METHOD(gated_act_backward), {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensorcall", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensorcall() {
  PyObject *m = PyModule_Create(&module);
  if (!m) return nullptr;
  PyObject *t = PyTuple_New(sizeof(names) / sizeof(names[0]));
  if (!t) return nullptr;
  for (size_t i = 0; i < sizeof(names) / sizeof(names[0]); ++i) PyTuple_SET_ITEM(t, i, PyUnicode_FromString(names[i]));
  if (PyModule_AddObject(m, "names", t) < 0) return nullptr;
  if (PyModule_AddStringConstant(m, "built_for", BNN_BUILT_FOR) < 0) return nullptr;
  return m;
}
