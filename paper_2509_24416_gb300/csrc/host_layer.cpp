// One call of a prepared layer from Python: the checks, the two output
// allocations and the two launches of rotate-quant + product in one native
// call.  A pass over a small layer lasts 8 us on the GPU; the same steps in
// Python took the host 32 us (three allocations 5, two stream look-ups 6, the two
// C calls with their launches 7, the rest interpreter time), this call about 9.
//
// Only the plain case is taken: a 2-D fp16 / bf16 CUDA tensor with unit column
// stride and the layer's K columns, and weights in a layout its width names.
// Anything else returns None, and the Python path goes on with it (and raises
// what it always raised).
//
// The microscaled operators have the same: mx_quantize, mx_dequantize, mx_layer,
// mx_route and mx_experts are mx.py's calls of those names without the interpreter
// between their C calls.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/clq_mx.h"

namespace {

// Layout of a weight code array of `width` bytes a row for K codes, or -1.
int codes_layout(int64_t width, int64_t K) {
  if (width == K) return CLQ_CODES_E4M3;
  if (2 * width == K) return CLQ_CODES_INT4_PACKED;
  if (width == 2 * K) return CLQ_CODES_E4M3_SPLIT;
  if (4 * width == 3 * K) return CLQ_CODES_E2M3;
  return -1;
}

int64_t codes_width(int64_t codes, int64_t K) {
  switch (codes) {
    case CLQ_CODES_INT4_PACKED: return K / 2;
    case CLQ_CODES_E4M3: return K;
    case CLQ_CODES_E4M3_SPLIT: return 2 * K;
    case CLQ_CODES_E2M3: return K / 4 * 3;
    default: return -1;
  }
}

// layer(X, perm, We, s_w, bias | None, b, K, a_codes) -> Y [M, N] on the current
// stream, whose pool the buffers come from; None: not the plain case; an int:
// status | 256 * (0 rotate-quant, 1 product).
PyObject* layer(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 8) {
    PyErr_SetString(PyExc_TypeError, "layer() takes 8 arguments");
    return nullptr;
  }
  for (int i = 0; i < 4; ++i)
    if (!THPVariable_Check(args[i])) Py_RETURN_NONE;
  const bool has_bias = args[4] != Py_None;
  if (has_bias && !THPVariable_Check(args[4])) Py_RETURN_NONE;
  const at::Tensor& X = THPVariable_Unpack(args[0]);
  const at::Tensor& We = THPVariable_Unpack(args[2]);
  const long b = PyLong_AsLong(args[5]);
  const long K = PyLong_AsLong(args[6]);
  const long a_codes = PyLong_AsLong(args[7]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  if (!X.is_cuda() || X.dim() != 2 || X.stride(1) != 1 || X.size(1) != K || We.dim() != 2)
    Py_RETURN_NONE;
  const at::ScalarType dt = X.scalar_type();
  if (dt != at::kHalf && dt != at::kBFloat16) Py_RETURN_NONE;
  if (has_bias && THPVariable_Unpack(args[4]).scalar_type() != dt) Py_RETURN_NONE;
  const int64_t M = X.size(0), N = We.size(0), ld = X.stride(0);
  const int w_codes = codes_layout(We.size(1), K);
  const int64_t width = codes_width(a_codes, K);
  // (8-bit weights go with 8-bit activations only)
  if (w_codes < 0 || width < 0 ||
      (w_codes == CLQ_CODES_E4M3_SPLIT && a_codes != CLQ_CODES_E4M3_SPLIT) ||
      M > INT32_MAX || N > INT32_MAX || ld > INT32_MAX || b < 0 || b > INT32_MAX)
    Py_RETURN_NONE;
  void* stream = c10::cuda::getCurrentCUDAStream().stream();
  // Activation codes and, behind them, their fp32 scales: one buffer.
  const int64_t codes_bytes = (M * width + 15) / 16 * 16;
  at::Tensor codes = at::empty({codes_bytes + 4 * M}, X.options().dtype(at::kByte));
  at::Tensor Y = at::empty({M, N}, X.options());
  uint8_t* Xq = codes.data_ptr<uint8_t>();
  float* s_x = reinterpret_cast<float*>(Xq + codes_bytes);
  const clq_dtype cdt = dt == at::kHalf ? CLQ_F16 : CLQ_BF16;
  const void* x = X.data_ptr();
  const int32_t* perm = static_cast<const int32_t*>(THPVariable_Unpack(args[1]).data_ptr());
  const uint8_t* w = static_cast<const uint8_t*>(We.data_ptr());
  const float* s_w = static_cast<const float*>(THPVariable_Unpack(args[3]).data_ptr());
  const void* bias = has_bias ? THPVariable_Unpack(args[4]).data_ptr() : nullptr;
  void* y = Y.data_ptr();
  long where = 0;
  clq_status st;
  Py_BEGIN_ALLOW_THREADS
  st = clq_rotate_quant_act(x, cdt, static_cast<int32_t>(M), static_cast<int32_t>(K),
                            static_cast<int32_t>(ld), perm, static_cast<int32_t>(b),
                            static_cast<clq_codes>(a_codes), Xq, s_x, nullptr, stream);
  if (st == CLQ_OK) {
    where = 1;
    st = clq_linear(Xq, static_cast<clq_codes>(a_codes), s_x, w, w_codes, s_w, bias,
                    static_cast<int32_t>(M), static_cast<int32_t>(N), static_cast<int32_t>(K),
                    static_cast<int32_t>(b), cdt, y, nullptr, stream);
  }
  Py_END_ALLOW_THREADS
  if (st != CLQ_OK) return PyLong_FromLong(st | (where << 8));
  return THPVariable_Wrap(Y);
  END_HANDLE_TH_ERRORS
}

// --------------------------------------------------------- microscaled ---
// Arguments of a call; `plain` falls when one is not of the expected kind.
struct Args {
  PyObject* const* v;
  bool plain = true;
  const at::Tensor* tensor(int i) {
    if (THPVariable_Check(v[i])) return &THPVariable_Unpack(v[i]);
    plain = false;
    return nullptr;
  }
  const at::Tensor* maybe(int i) { return v[i] == Py_None ? nullptr : tensor(i); }
  long num(int i) {
    const long x = PyLong_AsLong(v[i]);
    if (x == -1 && PyErr_Occurred()) {
      PyErr_Clear();
      plain = false;
    }
    return x;
  }
};

template <typename T>
T* data(const at::Tensor* t) {
  return t == nullptr ? nullptr : static_cast<T*>(t->data_ptr());
}

bool rows16(const at::Tensor* t) {
  return t != nullptr && t->is_cuda() && t->dim() == 2 && t->stride(1) == 1 &&
         (t->scalar_type() == at::kHalf || t->scalar_type() == at::kBFloat16) &&
         t->size(0) <= INT32_MAX && t->stride(0) <= INT32_MAX;
}
clq_dtype dtype_of(const at::Tensor& t) {
  return t.scalar_type() == at::kHalf ? CLQ_F16 : CLQ_BF16;
}
bool dense(const at::Tensor* t, at::ScalarType type, int64_t numel, const at::Tensor& like) {
  return t == nullptr || (t->scalar_type() == type && t->numel() == numel && t->is_contiguous() &&
                          t->device() == like.device());
}
// Columns of an input that give K codes, or -1.
int64_t codes_of(int64_t columns, long act) {
  if (act != CLQ_MX_ACT_SWIGLU) return columns;
  return columns % 2 == 0 ? columns / 2 : -1;
}
PyObject* status_of(clq_status st, long where) { return PyLong_FromLong(st | (where << 8)); }
// The interpreter's lock is given up while the C calls run: a full launch queue blocks them.
struct Unlocked {
  PyThreadState* state = PyEval_SaveThread();
  ~Unlocked() { PyEval_RestoreThread(state); }
};
template <typename... P, typename... A>
clq_status unlocked(clq_status (*call)(P...), A... args) {
  const Unlocked u;
  return call(args...);
}
void* current_stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// mx_quantize(X, fmt, perm | None, b, act) -> (codes, scales, row_scale | None), None or a
// status.
PyObject* mx_quantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 5) Py_RETURN_NONE;
  Args a{args};
  const at::Tensor *X = a.tensor(0), *perm = a.maybe(2);
  const long fmt = a.num(1), b = a.num(3), act = a.num(4);
  if (!a.plain || act < 0 || !rows16(X)) Py_RETURN_NONE;
  const int64_t M = X->size(0), K = codes_of(X->size(1), act);
  if (K < 32 || K > 16384 || K % 32 != 0 || !dense(perm, at::kInt, K, *X)) Py_RETURN_NONE;
  const int64_t block = fmt == CLQ_MX_BLOCK16 ? 16 : 32;
  at::Tensor codes = at::empty({M, K / 2}, X->options().dtype(at::kByte));
  at::Tensor scales =
      at::empty({(M + 127) / 128, (K / block + 3) / 4, 32, 4, 4}, X->options().dtype(at::kByte));
  at::Tensor rows;
  if (fmt == CLQ_MX_BLOCK16) rows = at::empty({M}, X->options().dtype(at::kFloat));
  uint8_t *cq = codes.data_ptr<uint8_t>(), *cs = scales.data_ptr<uint8_t>();
  float* cr = fmt == CLQ_MX_BLOCK16 ? rows.data_ptr<float>() : nullptr;
  const clq_status st = unlocked(clq_mx_quantize,
      X->data_ptr(), dtype_of(*X), static_cast<int32_t>(M), static_cast<int32_t>(K),
      static_cast<int32_t>(X->stride(0)), data<int32_t>(perm), static_cast<int32_t>(b),
      static_cast<clq_mx_act>(act), static_cast<clq_mx_format>(fmt), cq, cs, cr, nullptr, 0, static_cast<int32_t>(M), current_stream());
  if (st != CLQ_OK) return status_of(st, 0);
  PyObject* r = PyTuple_New(3);
  PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(codes));
  PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(scales));
  if (fmt == CLQ_MX_BLOCK16) {
    PyTuple_SET_ITEM(r, 2, THPVariable_Wrap(rows));
  } else {
    Py_INCREF(Py_None);
    PyTuple_SET_ITEM(r, 2, Py_None);
  }
  return r;
  END_HANDLE_TH_ERRORS
}

// mx_dequantize(codes, scales, row_scale | None, fmt, dtype) -> values, or a status; the
// arrays of an MXTensor.
PyObject* mx_dequantize(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 5) Py_RETURN_NONE;
  Args a{args};
  const at::Tensor *codes = a.tensor(0), *scales = a.tensor(1), *rows = a.maybe(2);
  const long fmt = a.num(3), dtype = a.num(4);
  if (!a.plain || codes->dim() != 2 || !codes->is_cuda() || codes->size(0) > INT32_MAX)
    Py_RETURN_NONE;
  const int64_t M = codes->size(0), K = 2 * codes->size(1);
  at::Tensor out = at::empty(
      {M, K}, codes->options().dtype(dtype == CLQ_F16 ? at::kHalf : at::kBFloat16));
  const clq_status st = unlocked(clq_mx_dequantize, data<uint8_t>(codes), data<uint8_t>(scales), data<float>(rows), static_cast<int32_t>(M),
      static_cast<int32_t>(K), static_cast<clq_mx_format>(fmt), static_cast<clq_dtype>(dtype),
      out.data_ptr(), current_stream());
  if (st != CLQ_OK) return status_of(st, 0);
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

// Codes, scales and row scales of `rows` rows in one buffer.
struct Space {
  at::Tensor buffer;
  uint8_t *codes, *scales;
  float* row_scale;
  Space(int64_t rows, int64_t K, long fmt, const at::Tensor& like) {
    const int64_t c = (rows * (K / 2) + 255) / 256 * 256;
    const int64_t s = static_cast<int64_t>(clq_mx_scale_bytes(
        static_cast<int32_t>(rows), static_cast<int32_t>(K), static_cast<clq_mx_format>(fmt)));
    buffer = at::empty({c + s + (fmt == CLQ_MX_BLOCK16 ? 4 * rows : 0)},
                       like.options().dtype(at::kByte));
    codes = buffer.data_ptr<uint8_t>();
    scales = codes + c;
    row_scale = fmt == CLQ_MX_BLOCK16 ? reinterpret_cast<float*>(scales + s) : nullptr;
  }
};

// mx_layer(X, fmt, perm | None, b, act, codes, scales, row_scale | None, bias | None) -> Y
// [M, N], None or status | 256 * (0 quantize, 1 product); the arrays of the layer's MXTensor.
PyObject* mx_layer(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 9) Py_RETURN_NONE;
  Args a{args};
  const at::Tensor *X = a.tensor(0), *perm = a.maybe(2), *wq = a.tensor(5), *ws = a.tensor(6),
                   *wr = a.maybe(7), *bias = a.maybe(8);
  const long fmt = a.num(1), b = a.num(3), act = a.num(4);
  if (!a.plain || act < 0 || !rows16(X) || wq->dim() != 2 || wq->device() != X->device()) Py_RETURN_NONE;
  const int64_t M = X->size(0), K = codes_of(X->size(1), act), N = wq->size(0);
  if (K != 2 * wq->size(1) || !dense(perm, at::kInt, K, *X) ||
      !dense(bias, X->scalar_type(), N, *X) || M == 0)
    Py_RETURN_NONE;
  const Space q(M, K, fmt, *X);
  at::Tensor Y = at::empty({M, N}, X->options());
  void* stream = current_stream();
  const clq_dtype dt = dtype_of(*X);
  long where = 0;
  clq_status st = unlocked(clq_mx_quantize,
      X->data_ptr(), dt, static_cast<int32_t>(M), static_cast<int32_t>(K),
      static_cast<int32_t>(X->stride(0)), data<int32_t>(perm), static_cast<int32_t>(b),
      static_cast<clq_mx_act>(act), static_cast<clq_mx_format>(fmt), q.codes, q.scales, q.row_scale,
      nullptr, 0, static_cast<int32_t>(M), stream);
  if (st == CLQ_OK) {
    where = 1;
    st = unlocked(clq_mx_linear, q.codes, q.scales, q.row_scale, data<uint8_t>(wq), data<uint8_t>(ws),
                       data<float>(wr), data<void>(bias), static_cast<int32_t>(M),
                       static_cast<int32_t>(N), static_cast<int32_t>(K), static_cast<int32_t>(b),
                       static_cast<clq_mx_format>(fmt), dt, Y.data_ptr(), stream);
  }
  if (st != CLQ_OK) return status_of(st, where);
  return THPVariable_Wrap(Y);
  END_HANDLE_TH_ERRORS
}

// mx_route(logits, k, scoring, balance | None, groups, top_groups, group_top, renormalize,
// scale) -> (experts, weights), None or a status.
PyObject* mx_route(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 9) Py_RETURN_NONE;
  Args a{args};
  const at::Tensor *L = a.tensor(0), *balance = a.maybe(3);
  const long k = a.num(1), scoring = a.num(2), groups = a.num(4), top_groups = a.num(5),
             group_top = a.num(6), renormalize = a.num(7);
  const double scale = PyFloat_AsDouble(args[8]);
  if (PyErr_Occurred()) {
    PyErr_Clear();
    Py_RETURN_NONE;
  }
  if (!a.plain || !L->is_cuda() || L->dim() != 2 || L->stride(1) != 1 || k < 1 || k > 32 ||
      L->size(0) > INT32_MAX || L->stride(0) > INT32_MAX || !dense(balance, at::kFloat, L->size(1), *L))
    Py_RETURN_NONE;
  const at::ScalarType t = L->scalar_type();
  if (t != at::kFloat && t != at::kHalf && t != at::kBFloat16) Py_RETURN_NONE;
  const int64_t T = L->size(0);
  at::Tensor experts = at::empty({T, k}, L->options().dtype(at::kInt));
  at::Tensor weights = at::empty({T, k}, L->options().dtype(at::kFloat));
  const clq_status st = unlocked(clq_mx_route, L->data_ptr(), t == at::kFloat ? CLQ_F32 : dtype_of(*L), static_cast<int32_t>(T),
      static_cast<int32_t>(L->size(1)), static_cast<int32_t>(L->stride(0)), data<float>(balance),
      static_cast<int32_t>(k), static_cast<int32_t>(scoring), static_cast<int32_t>(groups),
      static_cast<int32_t>(top_groups), static_cast<int32_t>(group_top),
      static_cast<int32_t>(renormalize), static_cast<float>(scale), experts.data_ptr<int32_t>(),
      weights.data_ptr<float>(), current_stream());
  if (st != CLQ_OK) return status_of(st, 0);
  PyObject* r = PyTuple_New(2);
  PyTuple_SET_ITEM(r, 0, THPVariable_Wrap(experts));
  PyTuple_SET_ITEM(r, 1, THPVariable_Wrap(weights));
  return r;
  END_HANDLE_TH_ERRORS
}

// mx_experts(X, experts, weights, fmt, perm | None, b, act, codes1, scales1, row_scale1 |
// None, bias1 | None, codes2, scales2, row_scale2 | None, bias2 | None) -> out [T, N], None
// or status | 256 * step.
PyObject* mx_experts(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 15) Py_RETURN_NONE;
  Args a{args};
  const at::Tensor *X = a.tensor(0), *experts = a.tensor(1), *weights = a.tensor(2),
                   *perm = a.maybe(4), *q1 = a.tensor(7), *s1 = a.tensor(8), *r1 = a.maybe(9),
                   *bias1 = a.maybe(10), *q2 = a.tensor(11), *s2 = a.tensor(12), *r2 = a.maybe(13),
                   *bias2 = a.maybe(14);
  const long fmt = a.num(3), b = a.num(5), act = a.num(6);
  if (!a.plain || !rows16(X) || q1->dim() != 3 || q2->dim() != 3 || experts->dim() != 2 ||
      q1->device() != X->device() || q2->device() != X->device())
    Py_RETURN_NONE;
  const int32_t T = static_cast<int32_t>(X->size(0)), k = static_cast<int32_t>(experts->size(1));
  const int32_t E = static_cast<int32_t>(q1->size(0)), N1 = static_cast<int32_t>(q1->size(1));
  const int32_t K = static_cast<int32_t>(2 * q1->size(2)), F = static_cast<int32_t>(2 * q2->size(2));
  const int32_t N = static_cast<int32_t>(q2->size(1));
  if (T == 0 || X->size(1) != K || !dense(perm, at::kInt, K, *X) ||
      !dense(experts, at::kInt, static_cast<int64_t>(T) * k, *X) ||
      !dense(weights, at::kFloat, static_cast<int64_t>(T) * k, *X) ||
      !dense(bias1, X->scalar_type(), static_cast<int64_t>(E) * N1, *X) ||
      !dense(bias2, X->scalar_type(), static_cast<int64_t>(E) * N, *X))
    Py_RETURN_NONE;
  const size_t plan_bytes = clq_mx_plan_bytes(T, k, E);
  if (plan_bytes == 0) Py_RETURN_NONE;
  const int32_t R = clq_mx_plan_rows(T, k, E);
  const int64_t row_bytes = (static_cast<int64_t>(T) * k * 4 + 255) / 256 * 256;
  at::Tensor out = at::empty({T, N}, X->options());
  const at::Tensor plan = at::empty({static_cast<int64_t>(plan_bytes) + row_bytes},
                                    X->options().dtype(at::kByte));
  int32_t* rows = static_cast<int32_t*>(plan.data_ptr());
  void* space = plan.data_ptr<uint8_t>() + row_bytes;
  const Space x(R, K, fmt, *X), h(R, F, fmt, *X);
  const at::Tensor Y = at::empty({R, N}, X->options());
  const clq_mx_format f = static_cast<clq_mx_format>(fmt);
  const clq_dtype dt = dtype_of(*X);
  void* st = current_stream();
  clq_status r = unlocked(clq_mx_plan, data<int32_t>(experts), T, k, E, rows, space, plan_bytes, st);
  if (r != CLQ_OK) return status_of(r, 0);
  r = unlocked(clq_mx_quantize, X->data_ptr(), dt, T, K, static_cast<int32_t>(X->stride(0)),
                      data<int32_t>(perm), static_cast<int32_t>(b), CLQ_MX_ACT_NONE, f, x.codes,
                      x.scales, x.row_scale, rows, k, R, st);
  if (r != CLQ_OK) return status_of(r, 1);
  if (f == CLQ_MX_BLOCK32) {
    r = unlocked(clq_mx_grouped_linear_act, x.codes, x.scales, space, data<uint8_t>(q1),
                 data<uint8_t>(s1), data<void>(bias1), T, k, E, N1, K, static_cast<int32_t>(b), dt,
                 static_cast<clq_mx_act>(act), h.codes, h.scales, st);
    if (r != CLQ_OK) return status_of(r, 4);
  } else {  // a row's scale needs the whole row
    const at::Tensor H = at::empty({R, N1}, X->options());
    r = unlocked(clq_mx_grouped_linear, x.codes, x.scales, x.row_scale, space, data<uint8_t>(q1),
                 data<uint8_t>(s1), data<float>(r1), data<void>(bias1), T, k, E, N1, K,
                 static_cast<int32_t>(b), f, dt, H.data_ptr(), st);
    if (r != CLQ_OK) return status_of(r, 2);
    r = unlocked(clq_mx_quantize_rows, H.data_ptr(), dt, space, T, k, E, F, N1,
                 static_cast<clq_mx_act>(act), f, h.codes, h.scales, h.row_scale, st);
    if (r != CLQ_OK) return status_of(r, 5);
  }
  r = unlocked(clq_mx_grouped_linear, h.codes, h.scales, h.row_scale, space, data<uint8_t>(q2),
                            data<uint8_t>(s2), data<float>(r2), data<void>(bias2), T, k, E, N, F, 1,
                            f, dt, Y.data_ptr(), st);
  if (r != CLQ_OK) return status_of(r, 2);
  r = unlocked(clq_mx_combine, Y.data_ptr(), dt, rows, data<float>(weights), T, k, N, R, out.data_ptr(), st);
  if (r != CLQ_OK) return status_of(r, 3);
  return THPVariable_Wrap(out);
  END_HANDLE_TH_ERRORS
}

#define CLQ_METHOD(name, doc) \
  {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, doc}

PyMethodDef methods[] = {
    {"layer", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(layer)), METH_FASTCALL,
     "Rotate-quant and product of one prepared layer."},
    CLQ_METHOD(mx_quantize, "Rows to codes and scales."),
    CLQ_METHOD(mx_dequantize, "Codes and scales to values."),
    CLQ_METHOD(mx_layer, "Quantization and product of one microscaled layer."),
    CLQ_METHOD(mx_route, "Routing of tokens to experts."),
    CLQ_METHOD(mx_experts, "A feed-forward of experts."),
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_clq_host", nullptr, -1, methods,
                      nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__clq_host(void) { return PyModule_Create(&module); }
