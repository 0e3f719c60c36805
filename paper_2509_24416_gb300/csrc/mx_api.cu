// C ABI of the microscaled operators (declared in include/clq_mx.h): argument checks
// and launches.  Nothing here allocates device memory or synchronizes.
#include <cmath>
#include <cstdint>

#include <cuda_runtime.h>

#include "mx_kernels.h"
#include "overlap.h"

namespace {

using namespace clq;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
bool valid_dtype(int d) { return d == CLQ_F16 || d == CLQ_BF16; }
bool valid_format4(int f) { return f == CLQ_MX_BLOCK32 || f == CLQ_MX_BLOCK16; }
bool valid_format(int f) { return valid_format4(f) || f == CLQ_MX_BLOCK32_E4M3; }
bool valid_act(int a) { return a >= CLQ_MX_ACT_NONE && a <= CLQ_MX_ACT_SWIGLU; }
// Rows of an output that meet other rows (or other places) of an input than their own.
bool rows_overlap(const void* out, int64_t ld_out, const void* in, int64_t ld_in, int64_t rows, int64_t columns) {
  return overlaps(out, {ld_out, 0}, in, {ld_in, 0}, {rows, 1}, columns);
}
constexpr int kMaxRows = (1 << 30) - 1;  // row indices and a grid's step beyond them fit an int
bool valid_k(int K) { return K >= 32 && K <= 16384 && K % 32 == 0; }
bool valid_b(int b, int K) { return b >= 1 && b <= 256 && (b & (b - 1)) == 0 && K % b == 0; }
clq_status from_cuda(cudaError_t e) { return e == cudaSuccess ? CLQ_OK : CLQ_ERR_CUDA; }

// Checks of a code array; a null scale a row only where the format has none.
clq_status check_codes(const uint8_t* q, const uint8_t* s, const float* rows, int fmt,
                       int row_align) {
  if (q == nullptr || s == nullptr || (fmt == CLQ_MX_BLOCK16 && rows == nullptr))
    return CLQ_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(s, 16) || (rows != nullptr && !aligned(rows, row_align)))
    return CLQ_ERR_ALIGN;
  return CLQ_OK;
}

bool valid_routing(int T, int k, int E) {
  return T >= 0 && E >= 1 && E <= 512 && k >= 1 && k <= 32 && k <= E &&
         static_cast<int64_t>(T) * k + 128ll * E <= kMaxRows;
}

// The experts' products, their output in Y or, behind `act`, as codes in Yq / Ys.
clq_status grouped(const uint8_t* Xq, const uint8_t* Xs, const float* s_x, const void* plan,
                   const uint8_t* Wq, const uint8_t* Ws, const float* s_w, const void* bias, int T,
                   int k, int E, int N, int K, int b, int fmt, int dtype, void* Y, int act,
                   uint8_t* Yq, uint8_t* Ys, void* stream) {
  if (!valid_dtype(dtype) || !valid_format4(fmt) || N < 0) return CLQ_ERR_INVALID_ARG;
  if (!valid_k(K) || !valid_b(b, K) || !valid_routing(T, k, E) ||
      static_cast<int64_t>(E) * N >= (1ll << 31))
    return CLQ_ERR_SHAPE;
  if (T == 0 || N == 0) return CLQ_OK;
  if ((Y == nullptr && Yq == nullptr) || plan == nullptr) return CLQ_ERR_INVALID_ARG;
  if (!aligned(Y, 16) || !aligned(plan, 16) || (bias != nullptr && !aligned(bias, 2)))
    return CLQ_ERR_ALIGN;
  clq_status st = check_codes(Xq, Xs, s_x, fmt, 4);
  if (st == CLQ_OK) st = check_codes(Wq, Ws, s_w, fmt, 4);
  if (st != CLQ_OK) return st;
  mx::GemmArgs g{};
  if ((st = device_status(&g.status)) != CLQ_OK) return st;
  const mx::PlanLayout pl = mx::plan_layout(T, k, E);
  g.s_x = s_x;
  g.s_w = s_w;
  g.bias = bias;
  g.Y = Y;
  g.Yq = Yq;
  g.Ys = Ys;
  g.act = act;
  if (Yq != nullptr)
    g.y_chunks = mx::scale_chunks(act == CLQ_MX_ACT_SWIGLU ? N / 2 : N, CLQ_MX_BLOCK32);
  g.x_rows = mx::plan_rows(T, k, E);
  g.M = g.x_rows;
  g.N = N;
  g.K = K;
  g.inv_b = 1.0f / static_cast<float>(b);
  g.chunks = mx::scale_chunks(K, fmt);
  g.w_blocks = (N + mx::kRowBlock - 1) / mx::kRowBlock;
  g.experts = E;
  return from_cuda(mx::launch_gemm(Xq, Xs, Wq, Ws, g, fmt, dtype, plan, &pl, T, k,
                                   static_cast<cudaStream_t>(stream)));
}

// The product of two code arrays, with an activation and a residual behind it if `post`.
clq_status dense(const uint8_t* Xq, const uint8_t* Xs, const float* s_x, const uint8_t* Wq,
                 const uint8_t* Ws, const float* s_w, const void* bias, int32_t M, int32_t N,
                 int32_t K, int32_t b, int fmt, int dtype, bool post, int act, const void* residual,
                 int32_t ldr, void* Y, void* stream) {
  if (!valid_dtype(dtype) || !valid_format(fmt) || M < 0 || N < 0) return CLQ_ERR_INVALID_ARG;
  if (!valid_k(K) || !valid_b(b, K) || M > kMaxRows || N > kMaxRows) return CLQ_ERR_SHAPE;
  if (M == 0 || N == 0) return CLQ_OK;
  if (Y == nullptr) return CLQ_ERR_INVALID_ARG;
  if (!aligned(Y, 16) || (bias != nullptr && !aligned(bias, 2))) return CLQ_ERR_ALIGN;
  clq_status st = check_codes(Xq, Xs, s_x, fmt, 4);
  if (st == CLQ_OK) st = check_codes(Wq, Ws, s_w, fmt, 4);
  if (st != CLQ_OK) return st;
  mx::GemmArgs g{};
  if ((st = device_status(&g.status)) != CLQ_OK) return st;
  g.s_x = s_x;
  g.s_w = s_w;
  g.bias = bias;
  g.Y = Y;
  g.M = M;
  g.N = N;
  g.K = K;
  g.inv_b = 1.0f / static_cast<float>(b);
  g.chunks = mx::scale_chunks(K, fmt);
  g.w_blocks = (N + mx::kRowBlock - 1) / mx::kRowBlock;
  g.experts = 1;
  g.x_rows = M;
  g.post = post;
  g.act = act;
  g.residual = residual;
  g.ldr = ldr;
  return from_cuda(mx::launch_gemm(Xq, Xs, Wq, Ws, g, fmt, dtype, nullptr, nullptr, M, 1,
                                   static_cast<cudaStream_t>(stream)));
}

}  // namespace

extern "C" {

size_t clq_mx_scale_bytes(int32_t rows, int32_t K, clq_mx_format fmt) {
  if (rows < 0 || !valid_k(K) || !valid_format(fmt)) return 0;
  return (static_cast<size_t>(rows) + 127) / 128 * mx::scale_chunks(K, fmt) * 512;
}

clq_status clq_mx_quantize(const void* X, clq_dtype dtype, int32_t M, int32_t K, int32_t ldx,
                           const int32_t* perm, int32_t b, clq_mx_act act, clq_mx_format fmt,
                           uint8_t* codes, uint8_t* scales, float* row_scale,
                           const int32_t* out_rows, int32_t k, int32_t rows, void* stream) {
  if (!valid_dtype(dtype) || !valid_format(fmt) || act < CLQ_MX_ACT_NONE ||
      act > CLQ_MX_ACT_SWIGLU || M < 0 || rows < 0 || (out_rows != nullptr && k < 1))
    return CLQ_ERR_INVALID_ARG;
  const int64_t width = act == CLQ_MX_ACT_SWIGLU ? 2ll * K : K;
  if (!valid_k(K) || !valid_b(b, K) || ldx < width || M > kMaxRows) return CLQ_ERR_SHAPE;
  if (out_rows == nullptr && rows < M) return CLQ_ERR_SHAPE;
  if (ldx % 8 != 0) return CLQ_ERR_ALIGN;
  if (M == 0) return CLQ_OK;
  if (X == nullptr) return CLQ_ERR_INVALID_ARG;
  if (!aligned(X, 16) || (perm != nullptr && !aligned(perm, 4)) ||
      (out_rows != nullptr && !aligned(out_rows, 4)))
    return CLQ_ERR_ALIGN;
  clq_status st = check_codes(codes, scales, row_scale, fmt, 4);
  if (st != CLQ_OK) return st;
  mx::QuantArgs a{};
  if ((st = device_status(&a.status)) != CLQ_OK) return st;
  a.X = X;
  a.M = M;
  a.K = K;
  a.ld = ldx;
  a.perm = perm;
  a.b = b;
  a.act = act;
  a.codes = codes;
  a.scales = scales;
  a.row_scale = row_scale;
  a.out_rows = out_rows;
  a.k = k;
  a.rows = rows;
  return from_cuda(mx::launch_quantize(a, dtype, fmt, static_cast<cudaStream_t>(stream)));
}

clq_status clq_mx_dequantize(const uint8_t* codes, const uint8_t* scales, const float* row_scale,
                             int32_t M, int32_t K, clq_mx_format fmt, clq_dtype dtype, void* out,
                             void* stream) {
  if (!valid_dtype(dtype) || !valid_format(fmt) || M < 0) return CLQ_ERR_INVALID_ARG;
  if (!valid_k(K) || M > kMaxRows) return CLQ_ERR_SHAPE;
  if (M == 0) return CLQ_OK;
  if (out == nullptr) return CLQ_ERR_INVALID_ARG;
  if (!aligned(out, 16)) return CLQ_ERR_ALIGN;
  clq_status st = check_codes(codes, scales, row_scale, fmt, 4);
  if (st != CLQ_OK) return st;
  int32_t* status = nullptr;
  if ((st = device_status(&status)) != CLQ_OK) return st;
  return from_cuda(mx::launch_dequantize(codes, scales, row_scale, M, K, fmt, dtype, out,
                                         static_cast<cudaStream_t>(stream)));
}

clq_status clq_mx_linear(const uint8_t* Xq, const uint8_t* Xs, const float* s_x,
                         const uint8_t* Wq, const uint8_t* Ws, const float* s_w, const void* bias,
                         int32_t M, int32_t N, int32_t K, int32_t b, clq_mx_format fmt,
                         clq_dtype dtype, void* Y, void* stream) {
  return dense(Xq, Xs, s_x, Wq, Ws, s_w, bias, M, N, K, b, fmt, dtype, false, CLQ_MX_ACT_NONE,
               nullptr, 0, Y, stream);
}

clq_status clq_mx_linear_post(const uint8_t* Xq, const uint8_t* Xs, const float* s_x,
                              const uint8_t* Wq, const uint8_t* Ws, const float* s_w,
                              const void* bias, int32_t M, int32_t N, int32_t K, int32_t b,
                              clq_mx_format fmt, clq_dtype dtype, clq_mx_act act,
                              const void* residual, int32_t ldr, void* Y, void* stream) {
  if (!valid_act(act)) return CLQ_ERR_INVALID_ARG;
  const bool gated = act == CLQ_MX_ACT_SWIGLU;
  if (gated && N > 0 && N % 16 != 0) return CLQ_ERR_SHAPE;
  if (residual != nullptr && ldr < (gated ? N / 2 : N)) return CLQ_ERR_SHAPE;
  if (!aligned(residual, 2)) return CLQ_ERR_ALIGN;
  if (residual != nullptr && residual == Y && M > 1 && ldr != (gated ? N / 2 : N)) return CLQ_ERR_INVALID_ARG;
  if (residual != nullptr && Y != nullptr && aligned(Y, 2) && rows_overlap(Y, gated ? N / 2 : N, residual, ldr, M, gated ? N / 2 : N))
    return CLQ_ERR_INVALID_ARG;
  return dense(Xq, Xs, s_x, Wq, Ws, s_w, bias, M, N, K, b, fmt, dtype,
               act != CLQ_MX_ACT_NONE || residual != nullptr, act, residual, ldr, Y, stream);
}

clq_status clq_mx_rms_norm(const void* X, clq_dtype dtype, int32_t M, int32_t K, int32_t ldx,
                           const void* residual, int32_t ldr, const void* weight, float eps,
                           const int32_t* perm, int32_t b, clq_mx_format fmt, uint8_t* codes,
                           uint8_t* scales, float* row_scale, void* sum, int32_t lds,
                           void* stream) {
  // (squares below fp32's normal numbers have lost digits, which only a normal eps outweighs)
  if (!valid_dtype(dtype) || !valid_format(fmt) || M < 0 || !(eps >= 0x1p-126f) || std::isinf(eps) ||
      (residual == nullptr) != (sum == nullptr))
    return CLQ_ERR_INVALID_ARG;
  const bool both = residual != nullptr;
  if (!valid_k(K) || !valid_b(b, K) || M > kMaxRows || ldx < K || (both && (ldr < K || lds < K)))
    return CLQ_ERR_SHAPE;
  if (ldx % 8 != 0 || (both && (ldr % 8 != 0 || lds % 8 != 0))) return CLQ_ERR_ALIGN;
  if (M == 0) return CLQ_OK;
  if (X == nullptr) return CLQ_ERR_INVALID_ARG;
  if (both && M > 1 && ((sum == X && lds != ldx) || (sum == residual && lds != ldr))) return CLQ_ERR_INVALID_ARG;
  if (!aligned(X, 16) || !aligned(residual, 16) || !aligned(sum, 16) || !aligned(weight, 16) ||
      !aligned(perm, 4))
    return CLQ_ERR_ALIGN;
  if (both && (rows_overlap(sum, lds, X, ldx, M, K) || rows_overlap(sum, lds, residual, ldr, M, K)))
    return CLQ_ERR_INVALID_ARG;
  clq_status st = check_codes(codes, scales, row_scale, fmt, 4);
  if (st != CLQ_OK) return st;
  mx::NormArgs a{};
  if ((st = device_status(&a.status)) != CLQ_OK) return st;
  a.X = X;
  a.residual = residual;
  a.weight = weight;
  a.sum = sum;
  a.M = M;
  a.K = K;
  a.ldx = ldx;
  a.ldr = ldr;
  a.lds = lds;
  a.eps = eps;
  a.inv_k = static_cast<float>(1.0 / K);
  a.inv_k_low = static_cast<float>(1.0 / K - a.inv_k);
  a.perm = perm;
  a.b = b;
  a.codes = codes;
  a.scales = scales;
  a.row_scale = row_scale;
  return from_cuda(mx::launch_norm(a, dtype, fmt, static_cast<cudaStream_t>(stream)));
}

clq_status clq_mx_route(const void* logits, int32_t dtype, int32_t T, int32_t E, int32_t ld,
                        const float* balance, int32_t k, int32_t scoring, int32_t groups,
                        int32_t top_groups, int32_t group_top, int32_t renormalize, float scale,
                        int32_t* experts, float* weights, void* stream) {
  if (!(valid_dtype(dtype) || dtype == CLQ_F32) || T < 0 || scoring < 0 || scoring > 1 ||
      group_top < 1 || group_top > 2 || !std::isfinite(scale))
    return CLQ_ERR_INVALID_ARG;
  if (!valid_routing(T, k, E) || ld < E || groups < 1 || groups > 32 || E % groups != 0 ||
      top_groups < 1 || top_groups > groups)
    return CLQ_ERR_SHAPE;
  if (T == 0) return CLQ_OK;
  if (logits == nullptr || experts == nullptr || weights == nullptr) return CLQ_ERR_INVALID_ARG;
  if (!aligned(logits, dtype == CLQ_F32 ? 4 : 2) || !aligned(experts, 4) || !aligned(weights, 4) ||
      (balance != nullptr && !aligned(balance, 4)))
    return CLQ_ERR_ALIGN;
  int32_t* status = nullptr;
  const clq_status st = device_status(&status);
  if (st != CLQ_OK) return st;
  mx::RouteArgs a{};
  a.logits = logits;
  a.balance = balance;
  a.experts = experts;
  a.weights = weights;
  a.T = T;
  a.E = E;
  a.ld = ld;
  a.k = k;
  a.scoring = scoring;
  a.groups = groups;
  a.top_groups = top_groups;
  a.group_top = group_top;
  a.renormalize = renormalize;
  a.scale = scale;
  return from_cuda(mx::launch_route(a, dtype, static_cast<cudaStream_t>(stream)));
}

int32_t clq_mx_plan_rows(int32_t T, int32_t k, int32_t E) {
  return valid_routing(T, k, E) ? mx::plan_rows(T, k, E) : 0;
}

size_t clq_mx_plan_bytes(int32_t T, int32_t k, int32_t E) {
  return valid_routing(T, k, E) ? mx::plan_layout(T, k, E).bytes : 0;
}

clq_status clq_mx_plan(const int32_t* experts, int32_t T, int32_t k, int32_t E, int32_t* out_rows,
                       void* plan, size_t plan_bytes, void* stream) {
  if (!valid_routing(T, k, E)) return CLQ_ERR_SHAPE;
  if (T == 0) return CLQ_OK;
  if (experts == nullptr || out_rows == nullptr || plan == nullptr) return CLQ_ERR_INVALID_ARG;
  if (!aligned(experts, 4) || !aligned(out_rows, 4) || !aligned(plan, 16)) return CLQ_ERR_ALIGN;
  const mx::PlanLayout pl = mx::plan_layout(T, k, E);
  if (plan_bytes < pl.bytes) return CLQ_ERR_SHAPE;
  int32_t* status = nullptr;
  const clq_status st = device_status(&status);
  if (st != CLQ_OK) return st;
  return from_cuda(mx::launch_plan(experts, T, k, E, out_rows, plan, pl,
                                   static_cast<cudaStream_t>(stream)));
}

clq_status clq_mx_grouped_linear(const uint8_t* Xq, const uint8_t* Xs, const float* s_x,
                                 const void* plan, const uint8_t* Wq, const uint8_t* Ws,
                                 const float* s_w, const void* bias, int32_t T, int32_t k,
                                 int32_t E, int32_t N, int32_t K, int32_t b, clq_mx_format fmt,
                                 clq_dtype dtype, void* Y, void* stream) {
  return grouped(Xq, Xs, s_x, plan, Wq, Ws, s_w, bias, T, k, E, N, K, b, fmt, dtype, Y,
                 CLQ_MX_ACT_NONE, nullptr, nullptr, stream);
}

clq_status clq_mx_grouped_linear_act(const uint8_t* Xq, const uint8_t* Xs, const void* plan,
                                     const uint8_t* Wq, const uint8_t* Ws, const void* bias,
                                     int32_t T, int32_t k, int32_t E, int32_t N, int32_t K,
                                     int32_t b, clq_dtype dtype, clq_mx_act act, uint8_t* Yq,
                                     uint8_t* Ys, void* stream) {
  if (act < CLQ_MX_ACT_NONE || act > CLQ_MX_ACT_SWIGLU) return CLQ_ERR_INVALID_ARG;
  const bool gated = act == CLQ_MX_ACT_SWIGLU;
  if (N > 0 && (N % (gated ? 64 : 32) != 0 || !valid_k(gated ? N / 2 : N))) return CLQ_ERR_SHAPE;
  if (T > 0 && N > 0 && (Yq == nullptr || Ys == nullptr)) return CLQ_ERR_INVALID_ARG;
  if (!aligned(Yq, 16) || !aligned(Ys, 16)) return CLQ_ERR_ALIGN;
  return grouped(Xq, Xs, nullptr, plan, Wq, Ws, nullptr, bias, T, k, E, N, K, b, CLQ_MX_BLOCK32,
                 dtype, nullptr, act, Yq, Ys, stream);
}

clq_status clq_mx_quantize_rows(const void* X, clq_dtype dtype, const void* plan, int32_t T,
                                int32_t k, int32_t E, int32_t K, int32_t ldx, clq_mx_act act,
                                clq_mx_format fmt, uint8_t* codes, uint8_t* scales,
                                float* row_scale, void* stream) {
  if (!valid_dtype(dtype) || !valid_format4(fmt) || act < CLQ_MX_ACT_NONE || act > CLQ_MX_ACT_SWIGLU)
    return CLQ_ERR_INVALID_ARG;
  if (!valid_k(K) || !valid_routing(T, k, E) || ldx < (act == CLQ_MX_ACT_SWIGLU ? 2ll * K : K))
    return CLQ_ERR_SHAPE;
  if (ldx % 8 != 0) return CLQ_ERR_ALIGN;
  if (T == 0) return CLQ_OK;
  if (X == nullptr || plan == nullptr) return CLQ_ERR_INVALID_ARG;
  if (!aligned(X, 16) || !aligned(plan, 16)) return CLQ_ERR_ALIGN;
  clq_status st = check_codes(codes, scales, row_scale, fmt, 4);
  if (st != CLQ_OK) return st;
  mx::QuantArgs a{};
  if ((st = device_status(&a.status)) != CLQ_OK) return st;
  const mx::PlanLayout pl = mx::plan_layout(T, k, E);
  const uint8_t* p = static_cast<const uint8_t*>(plan);
  a.X = X;
  a.M = a.rows = mx::plan_rows(T, k, E);
  a.K = K;
  a.ld = ldx;
  a.b = 1;
  a.act = act;
  a.codes = codes;
  a.scales = scales;
  a.row_scale = row_scale;
  a.tiles = reinterpret_cast<const mx::RowTile*>(p + pl.tiles128_off);
  a.tile_count = reinterpret_cast<const int32_t*>(p + pl.counts_off);
  return from_cuda(mx::launch_quantize(a, dtype, fmt, static_cast<cudaStream_t>(stream)));
}

clq_status clq_mx_combine(const void* Y, clq_dtype dtype, const int32_t* rows,
                          const float* weights, int32_t T, int32_t k, int32_t D, int32_t R,
                          void* out, void* stream) {
  if (!valid_dtype(dtype) || T < 0 || k < 1 || R < 0) return CLQ_ERR_INVALID_ARG;
  if (D < 8 || D % 8 != 0 || D > (1 << 24) || T > kMaxRows || k > kMaxRows) return CLQ_ERR_SHAPE;
  if (T == 0) return CLQ_OK;
  if (Y == nullptr || rows == nullptr || weights == nullptr || out == nullptr)
    return CLQ_ERR_INVALID_ARG;
  if (!aligned(Y, 16) || !aligned(out, 16) || !aligned(rows, 4) || !aligned(weights, 4))
    return CLQ_ERR_ALIGN;
  int32_t* status = nullptr;
  const clq_status st = device_status(&status);
  if (st != CLQ_OK) return st;
  return from_cuda(mx::launch_combine(Y, dtype, rows, weights, T, k, D, R, out, status,
                                      static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
