// Rotary positions over several axes: the kernel and its C entry (include/clq_rope.h).
//
// out = x turned by pos f, pair by pair: 2 bytes in and 2 out a value for 3 operations, bound by
// memory as long as what a thread does before its first head (positions, angles, sines and
// cosines of its pairs, which the heads of a token share) is spread over enough heads.  Measured,
// us: 16384 tokens of 48 heads of 128 values 60 interleaved (6.7 TB/s), 66 as halves; 8192 of 32 of
// 72 10.3 and 13 to 16; 65536 of 2 of 128 12.7 and 14.7; one token of 40 heads 1.9.  Two heads
// ahead as halves 71 for 66, three blocks a SM (68 registers) 79; a thread of 16 neighbouring
// values instead of eight 71 for 60; sines by sincospif and a 64-bit division a thread 74 as
// halves.
#include <algorithm>
#include <cstdint>

#include <cuda_runtime.h>

#include "../../include/clq_rope.h"
#include "clq_device.cuh"
#include "clq_kernels.h"
#include "overlap.h"

namespace clq {
namespace rope {
namespace {

constexpr int MAX_AXES = 4;
constexpr int HEADS = 8;  // of a thread, where there are many
constexpr int THREADS = 256;

struct Args {
  const uint16_t* x;
  uint16_t* out;
  const int32_t* positions;
  const uint64_t* turns;
  int64_t xt, xh, ot, oh;  // strides of tokens and heads
  int32_t T, H, D, P, ld, axes;
  int32_t first[MAX_AXES];  // pair behind the last one of each axis
  int32_t inverse;
  int32_t units;  // threads of a head
  int32_t split;  // of them in a block
  int32_t group;  // threads that share the heads of a token, each taking every group-th
};

// V values in one load, as words of two.
template <int V>
struct Values {
  uint32_t w[V > 1 ? V / 2 : 1];
  __device__ __forceinline__ void load(const uint16_t* p) {
    if constexpr (V == 8) {
      const uint4 r = *reinterpret_cast<const uint4*>(p);
      w[0] = r.x, w[1] = r.y, w[2] = r.z, w[3] = r.w;
    } else if constexpr (V == 4) {
      const uint2 r = *reinterpret_cast<const uint2*>(p);
      w[0] = r.x, w[1] = r.y;
    } else if constexpr (V == 2) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *p;
    }
  }
  __device__ __forceinline__ void store(uint16_t* p) const {
    if constexpr (V == 8)
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (V == 4)
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else if constexpr (V == 2)
      *reinterpret_cast<uint32_t*>(p) = w[0];
    else
      *p = static_cast<uint16_t>(w[0]);
  }
};

template <typename T>
__device__ __forceinline__ float2 two(uint32_t w) {
  return make_float2(Num<T>::to_f(static_cast<uint16_t>(w)), Num<T>::to_f(static_cast<uint16_t>(w >> 16)));
}
__device__ __forceinline__ uint32_t halves_of(bool lo, bool hi, uint32_t a, uint32_t b) {
  return (lo ? a & 0xFFFFu : b & 0xFFFFu) | (hi ? a & 0xFFFF0000u : b & 0xFFFF0000u);
}

// A thread's part of a head, its unit.  HALVES: vectors i .. and P + i .. of V values, V pairs;
// else one vector of neighbours, V / 2 pairs (V = 1: two single values).  Units behind the pairs
// hold values that stay.  A block has blockDim.y tokens, blockDim.x threads of one (units first).
// AHEAD: heads whose loads are under way together.
template <typename T, int V, bool HALVES, int AHEAD>
__global__ void __launch_bounds__(THREADS, HALVES ? 5 : 4) rope_kernel(Args a) {
  constexpr bool TWO = HALVES || V == 1;  // vectors of a unit
  constexpr int PAIRS = TWO ? V : V / 2;
  pdl_wait();
  pdl_launch_dependents();
  const int token = blockIdx.x * blockDim.y + threadIdx.y;
  const int lead = blockIdx.y * (blockDim.x / a.split) + threadIdx.x / a.split;
  const int unit = blockIdx.z * a.split + threadIdx.x % a.split;
  if (token >= a.T || lead >= a.group || unit >= a.units) return;
  int at0 = unit * (TWO ? 2 * V : V), at1 = at0 + V, p0 = unit * PAIRS;
  if (HALVES) {
    const int pair_units = a.P / V;
    if (unit < pair_units) {
      at0 = unit * V;
      at1 = a.P + at0;
    } else {
      at0 = 2 * a.P + (unit - pair_units) * 2 * V;
      at1 = at0 + V;
      p0 = a.P;
    }
  }
  const bool second = TWO && at1 < a.D;  // (a head's last unit may have one vector only)
  const uint16_t* x = a.x + token * a.xt + lead * a.xh;
  uint16_t* out = a.out + token * a.ot + lead * a.oh;
  const int64_t xs = a.group * a.xh, os = a.group * a.oh;
  Values<V> u[AHEAD], w[TWO ? AHEAD : 1];
  auto load = [&](int h0) {
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      if (h0 + q * a.group < a.H) {
        u[q].load(x + q * xs + at0);
        if (second) w[TWO ? q : 0].load(x + q * xs + at1);
      }
    }
  };
  load(lead);
  float c[PAIRS], s[PAIRS];
  const int32_t* positions = a.positions + static_cast<int64_t>(token) * a.ld;
#pragma unroll
  for (int k = 0; k < PAIRS; ++k) {
    c[k] = 1.f;
    s[k] = 0.f;
    const int p = p0 + k;
    if (p < a.P) {
      int axis = 0;
#pragma unroll
      for (int m = 0; m < MAX_AXES - 1; ++m) axis += m + 1 < a.axes && p >= a.first[m] ? 1 : 0;
      const uint64_t turn =
          static_cast<uint64_t>(static_cast<int64_t>(__ldg(positions + axis))) * __ldg(a.turns + p);
      // in [-pi, pi), where the fast sine and cosine are within 2^-21
      __sincosf(static_cast<float>(static_cast<int32_t>(turn >> 32)) * (3.14159265f * 0x1p-31f), &s[k],
                &c[k]);
      if (a.inverse) s[k] = -s[k];
    }
  }
  const int turned = a.P - p0;  // of this unit's pairs; the others' values stay bit by bit
  for (int h0 = lead; h0 < a.H; h0 += AHEAD * a.group) {
    if (h0 != lead) load(h0);
#pragma unroll
    for (int q = 0; q < AHEAD; ++q) {
      if (h0 + q * a.group >= a.H) break;
      Values<V>&f = u[q], &g = w[TWO ? q : 0];
      if constexpr (TWO) {
#pragma unroll
        for (int k = 0; k < V; k += 2) {
          const float2 c2 = make_float2(c[k], V > 1 ? c[(k + 1) % V] : 1.f);
          const float2 s2 = make_float2(s[k], V > 1 ? s[(k + 1) % V] : 0.f);
          const float2 v0 = two<T>(f.w[k / 2]), v1 = two<T>(g.w[k / 2]);
          const float2 y0 = __ffma2_rn(v0, c2, __fmul2_rn(v1, make_float2(-s2.x, -s2.y)));
          const float2 y1 = __ffma2_rn(v1, c2, __fmul2_rn(v0, s2));
          const bool lo = k < turned, hi = V > 1 && k + 1 < turned;
          f.w[k / 2] = halves_of(lo, hi, Num<T>::pack2(y0.x, y0.y), f.w[k / 2]);
          g.w[k / 2] = halves_of(lo, hi, Num<T>::pack2(y1.x, y1.y), g.w[k / 2]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < PAIRS; ++k) {
          const float2 v = two<T>(f.w[k]);
          const float2 y = __ffma2_rn(v, make_float2(c[k], c[k]),
                                      __fmul2_rn(make_float2(v.y, v.x), make_float2(-s[k], s[k])));
          if (k < turned) f.w[k] = Num<T>::pack2(y.x, y.y);
        }
      }
      f.store(out + q * os + at0);
      if (second) g.store(out + q * os + at1);
    }
    x += AHEAD * xs;
    out += AHEAD * os;
  }
}

template <typename T, bool HALVES, int AHEAD>
auto pick(int V) {
  return V == 8   ? rope_kernel<T, 8, HALVES, AHEAD>
         : V == 4 ? rope_kernel<T, 4, HALVES, AHEAD>
         : V == 2 ? rope_kernel<T, 2, HALVES, AHEAD>
                  : rope_kernel<T, 1, HALVES, AHEAD>;
}

template <typename T>
cudaError_t launch(int V, bool halves, const Args& a, dim3 grid, dim3 block, cudaStream_t st) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  void (*k)(Args) = halves                ? pick<T, true, 1>(V)
                    : a.H > 2 * a.group ? pick<T, false, 4>(V)
                                        : pick<T, false, 2>(V);
  return cudaLaunchKernelEx(&cfg, k, a);
}

// Heads of D values that may share places: as dimensions one inside the other they do not.
bool overlap(int T, int H, int D, int64_t token_stride, int64_t head_stride) {
  if (T <= 1) return H > 1 && head_stride < D;
  if (H <= 1) return token_stride < D;
  const bool heads_inside = head_stride <= token_stride;
  const int64_t in = heads_inside ? head_stride : token_stride, n = heads_inside ? H : T;
  return in < D || std::max(head_stride, token_stride) < (n - 1) * in + D;
}

}  // namespace
}  // namespace rope
}  // namespace clq

extern "C" clq_status clq_rope(const void* x, clq_dtype dtype, int32_t T, int32_t H, int32_t D,
                            int64_t token_stride, int64_t head_stride, const int32_t* positions,
                            int32_t ld_positions, int32_t axes, const int32_t* host_sections,
                            const uint64_t* turns, clq_rope_pairs pairs, int32_t inverse, void* out,
                            int64_t out_token_stride, int64_t out_head_stride, void* stream) {
  using namespace clq;
  auto aligned = [](const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; };
  if ((dtype != CLQ_F16 && dtype != CLQ_BF16) || T < 0 || H < 0 || pairs < 0 || pairs > 1 ||
      axes < 1 || axes > rope::MAX_AXES || host_sections == nullptr)
    return CLQ_ERR_INVALID_ARG;
  rope::Args a{};
  int64_t P = 0;
  for (int i = 0; i < axes; ++i) {
    if (host_sections[i] < 0) return CLQ_ERR_INVALID_ARG;
    P += host_sections[i];
    a.first[i] = static_cast<int32_t>(std::min<int64_t>(P, 4096));
  }
  if (T >= (1 << 30) || D < 2 || D > 4096 || H > 65535 || P < 1 || 2 * P > D || token_stride < 0 || head_stride < 0 ||
      out_token_stride < 0 || out_head_stride < 0 || ld_positions < 0 ||
      rope::overlap(T, H, D, out_token_stride, out_head_stride))
    return CLQ_ERR_SHAPE;
  if (x != nullptr && x == out &&
      ((T > 1 && token_stride != out_token_stride) || (H > 1 && head_stride != out_head_stride)))
    return CLQ_ERR_INVALID_ARG;
  if (T == 0 || H == 0) return CLQ_OK;
  if (x == nullptr || out == nullptr || positions == nullptr || turns == nullptr)
    return CLQ_ERR_INVALID_ARG;
  if (!aligned(x, 2) || !aligned(out, 2) || !aligned(positions, 4) || !aligned(turns, 8))
    return CLQ_ERR_ALIGN;
  if (overlaps(out, {out_token_stride, out_head_stride}, x, {token_stride, head_stride}, {T, H}, D))
    return CLQ_ERR_INVALID_ARG;
  const clq_status st = device_check();
  if (st != CLQ_OK) return st;
  a.x = static_cast<const uint16_t*>(x);
  a.out = static_cast<uint16_t*>(out);
  a.positions = positions;
  a.turns = turns;
  a.xt = token_stride;
  a.xh = head_stride;
  a.ot = out_token_stride;
  a.oh = out_head_stride;
  a.T = T;
  a.H = H;
  a.D = D;
  a.P = static_cast<int32_t>(P);
  a.ld = ld_positions;
  a.axes = axes;
  a.inverse = inverse != 0;
  // The widest vector that addresses, strides and the head (its halves) allow.
  const bool halves = pairs == CLQ_ROPE_HALVES;
  int V = 8;
  auto fits = [&](int64_t n) { return n % V == 0; };
  while (V > 1 && !(aligned(x, 2 * V) && aligned(out, 2 * V) && fits(token_stride) && fits(head_stride) &&
                    fits(out_token_stride) && fits(out_head_stride) && fits(D) && (!halves || fits(P))))
    V /= 2;
  const int wide = halves || V == 1 ? 2 * V : V;  // values of a unit
  a.units = halves ? static_cast<int32_t>(P / V + (D - 2 * P + wide - 1) / wide) : (D + wide - 1) / wide;
  // A thread takes HEADS heads; fewer, down to one, where that leaves the GPU with idle lanes.
  const int sms = sm_count();
  if (sms <= 0) return CLQ_ERR_CUDA;
  const int64_t threads = static_cast<int64_t>(T) * a.units;
  a.group = static_cast<int32_t>(std::min<int64_t>(
      H, std::max<int64_t>((H + rope::HEADS - 1) / rope::HEADS, 2048ll * sms / threads)));
  a.split = std::min(a.units, rope::THREADS);
  const int x_heads = std::min(a.group, rope::THREADS / a.split);
  dim3 block(static_cast<unsigned>(a.split * x_heads)), grid;
  block.y = std::max(1u, rope::THREADS / block.x);
  grid.x = (static_cast<unsigned>(T) + block.y - 1) / block.y;
  grid.y = (a.group + x_heads - 1) / x_heads;
  grid.z = (a.units + a.split - 1) / a.split;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == CLQ_F16 ? rope::launch<__half>(V, halves, a, grid, block, s)
                                         : rope::launch<__nv_bfloat16>(V, halves, a, grid, block, s);
  return e == cudaSuccess ? CLQ_OK : CLQ_ERR_CUDA;
}
