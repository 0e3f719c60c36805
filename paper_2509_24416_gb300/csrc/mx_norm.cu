// Root-mean-square norm of rows, behind the addition of a residual and in front of their swap,
// rotation and quantization.
#include "mx_rows.cuh"
#include "mx_kernels.h"

namespace clq {
namespace mx {
namespace {

constexpr int NORM_ROWS = 32;  // rows that a block works on at a time, one warp each at least
constexpr int MAX_WARPS = 32;
constexpr int PACKED_THREADS = 288;  // at most, of rows that share warps

// A row's sum of squares, in one order whatever row of a block it is: a thread's 16 neighbours (a
// unit) as two halves of eight, each a chain of pairs; 32 units by halving exchanges, their sums by
// another.
//
// Sums outside fp32's range: a unit whose own reaches 2^100 counts its squares times 2^-160
// instead (`hi`), so that neither of a row's two sums overflows for finite values.
constexpr float kHuge = 0x1p100f, kDown = 0x1p-80f;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int m = 16; m > 0; m /= 2) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}

__device__ __forceinline__ float squares8(const float* v) {
  float2 s = __fmul2_rn(make_float2(v[0], v[1]), make_float2(v[0], v[1]));
#pragma unroll
  for (int i = 2; i < 8; i += 2)
    s = __ffma2_rn(make_float2(v[i], v[i + 1]), make_float2(v[i], v[i + 1]), s);
  return __fadd_rn(s.x, s.y);
}

__device__ __forceinline__ float squares_down(const float* v) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < U; ++i) s = __fmaf_rn(v[i] * kDown, v[i] * kDown, s);
  return s;
}

// 1 / sqrt(mean + eps) of the row with these sums; 1 / K in two parts, whose product with a sum is
// rounded once (1 / K in one part would bias every row by up to 2^-25).
__device__ __forceinline__ float inverse_root(float lo, float hi, const NormArgs& a) {
  if (hi == 0.f) return __frsqrt_rn(__fmaf_rn(lo, a.inv_k, __fmaf_rn(lo, a.inv_k_low, a.eps)));
  // (an infinite sum stays one: the second part may be negative)
  return __frsqrt_rn(__fmaf_rn(hi + lo * kDown * kDown, a.inv_k, a.eps * kDown * kDown)) * kDown;
}

// A row's two sums by one warp, unit(u, lo, hi) the sums of unit u: four warps' worth at a time.
template <typename F>
__device__ __forceinline__ float2 sum_units(int units, int lane, F unit) {
  float lo = 0.f, hi = 0.f;  // those of units 32 g .. + 31 in lane g
  for (int g0 = 0; 32 * g0 < units; g0 += 4) {
    float l[4], h[4];
    bool huge = false;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int u = 32 * (g0 + g) + lane;
      l[g] = h[g] = 0.f;
      if (u < units) unit(u, l[g], h[g]);
      huge = huge || h[g] != 0.f;
    }
    huge = __any_sync(0xffffffffu, huge);
#pragma unroll
    for (int g = 0; g < 4; ++g) l[g] = warp_sum(l[g]);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (huge) h[g] = warp_sum(h[g]);
      if (lane == g0 + g) {
        lo = l[g];
        hi = h[g];
      }
    }
  }
  lo = warp_sum(lo);
  if (__any_sync(0xffffffffu, hi != 0.f)) hi = warp_sum(hi);
  return make_float2(lo, hi);
}

// Eight sums rounded to T: their bits, and v the values of those.
template <typename T>
__device__ __forceinline__ uint4 add_rounded(float* v, const float* q) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h[i] = Num<T>::pack2(__fadd_rn(v[2 * i], q[2 * i]), __fadd_rn(v[2 * i + 1], q[2 * i + 1]));
    v[2 * i] = Num<T>::to_f(static_cast<uint16_t>(h[i]));
    v[2 * i + 1] = Num<T>::to_f(static_cast<uint16_t>(h[i] >> 16));
  }
  return make_uint4(h[0], h[1], h[2], h[3]);
}

// A thread's 16 values, in 16 bits each.
struct Raw {
  uint4 p[2];
  __device__ __forceinline__ void zero() { p[0] = p[1] = make_uint4(0, 0, 0, 0); }
  // (not through the read-only path: the sum may be written over its input)
  __device__ __forceinline__ void load(const uint16_t* src) {
    p[0] = reinterpret_cast<const uint4*>(src)[0];
    p[1] = reinterpret_cast<const uint4*>(src)[1];
  }
};

// A thread works on 16 neighbours of a row, a block on R rows at a time, in steps of gridDim R.  One
// pass: the next row's loads are under way while a row, held in 16 bits, is worked on, and one barrier
// covers its sum and its swap (what is staged are the rows, not the normed values: the factor and
// the weights are multiplied on behind it).  A row takes whole warps, or, where it is swapped and
// would leave lanes idle (`packed`), the threads that it needs, its units' sums being added up by
// one warp behind a second barrier (8192 x 1152, b = 64, with a residual 22 us for 26).  Bound by
// memory without a swap (16384 x 4608 with a residual to 8 bits 86 us, 6.2 TB/s; 32768 x 2048 71,
// 6.7), with one by instructions, some 700 for 16 values, and the reads of a random swap (16384 x 4608,
// b = 64, 124 us).  (The sums across warps read by every lane instead of exchanged: 16384 x 4608
// without a residual 58 us for 50.  64 values a thread behind bulk copies, as the quantization of
// many swapped rows has it: between 18 % slower, at 32768 x 1152, and 10 % faster, at 16384 x 8192
// without a residual.)
// THREADS: of a block at most.  Up to 288 three blocks fit a SM, in 72 registers a thread (in the 88
// to 112 that the swapped ones would take two: 8192 x 1152 in blocks of 16, swapped, 33 us for 23,
// 4096 x 4096 to 8 bits 37 for 33; four blocks spill, 27 us); 1024 have 64.  Rows of more than 8192
// values leave a SM one block, whose loads alone do not keep memory busy: with a residual and no swap
// the row behind the next one is asked into L2 (AHEAD; 4096 x 12288 66 us for 75; elsewhere it costs:
// 16384 x 4608 93 for 84, 4096 x 12288 without a residual 39 for 35, swapped 110 for 108, and 300 x 12288, whose
// blocks have no row behind the next one, 5.9 for 5.7).  Without a swap rows take whole warps however short they are:
// 65536 x 256 with half of the lanes 19 us, 25 with a residual (memory alone 8 and 17), 65536 x 1152 63 and 88 (34, 78).
template <typename T, int FMT, bool RESIDUAL, bool SWAP, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS <= 288 ? 3 : 1) norm_kernel(NormArgs a, int R, int packed) {
  extern __shared__ __align__(16) uint8_t stage_raw[];  // SWAP: two rows of 16 bits for each y
  __shared__ float2 sums[2][MAX_WARPS];
  __shared__ uint32_t maxima[2][MAX_WARPS];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __shared__ float2 unit_sums[SWAP ? PACKED_THREADS : 1];
  __shared__ float row_inv[NORM_ROWS];
  __shared__ uint32_t row_max[3][NORM_ROWS];
  constexpr bool AHEAD = RESIDUAL && !SWAP && THREADS > 512;
  const bool rows_packed = SWAP && packed;
  const int units = a.K / U;
  const int W = static_cast<int>(blockDim.x) / (32 * R);  // warps a row
  int y, x;
  if (SWAP && rows_packed) {
    y = min(static_cast<int>(threadIdx.x) / units, R);
    x = threadIdx.x - y * units;
  } else {
    y = warp / W;
    x = threadIdx.x - y * W * 32;
  }
  const bool on = (!SWAP || y < R) && x < units;
  int y0 = 0, y1 = 0;  // the rows that this warp's lanes are of
  if (SWAP && FMT == CLQ_MX_BLOCK16 && rows_packed) {
    y0 = __shfl_sync(0xffffffffu, y, 0);
    y1 = min(__shfl_sync(0xffffffffu, y, 31), R - 1);
    for (int i = threadIdx.x; i < 3 * NORM_ROWS; i += blockDim.x) (&row_max[0][0])[i] = 0;
    __syncthreads();
  }
  const int chunks = scale_chunks(a.K, FMT);
  const int step = gridDim.x * R;
  pdl_wait();
  pdl_launch_dependents();
  uint32_t src[SWAP ? U / 2 : 1];  // staged places, two 16-bit ones each
  uint32_t weight[U / 2];          // this thread's outputs' weights, two each
#pragma unroll
  for (int i = 0; i < U / 2; ++i) {
    weight[i] = 0;
    if (SWAP) src[i] = 0;
  }
  if (on) {
    const uint32_t one = Num<T>::pack2(1.f, 1.f);
    const uint16_t* w = static_cast<const uint16_t*>(a.weight);
    if (SWAP) {
      int p[U];
      if ((reinterpret_cast<uintptr_t>(a.perm) & 15) == 0) {
#pragma unroll
        for (int i = 0; i < U; i += 4) {
          const int4 q = __ldg(reinterpret_cast<const int4*>(a.perm + x * U + i));
          p[i] = q.x, p[i + 1] = q.y, p[i + 2] = q.z, p[i + 3] = q.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < U; ++i) p[i] = __ldg(a.perm + x * U + i);
      }
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (p[i] < 0 || p[i] >= a.K) {
          record_status(a.status, CLQ_ERR_DEVICE_INDEX);
          p[i] = 0;
        }
#pragma unroll
      for (int i = 0; i < U; i += 2) {
        weight[i / 2] = w == nullptr
                            ? one
                            : __ldg(w + p[i]) | (static_cast<uint32_t>(__ldg(w + p[i + 1])) << 16);
        src[i / 2] = static_cast<uint32_t>(staged_at<uint16_t>(p[i])) |
                     (static_cast<uint32_t>(staged_at<uint16_t>(p[i + 1])) << 16);
      }
    } else {
      const uint4* q = reinterpret_cast<const uint4*>(w) + 2 * x;
      const uint4 q0 = w == nullptr ? make_uint4(one, one, one, one) : __ldg(q);
      const uint4 q1 = w == nullptr ? make_uint4(one, one, one, one) : __ldg(q + 1);
      weight[0] = q0.x, weight[1] = q0.y, weight[2] = q0.z, weight[3] = q0.w;
      weight[4] = q1.x, weight[5] = q1.y, weight[6] = q1.z, weight[7] = q1.w;
    }
  }
  Raw in, res;
  auto fetch = [&](int row) {
    in.zero();
    if (RESIDUAL) res.zero();
    if (on && row < a.M) {
      in.load(static_cast<const uint16_t*>(a.X) + static_cast<size_t>(row) * a.ldx + x * U);
      if (RESIDUAL)
        res.load(static_cast<const uint16_t*>(a.residual) + static_cast<size_t>(row) * a.ldr + x * U);
    }
  };
  int row = blockIdx.x * R + y;
  fetch(row);
  int turn = 0, slot = 0;
  for (int r0 = blockIdx.x * R; r0 < a.M; r0 += step, row += step, turn ^= 1) {
    const bool live = on && row < a.M;
    float v[U];
    unpack8<T>(in.p[0], v);
    unpack8<T>(in.p[1], v + 8);
    if (RESIDUAL) {
      float q[U];
      unpack8<T>(res.p[0], q);
      unpack8<T>(res.p[1], q + 8);
      in.p[0] = add_rounded<T>(v, q);
      in.p[1] = add_rounded<T>(v + 8, q + 8);
      if (live) {
        uint4* to = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.sum) +
                                             static_cast<size_t>(row) * a.lds + x * U);
        to[0] = in.p[0];
        to[1] = in.p[1];
      }
    }
    if (SWAP && on) {
      const uint32_t h[U / 2] = {in.p[0].x, in.p[0].y, in.p[0].z, in.p[0].w,
                                 in.p[1].x, in.p[1].y, in.p[1].z, in.p[1].w};
      uint32_t* w = reinterpret_cast<uint32_t*>(
          reinterpret_cast<uint16_t*>(stage_raw) +
          static_cast<size_t>(turn * R + y) * staged_row<uint16_t>(a.K) + staged_at<uint16_t>(x * U));
#pragma unroll
      for (int i = 0; i < U / 2; ++i) w[i] = h[i];
    }
    fetch(row + step);
    if (AHEAD && on && x == 0 && row + 2 * step < a.M) {
      const size_t next = static_cast<size_t>(row + 2 * step);
      bulk_prefetch_l2(static_cast<const uint16_t*>(a.X) + next * a.ldx, 2 * a.K);
      bulk_prefetch_l2(static_cast<const uint16_t*>(a.residual) + next * a.ldr, 2 * a.K);
    }
    float lo = __fadd_rn(squares8(v), squares8(v + 8)), hi = 0.f;
    if (!(lo < kHuge)) {
      hi = squares_down(v);
      lo = 0.f;
    }
    float inv;
    if (rows_packed) {
      if (on) unit_sums[threadIdx.x] = make_float2(lo, hi);
      __syncthreads();
      for (int r = warp; r < R; r += blockDim.x / 32) {
        const float2 sum = sum_units(units, lane, [&](int u, float& l, float& h) {
          const float2 p = unit_sums[r * units + u];
          l = p.x;
          h = p.y;
        });
        if (lane == 0) row_inv[r] = inverse_root(sum.x, sum.y, a);
      }
      __syncthreads();
      inv = row_inv[on ? y : 0];
    } else {
      lo = warp_sum(lo);
      if (__any_sync(0xffffffffu, hi != 0.f)) hi = warp_sum(hi);
      if (W > 1) {
        if (lane == 0) sums[turn][warp] = make_float2(lo, hi);
      }
      if (W > 1 || SWAP) __syncthreads();
      if (W > 1) {
        const float2 p = lane < W ? sums[turn][y * W + lane] : make_float2(0.f, 0.f);
        lo = warp_sum(p.x);
        hi = p.y;
        if (__any_sync(0xffffffffu, hi != 0.f)) hi = warp_sum(hi);
      }
      inv = inverse_root(lo, hi, a);
    }
    if (SWAP) {
      const uint16_t* s = reinterpret_cast<const uint16_t*>(stage_raw) +
                          static_cast<size_t>(turn * R + (on ? y : 0)) * staged_row<uint16_t>(a.K);
      // (lanes without values of their own read what is there: no other lane looks at theirs)
#pragma unroll
      for (int i = 0; i < U; ++i) v[i] = Num<T>::to_f(s[(src[i / 2] >> (16 * (i & 1))) & 0xFFFFu]);
    }
#pragma unroll
    for (int i = 0; i < U; i += 2) {
      const float2 w2 = make_float2(Num<T>::to_f(static_cast<uint16_t>(weight[i / 2])),
                                    Num<T>::to_f(static_cast<uint16_t>(weight[i / 2] >> 16)));
      const float2 r = __fmul2_rn(__fmul2_rn(make_float2(v[i], v[i + 1]), both(inv)), w2);
      v[i] = r.x;
      v[i + 1] = r.y;
    }
    rotate(v, a.b, lane);
    float most = fabsf(v[0]);
#pragma unroll
    for (int i = 1; i + 1 < U; i += 2) most = absmax3(most, v[i], v[i + 1]);
    most = absmax3(most, v[U - 1], v[U - 1]);
    uint32_t amax = on ? __float_as_uint(most) : 0u;
    uint32_t byte;
    float f, srow = 0.f;
    bool bad;
    if (FMT != CLQ_MX_BLOCK16) {
      amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      bad = amax >= 0x7F800000u;
      byte = e8m0_byte<FMT>(amax);
      f = e8m0_inverse(byte);
    } else {
      uint32_t rmax;
      if (rows_packed) {
        for (int r = y0; r <= y1; ++r) {
          const uint32_t wmax = __reduce_max_sync(0xffffffffu, y == r ? amax : 0u);
          if (lane == 0 && wmax != 0) atomicMax(&row_max[slot][r], wmax);
        }
        __syncthreads();
        rmax = on ? row_max[slot][y] : 0u;
        slot = slot == 2 ? 0 : slot + 1;
        // used again in two rows' time, behind the next rows' barriers
        if (on && x == 0) row_max[slot == 2 ? 0 : slot + 1][y] = 0;
      } else {
        rmax = __reduce_max_sync(0xffffffffu, amax);
        if (W > 1) {
          if (lane == 0) maxima[turn][warp] = rmax;
          __syncthreads();
          rmax = __reduce_max_sync(0xffffffffu, lane < W ? maxima[turn][y * W + lane] : 0u);
        }
      }
      bad = rmax >= 0x7F800000u;
      srow = row_scale_of(rmax);
      byte = bad ? 0u : e4m3_byte(__fdiv_rn(__uint_as_float(amax), __fmul_rn(6.f, srow)));
      f = byte == 0 ? 0.f : __frcp_rn(__fmul_rn(e4m3_value(byte), srow));
    }
    scale_by<U>(v, f);
    auto q = Codes16<FMT>::of(v);
    if (bad) q = Codes16<FMT>::zero();
    constexpr int LANES = FMT != CLQ_MX_BLOCK16 ? 2 : 1;
    const int blk = x / LANES, blocks = units / LANES;
    if (live) {
      reinterpret_cast<decltype(q)*>(a.codes + static_cast<size_t>(row) * code_bytes(a.K, FMT))[x] = q;
      if (x % LANES == 0) {
        uint8_t* p = a.scales + (static_cast<size_t>(row / kRowBlock) * chunks + (blk >> 2)) * 512 +
                     (row & 31) * 16 + ((row >> 5) & 3) * 4;
        p[blk & 3] = static_cast<uint8_t>(byte);
        if (blk == blocks - 1)
          for (int i = (blk & 3) + 1; i < 4; ++i) p[i] = 0;
      }
      if (FMT == CLQ_MX_BLOCK16 && x == 0) a.row_scale[row] = srow;
    }
  }
}

template <typename T, int FMT, int THREADS>
auto pick_norm(const NormArgs& a) {
  const bool res = a.residual != nullptr;
  if (a.perm != nullptr)
    return res ? norm_kernel<T, FMT, true, true, THREADS> : norm_kernel<T, FMT, false, true, THREADS>;
  return res ? norm_kernel<T, FMT, true, false, THREADS> : norm_kernel<T, FMT, false, false, THREADS>;
}

template <typename T, int FMT>
cudaError_t norm_t(const NormArgs& a, cudaStream_t st) {
  const int units = a.K / U, W = (units + 31) / 32;
  // Rows of a block: up to 256 threads, no more than leave every SM two blocks; with rows that share
  // warps those of up to 288 threads that leave the fewest lanes idle.
  const int most = std::min(NORM_ROWS, a.M / (2 * sm_count()));
  int R = std::max(1, std::min(8 / W, most)), threads = 32 * W * R, packed = 0;
  if (a.perm != nullptr && units % 32 != 0) {
    double best = static_cast<double>(units) / (32 * W);
    for (int r = 2; r <= most && r * units <= PACKED_THREADS; ++r) {
      const int n = (r * units + 31) / 32 * 32;
      const double used = static_cast<double>(r * units) / n;
      if (used > best + 1e-9 || (packed && n <= 256 && used > best - 1e-9)) {
        best = used;
        R = r;
        threads = n;
        packed = 1;
      }
    }
  }
  const size_t smem = a.perm == nullptr ? 0 : static_cast<size_t>(2 * R) * staged_row<uint16_t>(a.K) * 2;
  void (*k)(NormArgs, int, int) = threads <= 288   ? pick_norm<T, FMT, 288>(a)
                                  : threads <= 512 ? pick_norm<T, FMT, 512>(a)
                                                   : pick_norm<T, FMT, 1024>(a);
  int per_sm = 0;
  const cudaError_t e = kernel_setup(reinterpret_cast<const void*>(k), smem, threads, &per_sm);
  if (e != cudaSuccess) return e;
  const int grid = std::min((a.M + R - 1) / R, std::max(1, per_sm) * sm_count());
  return launch_pdl(k, grid, threads, smem, st, a, R, packed);
}

template <typename T>
cudaError_t norm_f(const NormArgs& a, int fmt, cudaStream_t st) {
  if (fmt == CLQ_MX_BLOCK32) return norm_t<T, CLQ_MX_BLOCK32>(a, st);
  if (fmt == CLQ_MX_BLOCK16) return norm_t<T, CLQ_MX_BLOCK16>(a, st);
  return norm_t<T, CLQ_MX_BLOCK32_E4M3>(a, st);
}

}  // namespace

cudaError_t launch_norm(const NormArgs& a, int dtype, int fmt, cudaStream_t st) {
  if (sm_count() <= 0) return cudaErrorInvalidDevice;
  return dtype == CLQ_F16 ? norm_f<__half>(a, fmt, st) : norm_f<__nv_bfloat16>(a, fmt, st);
}

}  // namespace mx
}  // namespace clq
