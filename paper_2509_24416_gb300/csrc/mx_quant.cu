// Rows -> E2M1 codes with block scales, and back.
#include "mx_quant_wide.cuh"

namespace clq {
namespace mx {
namespace {

constexpr int U = 16;  // values a thread holds: half a block of 32, or one of 16
constexpr int MAX_ROWS = 256;  // rows that a block works on at a time

// A row's values as they are staged for the swap: the input's own 16 bits, or fp32 behind
// an activation.
template <typename T, int ACT>
struct Staged {
  using type = float;
};
template <typename T>
struct Staged<T, CLQ_MX_ACT_NONE> {
  using type = uint16_t;
};

// v H_b: stages 1, 2, 4, 8 in a thread's values, 16 and up between lanes (K % b == 0, so the
// b / 16 lanes of a block are neighbours, all on or all off).
__device__ __forceinline__ void rotate(float (&v)[U], int b, int lane) {
  if (b > 1) {
#pragma unroll
    for (int i = 0; i < U; i += 2) {
      const float p = v[i], q = v[i + 1];
      v[i] = __fadd_rn(p, q);
      v[i + 1] = __fsub_rn(p, q);
    }
  }
  // two values an instruction; q - p as p (-1) + q, whose product is exact
  auto fma2 = [](float& x0, float& x1, float f, float y0, float y1) {
    const float2 r = __ffma2_rn(make_float2(x0, x1), make_float2(f, f), make_float2(y0, y1));
    x0 = r.x;
    x1 = r.y;
  };
#pragma unroll
  for (int h = 2; h < U; h *= 2) {
    if (h < b) {
#pragma unroll
      for (int i = 0; i < U; i += 2)
        if ((i & h) == 0) {
          const float p0 = v[i], p1 = v[i + 1];
          fma2(v[i], v[i + 1], 1.f, v[i + h], v[i + h + 1]);
          fma2(v[i + h], v[i + h + 1], -1.f, p0, p1);
        }
    }
  }
  for (int m = 1; m * U < b; m *= 2) {
    const float sign = (lane & m) ? -1.f : 1.f;
#pragma unroll
    for (int i = 0; i < U; i += 2) {
      const float o0 = __shfl_xor_sync(0xffffffffu, v[i], m);
      const float o1 = __shfl_xor_sync(0xffffffffu, v[i + 1], m);
      fma2(v[i], v[i + 1], sign, o0, o1);
    }
  }
}

// Where element e of a row is staged: one word is left out after every 32, so that the
// lanes' reads of evenly spaced elements (a swap vector ascends in each half) fall on
// different banks.
template <typename S>
__host__ __device__ __forceinline__ int staged_at(int e) {
  constexpr int W = 4 / sizeof(S);  // elements a word
  return e + W * (e / (32 * W));
}
template <typename S>
__host__ __device__ __forceinline__ int staged_row(int K) {
  return (staged_at<S>(K) + 7) / 8 * 8;
}

// A block works on R = a.block_rows rows at a time, thread t on values 16 x .. + 15 of row y,
// t = y K / 16 + x (lanes of a warp may be of different rows; those that share a block of
// the rotation or a scale are neighbours in one warp, since both divide K).  One pass over X,
// bound by memory where nothing is applied, else by instructions and, with a swap, by shared
// memory (a random swap's reads take 3.5 turns on the banks, the rotation's shuffles the
// rest): the next row's loads are issued before a row is worked on, and a row costs one
// barrier for its swap (two staging buffers in turn) and one for its largest value (three
// slots in turn).  Two rows a thread, a staged word holding an element of both, were slower
// (8192 x 1152 swapped 18.0 us for 17.2, 16384 x 4608 without 39.4 for 35.3: registers).
template <typename T, int FMT, int ACT, bool SWAP>
__global__ void __launch_bounds__(1024) quantize_kernel(QuantArgs a) {
  using S = typename Staged<T, ACT>::type;
  extern __shared__ __align__(16) uint8_t stage_raw[];  // SWAP: two rows of S for each y
  __shared__ uint32_t row_max[3][MAX_ROWS];
  constexpr int NV = ACT == CLQ_MX_ACT_SWIGLU ? 4 : 2;  // 16-byte loads of a thread
  const int units = a.K / U, R = a.block_rows;
  const int lane = threadIdx.x & 31;
  const bool on = static_cast<int>(threadIdx.x) < R * units;
  const int y = on ? threadIdx.x / units : R, x = threadIdx.x - y * units;
  const int chunks = scale_chunks(a.K, FMT);
  // the rows that this warp's lanes are of
  const int y0 = __shfl_sync(0xffffffffu, y, 0), y1 = __shfl_sync(0xffffffffu, y, 31);
  if (FMT == CLQ_MX_BLOCK16) {
    for (int i = threadIdx.x; i < 3 * MAX_ROWS; i += blockDim.x) (&row_max[0][0])[i] = 0;
    __syncthreads();
  }
  pdl_wait();
  pdl_launch_dependents();
  uint32_t src[SWAP ? U / 2 : 1];  // two 16-bit indices each
  if (SWAP && on) {
#pragma unroll
    for (int i = 0; i < U; i += 4) {
      int p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        p[j] = __ldg(a.perm + x * U + i + j);
        if (p[j] < 0 || p[j] >= a.K) {
          record_status(a.status, CLQ_ERR_DEVICE_INDEX);
          p[j] = 0;
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) p[j] = staged_at<S>(p[j]);
      src[i / 2] = static_cast<uint32_t>(p[0] | (p[1] << 16));
      src[i / 2 + 1] = static_cast<uint32_t>(p[2] | (p[3] << 16));
    }
  }
  const int step = gridDim.x * R;
  // rows of a plan: whole blocks of 128, each with its first rows in use
  const int M = a.tiles == nullptr ? a.M : min(a.M, __ldg(a.tile_count) * kRowBlock);
  auto used = [&](int row) {
    return row < M && (a.tiles == nullptr ||
                       (row & (kRowBlock - 1)) < __ldg(&a.tiles[row / kRowBlock].rows));
  };
  uint4 raw[NV];
  bool next = false;
  auto fetch = [&](int row) {
    next = on && used(row);
    if (next) {
      const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.X) +
                                                      static_cast<size_t>(row) * a.ld) +
                       static_cast<size_t>(x) * NV;
#pragma unroll
      for (int i = 0; i < NV; ++i) raw[i] = __ldg(p + i);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) raw[i] = make_uint4(0, 0, 0, 0);
    }
  };
  fetch(blockIdx.x * R + y);
  int turn = 0, slot = 0;
  for (int r0 = blockIdx.x * R; r0 < M; r0 += step, turn ^= 1) {
    const int row = r0 + y;
    const bool live = next;
    float v[U];
    if constexpr (ACT == CLQ_MX_ACT_SWIGLU) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float g[8], u[8];
        unpack8<T>(raw[2 * h], g);
        unpack8<T>(raw[2 * h + 1], u);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float2 y = swiglu_fast(make_float2(g[i], g[i + 1]), make_float2(u[i], u[i + 1]));
          v[8 * h + i] = y.x;
          v[8 * h + i + 1] = y.y;
        }
      }
    } else if constexpr (ACT == CLQ_MX_ACT_GELU || !SWAP) {
      unpack8<T>(raw[0], v);
      unpack8<T>(raw[1], v + 8);
      if (ACT == CLQ_MX_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < U; i += 2) {
          const float2 y = gelu_fast(make_float2(v[i], v[i + 1]));
          v[i] = y.x;
          v[i + 1] = y.y;
        }
      }
    }
    if constexpr (SWAP) {
      S* s = reinterpret_cast<S*>(stage_raw) +
             static_cast<size_t>(turn * R + y) * staged_row<S>(a.K);
      if (on) {
        uint32_t* w = reinterpret_cast<uint32_t*>(s + staged_at<S>(x * U));
        if constexpr (ACT == CLQ_MX_ACT_NONE) {
          const uint32_t r[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w,
                                 raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = r[i];
        } else {
#pragma unroll
          for (int i = 0; i < U; ++i) w[i] = __float_as_uint(v[i]);
        }
      }
      fetch(row + step);
      __syncthreads();
      if (on) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const S e = s[(src[i / 2] >> (16 * (i & 1))) & 0xFFFFu];
          if constexpr (ACT == CLQ_MX_ACT_NONE)
            v[i] = Num<T>::to_f(e);
          else
            v[i] = e;
        }
      } else {
#pragma unroll
        for (int i = 0; i < U; ++i) v[i] = 0.f;
      }
    } else {
      fetch(row + step);
    }
    rotate(v, a.b, lane);
    // Largest absolute value; from here on by its bits, a NaN's being above an infinity's.
    float most = fabsf(v[0]);
#pragma unroll
    for (int i = 1; i + 1 < U; i += 2) most = absmax3(most, v[i], v[i + 1]);
    most = absmax3(most, v[U - 1], v[U - 1]);
    uint32_t amax = __float_as_uint(most);
    uint32_t byte;
    float inv, srow = 0.f;
    bool bad;
    if (FMT == CLQ_MX_BLOCK32) {
      amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      bad = amax >= 0x7F800000u;
      byte = e8m0_byte(amax);
      inv = e8m0_inverse(byte);
    } else {
      for (int r = y0; r <= min(y1, R - 1); ++r) {
        const uint32_t wmax = __reduce_max_sync(0xffffffffu, y == r ? amax : 0u);
        if (lane == 0 && wmax != 0) atomicMax(&row_max[slot][r], wmax);
      }
      __syncthreads();
      const uint32_t rmax = on ? row_max[slot][y] : 0u;
      slot = slot == 2 ? 0 : slot + 1;
      // used again in two rows' time, behind the next row's barrier
      if (on && x == 0) row_max[slot == 2 ? 0 : slot + 1][y] = 0;
      bad = rmax >= 0x7F800000u;
      srow = bad ? __uint_as_float(0x7FC00000u)
                 : fmaxf(__fmul_rn(__uint_as_float(rmax), 1.f / 2688.f), 0x1p-100f);
      byte = bad ? 0u : e4m3_byte(__fdiv_rn(__uint_as_float(amax), __fmul_rn(6.f, srow)));
      inv = byte == 0 ? 0.f : __frcp_rn(__fmul_rn(e4m3_value(byte), srow));
    }
    scale_by<U>(v, inv);
    uint2 q = make_uint2(e2m1x8(v), e2m1x8(v + 8));
    if (bad) q = make_uint2(0, 0);
    // The scale's byte, by the block's first lane; the last block's also zeroes those behind.
    constexpr int LANES = FMT == CLQ_MX_BLOCK32 ? 2 : 1;
    const bool writer = x % LANES == 0;
    const int blk = x / LANES, blocks = units / LANES;
    const int n = a.out_rows == nullptr ? 1 : a.k;
    if (live) {
      for (int j = 0; j < n; ++j) {
        const int at = a.out_rows == nullptr ? row : __ldg(a.out_rows + static_cast<size_t>(row) * a.k + j);
        if (at < 0) continue;
        if (at >= a.rows) {
          record_status(a.status, CLQ_ERR_DEVICE_INDEX);
          continue;
        }
        *reinterpret_cast<uint2*>(a.codes + static_cast<size_t>(at) * (a.K / 2) + x * 8) = q;
        if (writer) {
          uint8_t* p = a.scales + (static_cast<size_t>(at / kRowBlock) * chunks + (blk >> 2)) * 512 +
                       (at & 31) * 16 + ((at >> 5) & 3) * 4;
          p[blk & 3] = static_cast<uint8_t>(byte);
          if (blk == blocks - 1)
            for (int i = (blk & 3) + 1; i < 4; ++i) p[i] = 0;
        }
        if (FMT == CLQ_MX_BLOCK16 && x == 0) a.row_scale[at] = srow;
      }
    }
  }
}

constexpr int TURNS = 4;  // groups of eight codes that a thread takes of a row at a time

// One thread eight codes of a row, so that a warp's stores are whole lines; blockDim.y rows
// at a time.
template <typename T, int FMT>
__global__ void __launch_bounds__(256)
    dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                      const float* __restrict__ row_scale, int M, int K, T* out) {
  const int units = K / 8;
  const int chunks = scale_chunks(K, FMT);
  const int step = gridDim.x * blockDim.y;
  pdl_wait();
  pdl_launch_dependents();
  for (int x0 = threadIdx.x; x0 < units; x0 += TURNS * blockDim.x) {
    uint32_t w[TURNS], byte[TURNS];
    float r = 1.f;
    // a row's loads are issued before the last one's values are stored
    auto fetch = [&](int row) {
      if (row >= M) return;
      const uint32_t* q = reinterpret_cast<const uint32_t*>(codes) + static_cast<size_t>(row) * units;
      const uint8_t* sc = scales + static_cast<size_t>(row / kRowBlock) * chunks * 512 +
                          (row & 31) * 16 + ((row >> 5) & 3) * 4;
#pragma unroll
      for (int i = 0; i < TURNS; ++i) {
        const int x = x0 + i * blockDim.x;
        if (x < units) {
          const int blk = FMT == CLQ_MX_BLOCK32 ? x >> 2 : x >> 1;
          w[i] = __ldg(q + x);
          byte[i] = __ldg(sc + (blk >> 2) * 512 + (blk & 3));
        }
      }
      if (FMT == CLQ_MX_BLOCK16) r = __ldg(row_scale + row);
    };
    int row = blockIdx.x * blockDim.y + threadIdx.y;
    fetch(row);
    for (; row < M; row += step) {
      uint32_t now[TURNS], scale[TURNS];
      const float rs = r;
#pragma unroll
      for (int i = 0; i < TURNS; ++i) {
        now[i] = w[i];
        scale[i] = byte[i];
      }
      fetch(row + step);
      uint4* dst = reinterpret_cast<uint4*>(out) + static_cast<size_t>(row) * units;
#pragma unroll
      for (int i = 0; i < TURNS; ++i) {
        const int x = x0 + i * blockDim.x;
        if (x >= units) break;
        const float s = FMT == CLQ_MX_BLOCK32 ? e8m0_value(scale[i]) : e4m3_value(scale[i]);
        uint32_t o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          // code times block scale is exact; one rounding by the row scale, one by T
          float2 v = __half22float2(e2m1_pair(now[i] >> (8 * j)));
          v = __fmul2_rn(v, make_float2(s, s));
          if (FMT == CLQ_MX_BLOCK16) v = __fmul2_rn(v, make_float2(rs, rs));
          o[j] = Num<T>::pack2(v.x, v.y);
        }
        dst[x] = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
  }
}

template <typename T, int FMT, int ACT>
auto pick(const int32_t* perm) {
  return perm != nullptr ? quantize_kernel<T, FMT, ACT, true> : quantize_kernel<T, FMT, ACT, false>;
}

// A launch of tx x ty threads that may start while the previous kernel finishes.
template <typename... KArgs, typename... Args>
cudaError_t launch_rows(void (*k)(KArgs...), int grid, int tx, int ty, size_t smem, cudaStream_t st,
                        Args... args) {
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(static_cast<unsigned>(tx), static_cast<unsigned>(ty));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, args...);
}

// Many swapped rows rotated by blocks of 64 or 128 (mx_quant_wide.cuh): enough for a tile
// and a quarter a SM, and rows long enough for bulk copies.  Measured, us, wide / 16 values a
// thread, b = 64, BLOCK32: 1152 values a row, 512 rows 6.4 / 4.6, 1024 rows 7.0 / 7.3, 2048 rows
// 7.9 / 9.2; 1024 rows of 2048 8.7 / 8.3, 2048 rows 10.0 / 10.8; 65536 threads' worth of rows of
// 256 values 10.3 / 9.0, of 512 8.9 / 10.9.
bool wide_fits(const QuantArgs& a) {
  return a.perm != nullptr && (a.b == 64 || a.b == 128) && a.act == CLQ_MX_ACT_NONE &&
         a.tiles == nullptr && a.K >= 512 && a.K / WIDE <= WIDE_THREADS &&
         static_cast<int64_t>(a.M) * (a.K / WIDE) >= 5ll * WIDE_THREADS * sm_count() / 4;
}

template <typename T, int FMT>
cudaError_t quantize_wide_t(const QuantArgs& args, cudaStream_t st) {
  QuantArgs a = args;
  const int per_row = a.K / WIDE;
  a.block_rows = WIDE_THREADS / per_row;
  const int threads = (a.block_rows * per_row + 31) / 32 * 32;
  const size_t smem = static_cast<size_t>(WIDE_STAGES) * a.block_rows * a.K * 2;
  auto k = a.b == 64 ? quantize_wide_kernel<T, FMT, 6> : quantize_wide_kernel<T, FMT, 7>;
  int per_sm = 0;
  const cudaError_t e = kernel_setup(reinterpret_cast<const void*>(k), smem, threads, &per_sm);
  if (e != cudaSuccess) return e;
  const int tiles = (a.M + a.block_rows - 1) / a.block_rows;
  return launch_pdl(k, std::min(tiles, std::max(1, per_sm) * sm_count()), threads, smem, st, a);
}

template <typename T, int FMT>
cudaError_t quantize_t(const QuantArgs& args, cudaStream_t st) {
  if (wide_fits(args)) return quantize_wide_t<T, FMT>(args, st);
  // Rows of a block: of those with up to 512 threads the number that leaves the fewest lanes
  // idle, among equals the smallest of at least 128 threads; with few rows no more than give
  // every SM two blocks (256 x 1152: 3.1 us with one row, 3.9 with four).
  QuantArgs a = args;
  const int units = a.K / U;
  int rows = 1;
  double best = 0;
  const int most = std::min(MAX_ROWS, a.M / (2 * sm_count()));
  for (int r = 1; r * units <= 512 && r <= most; ++r) {
    const int threads = (r * units + 31) / 32 * 32;
    const double used = static_cast<double>(r * units) / threads;
    if (used > best + 1e-9 || r * units <= 128) {
      best = used;
      rows = r;
    }
  }
  a.block_rows = rows;
  const int threads = (rows * units + 31) / 32 * 32;
  const size_t smem = a.perm == nullptr ? 0
                      : a.act == CLQ_MX_ACT_NONE
                          ? static_cast<size_t>(2 * rows) * staged_row<uint16_t>(a.K) * 2
                          : static_cast<size_t>(2 * rows) * staged_row<float>(a.K) * 4;
  void (*k)(QuantArgs) =
      a.act == CLQ_MX_ACT_GELU     ? pick<T, FMT, CLQ_MX_ACT_GELU>(a.perm)
      : a.act == CLQ_MX_ACT_SWIGLU ? pick<T, FMT, CLQ_MX_ACT_SWIGLU>(a.perm)
                                   : pick<T, FMT, CLQ_MX_ACT_NONE>(a.perm);
  int per_sm = 0;
  cudaError_t e = kernel_setup(reinterpret_cast<const void*>(k), smem, threads, &per_sm);
  if (e != cudaSuccess) return e;
  const int grid = std::min((a.M + rows - 1) / rows, std::max(1, per_sm) * sm_count());
  return launch_pdl(k, grid, threads, smem, st, a);
}

template <typename T, int FMT>
cudaError_t dequantize_t(const uint8_t* codes, const uint8_t* scales, const float* row_scale,
                         int M, int K, void* out, cudaStream_t st) {
  // the fewest turns of up to 256 threads, evenly long
  const int turns = (K / 8 + 255) / 256;
  const int tx = ((K / 8 + turns - 1) / turns + 31) / 32 * 32;
  const int ty = 256 / tx;
  const int grid = std::min((M + ty - 1) / ty, 8 * sm_count());
  return launch_rows(dequantize_kernel<T, FMT>, grid, tx, ty, 0, st, codes, scales, row_scale, M, K,
                     static_cast<T*>(out));
}

}  // namespace

cudaError_t launch_quantize(const QuantArgs& a, int dtype, int fmt, cudaStream_t st) {
  if (sm_count() <= 0) return cudaErrorInvalidDevice;
  if (dtype == CLQ_F16)
    return fmt == CLQ_MX_BLOCK32 ? quantize_t<__half, CLQ_MX_BLOCK32>(a, st)
                                 : quantize_t<__half, CLQ_MX_BLOCK16>(a, st);
  return fmt == CLQ_MX_BLOCK32 ? quantize_t<__nv_bfloat16, CLQ_MX_BLOCK32>(a, st)
                               : quantize_t<__nv_bfloat16, CLQ_MX_BLOCK16>(a, st);
}

cudaError_t launch_dequantize(const uint8_t* codes, const uint8_t* scales, const float* row_scale,
                              int M, int K, int fmt, int dtype, void* out, cudaStream_t st) {
  if (sm_count() <= 0) return cudaErrorInvalidDevice;
  if (dtype == CLQ_F16)
    return fmt == CLQ_MX_BLOCK32
               ? dequantize_t<__half, CLQ_MX_BLOCK32>(codes, scales, row_scale, M, K, out, st)
               : dequantize_t<__half, CLQ_MX_BLOCK16>(codes, scales, row_scale, M, K, out, st);
  return fmt == CLQ_MX_BLOCK32
             ? dequantize_t<__nv_bfloat16, CLQ_MX_BLOCK32>(codes, scales, row_scale, M, K, out, st)
             : dequantize_t<__nv_bfloat16, CLQ_MX_BLOCK16>(codes, scales, row_scale, M, K, out, st);
}

}  // namespace mx
}  // namespace clq
