// Rows -> E2M1 codes with block scales, and back.
#include "clq_device.cuh"
#include "mx_kernels.h"

namespace clq {
namespace mx {
namespace {

constexpr int U = 16;  // values a thread holds: half a block of 32, or one of 16

// Eight values -> eight E2M1 codes, value 0 in the low nibble; nearest, ties to
// even, saturating.
__device__ __forceinline__ uint32_t e2m1x8(const float* v) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}

__device__ __forceinline__ uint32_t e4m3_byte(float v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(v));
  return r & 0xFFu;
}

// Value of a non-negative E4M3 byte below 0x7F, exact.
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
  const uint32_t e = byte >> 3, m = byte & 7u;
  return e == 0 ? static_cast<float>(m) * 0x1p-9f
                : __uint_as_float(((e + 120u) << 23) | (m << 20));
}

__device__ __forceinline__ float e8m0_value(uint32_t byte) {
  return byte == 0 ? 0x1p-127f : byte == 255 ? __uint_as_float(0x7FC00000u)
                                             : __uint_as_float(byte << 23);
}

template <typename T>
__device__ __forceinline__ void unpack8(const uint4& p, float* v) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = Num<T>::to_f(static_cast<uint16_t>(w[i]));
    v[2 * i + 1] = Num<T>::to_f(static_cast<uint16_t>(w[i] >> 16));
  }
}

// The activations, each operation rounded by itself.
__device__ __forceinline__ float gelu(float x) {
  return __fmul_rn(__fmul_rn(0.5f, x), __fadd_rn(1.f, erff(__fmul_rn(x, 0.70710678118654752f))));
}
__device__ __forceinline__ float swiglu(float g, float u) {
  return __fmul_rn(__fdiv_rn(g, __fadd_rn(1.f, expf(-g))), u);
}

// blockDim.x threads a row (a multiple of 32; thread x holds values 16 x .. + 15),
// blockDim.y rows at a time.
template <typename T, int FMT, int ACT>
__global__ void __launch_bounds__(1024) quantize_kernel(QuantArgs a) {
  extern __shared__ float stage[];  // [blockDim.y][K] with a swap vector
  __shared__ uint32_t row_max[2][32];
  const int units = a.K / U;
  const int x = threadIdx.x, y = threadIdx.y, lane = x & 31;
  const bool on = x < units;
  const int chunks = scale_chunks(a.K, FMT);
  pdl_wait();
  pdl_launch_dependents();
  int src[U];
  if (a.perm != nullptr && on) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int p = a.perm[x * U + i];
      if (p < 0 || p >= a.K) {
        record_status(a.status, CLQ_ERR_DEVICE_INDEX);
        p = 0;
      }
      src[i] = p;
    }
  }
  int turn = 0;
  for (int r0 = blockIdx.x * blockDim.y; r0 < a.M; r0 += gridDim.x * blockDim.y, turn ^= 1) {
    const int row = r0 + y;
    const bool live = on && row < a.M;
    float v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = 0.f;
    if (live) {
      const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.X) +
                                                      static_cast<size_t>(row) * a.ld) +
                       static_cast<size_t>(x) * (ACT == CLQ_MX_ACT_SWIGLU ? 4 : 2);
      if (ACT == CLQ_MX_ACT_SWIGLU) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float g[8], u[8];
          unpack8<T>(__ldg(p + 2 * h), g);
          unpack8<T>(__ldg(p + 2 * h + 1), u);
#pragma unroll
          for (int i = 0; i < 8; ++i) v[8 * h + i] = swiglu(g[i], u[i]);
        }
      } else {
        unpack8<T>(__ldg(p), v);
        unpack8<T>(__ldg(p + 1), v + 8);
        if (ACT == CLQ_MX_ACT_GELU) {
#pragma unroll
          for (int i = 0; i < U; ++i) v[i] = gelu(v[i]);
        }
      }
    }
    if (a.perm != nullptr) {
      float* s = stage + static_cast<size_t>(y) * a.K;
      if (live) {
#pragma unroll
        for (int i = 0; i < U; i += 4)
          *reinterpret_cast<float4*>(s + x * U + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
      }
      __syncthreads();
      if (live) {
#pragma unroll
        for (int i = 0; i < U; ++i) v[i] = s[src[i]];
      }
      __syncthreads();
    }
    // H_b: stages 1, 2, 4, 8 in a thread's values, 16 and up between lanes (K % b ==
    // 0, so the b / 16 lanes of a block are neighbours, all on or all off).
#pragma unroll
    for (int h = 1; h < U; h *= 2) {
      if (h < a.b) {
#pragma unroll
        for (int i = 0; i < U; ++i)
          if ((i & h) == 0) {
            const float p = v[i], q = v[i + h];
            v[i] = __fadd_rn(p, q);
            v[i + h] = __fsub_rn(p, q);
          }
      }
    }
    for (int m = 1; m * U < a.b; m *= 2) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const float o = __shfl_xor_sync(0xffffffffu, v[i], m);
        v[i] = (lane & m) ? __fsub_rn(o, v[i]) : __fadd_rn(v[i], o);
      }
    }
    // Largest absolute value by its bits: a NaN's are above an infinity's.
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < U; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    uint32_t byte;
    float inv, srow = 0.f;
    if (FMT == CLQ_MX_BLOCK32) {
      amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
      const int e = static_cast<int>(amax >> 23) - 2 + ((amax & 0x7FFFFFu) > 0x400000u ? 1 : 0);
      const bool bad = amax >= 0x7F800000u;
      byte = bad ? 255u : static_cast<uint32_t>(max(e, 0));
      inv = bad ? 0.f : __uint_as_float((254u - byte) << 23);
      if (bad) {
#pragma unroll
        for (int i = 0; i < U; ++i) v[i] = 0.f;
      }
    } else {
      if (x == 0) row_max[turn][y] = 0;
      __syncthreads();
      const uint32_t wmax = __reduce_max_sync(0xffffffffu, amax);
      if (lane == 0 && wmax != 0) atomicMax(&row_max[turn][y], wmax);
      __syncthreads();
      const uint32_t rmax = row_max[turn][y];
      const bool bad = rmax >= 0x7F800000u;
      srow = bad ? __uint_as_float(0x7FC00000u)
                 : fmaxf(__fmul_rn(__uint_as_float(rmax), 1.f / 2688.f), 0x1p-100f);
      byte = bad ? 0u : e4m3_byte(__fdiv_rn(__uint_as_float(amax), __fmul_rn(6.f, srow)));
      inv = byte == 0 ? 0.f : __fdiv_rn(1.f, __fmul_rn(e4m3_value(byte), srow));
      if (bad) {
#pragma unroll
        for (int i = 0; i < U; ++i) v[i] = 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = __fmul_rn(v[i], inv);
    const uint2 q = make_uint2(e2m1x8(v), e2m1x8(v + 8));
    // Four scales a word: those of this lane and of three lanes (pairs) behind it.
    if (!on) byte = 0;
    constexpr int STEP = FMT == CLQ_MX_BLOCK32 ? 2 : 1;
    uint32_t word = byte;
#pragma unroll
    for (int j = 1; j < 4; ++j) word |= __shfl_down_sync(0xffffffffu, byte, j * STEP) << (8 * j);
    const bool writer = live && (lane & (4 * STEP - 1)) == 0;
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
          const size_t c = static_cast<size_t>(at / kRowBlock) * chunks + x / (4 * STEP);
          *reinterpret_cast<uint32_t*>(a.scales + c * 512 + (at & 31) * 16 + ((at >> 5) & 3) * 4) =
              word;
        }
        if (FMT == CLQ_MX_BLOCK16 && x == 0) a.row_scale[at] = srow;
      }
    }
  }
}

// One thread 16 codes of a row.
template <typename T, int FMT>
__global__ void dequantize_kernel(const uint8_t* __restrict__ codes,
                                  const uint8_t* __restrict__ scales,
                                  const float* __restrict__ row_scale, int M, int K, T* out) {
  const int units = K / U;
  const int chunks = scale_chunks(K, FMT);
  const size_t n = static_cast<size_t>(M) * units;
  pdl_wait();
  pdl_launch_dependents();
  for (size_t i = blockIdx.x * static_cast<size_t>(blockDim.x) + threadIdx.x; i < n;
       i += static_cast<size_t>(gridDim.x) * blockDim.x) {
    const int row = static_cast<int>(i / units);
    const int x = static_cast<int>(i - static_cast<size_t>(row) * units);
    const int blk = FMT == CLQ_MX_BLOCK32 ? x >> 1 : x;
    const uint32_t byte = scales[(static_cast<size_t>(row / kRowBlock) * chunks + (blk >> 2)) * 512 +
                                 (row & 31) * 16 + ((row >> 5) & 3) * 4 + (blk & 3)];
    const float s = FMT == CLQ_MX_BLOCK32 ? e8m0_value(byte) : e4m3_value(byte);
    const float r = FMT == CLQ_MX_BLOCK32 ? 1.f : row_scale[row];
    const uint2 q = reinterpret_cast<const uint2*>(codes)[i];
    uint32_t o[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      float v[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t c = ((j < 4 ? q.x : q.y) >> (8 * (j & 3) + 4 * h)) & 15u;
        const uint32_t m = c & 7u;
        const float mag = 0.25f * static_cast<float>(m < 2 ? 2 * m : (2 + (m & 1)) << (m >> 1));
        // code times block scale is exact; one rounding by the row scale, one by T
        v[h] = __fmul_rn(__fmul_rn((c & 8u) ? -mag : mag, s), r);
      }
      o[j] = Num<T>::pack2(v[0], v[1]);
    }
    uint4* dst = reinterpret_cast<uint4*>(out) + 2 * i;
    dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
    dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
  }
}

template <typename T, int FMT>
cudaError_t quantize_t(const QuantArgs& a, cudaStream_t st) {
  const int tx = (a.K / U + 31) / 32 * 32;
  const int ty = std::max(1, std::min(32, 256 / tx));
  const size_t smem = a.perm != nullptr ? static_cast<size_t>(ty) * a.K * 4 : 0;
  void (*k)(QuantArgs) = a.act == CLQ_MX_ACT_GELU     ? quantize_kernel<T, FMT, CLQ_MX_ACT_GELU>
                         : a.act == CLQ_MX_ACT_SWIGLU ? quantize_kernel<T, FMT, CLQ_MX_ACT_SWIGLU>
                                                      : quantize_kernel<T, FMT, CLQ_MX_ACT_NONE>;
  int per_sm = 0;
  cudaError_t e = kernel_setup(reinterpret_cast<const void*>(k), smem, tx * ty, &per_sm);
  if (e != cudaSuccess) return e;
  const int grid = std::min((a.M + ty - 1) / ty, std::max(1, per_sm) * sm_count());
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
  return cudaLaunchKernelEx(&cfg, k, a);
}

template <typename T, int FMT>
cudaError_t dequantize_t(const uint8_t* codes, const uint8_t* scales, const float* row_scale,
                         int M, int K, void* out, cudaStream_t st) {
  const size_t n = static_cast<size_t>(M) * (K / U);
  const int grid = static_cast<int>(std::min<size_t>((n + 255) / 256, 8u * sm_count()));
  return launch_pdl(dequantize_kernel<T, FMT>, grid, 256, 0, st, codes, scales, row_scale, M, K,
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
