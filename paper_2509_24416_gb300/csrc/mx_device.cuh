// E2M1 codes, block scales and activations on the device, shared by the quantization and
// the product's epilogue.
#pragma once

#include "clq_device.cuh"

namespace clq {
namespace mx {

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

// The values of the two codes in the low byte of w (the low nibble's first).
__device__ __forceinline__ __half2 e2m1_pair(uint32_t w) {
  uint32_t h;
  asm("{\n\t.reg .b8 a, b;\n\t"
      "mov.b16 {a, b}, %1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t}"
      : "=r"(h)
      : "h"(static_cast<uint16_t>(w)));
  return *reinterpret_cast<const __half2*>(&h);
}

__device__ __forceinline__ uint32_t e4m3_byte(float v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(v));
  return r & 0xFFu;
}

// Value of an E4M3 byte, exact.
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(byte)));
  return __half2float(__ushort_as_half(static_cast<uint16_t>(h)));
}

// Scale of a block whose largest absolute value has the bits amax: the exponent byte of
// 2^ceil(log2(amax / 6)), 255 for an infinity or a NaN.
__device__ __forceinline__ uint32_t e8m0_byte(uint32_t amax) {
  const int e = static_cast<int>(amax >> 23) - 2 + ((amax & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  return amax >= 0x7F800000u ? 255u : static_cast<uint32_t>(max(e, 0));
}
// 2^(127 - byte) for the bytes 0 .. 253 (of no use for 255).
__device__ __forceinline__ float e8m0_inverse(uint32_t byte) {
  return __uint_as_float((254u - byte) << 23);
}

// 2^(byte - 127), NaN for 255: only 0 and 255 have a mantissa bit.
__device__ __forceinline__ float e8m0_value(uint32_t byte) {
  return __uint_as_float((byte << 23) | (((byte + 1u) & 0xFEu) == 0u ? 0x400000u : 0u));
}

// Activations, within 2^-21 of |x| (of |g u| for swiglu) of the exact ones for every 16-bit x.  With erff, expf and a
// division of full precision (28 and 40 instructions a value) quantisation was bound by
// instructions (16384 x 4608, gelu, BLOCK16: 113 us, with these 75) and the product's epilogue
// took twice the tile's MMAs (65536 rows, 2048 channels of K = 2048: 232 us, with these 107).
// (Two values an instruction where there is one.)
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2e = 1.44269504088896341f;
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 swiglu_fast(float2 g, float2 u) {
  const float2 n = __fmul2_rn(g, both(-kLog2e));
  const float2 d = __fadd2_rn(make_float2(exp2_fast(n.x), exp2_fast(n.y)), both(1.f));
  return __fmul2_rn(__fmul2_rn(g, make_float2(rcp_fast(d.x), rcp_fast(d.y))), u);
}
// max(x, 0) - |x| / 2 erfc(|x| / sqrt 2); erfc(y) = exp(-y^2) f(t), t = 1 / (1 + 0.33 y), f t
// times the polynomial of degree 7 with the smallest relative error up to y = 9.5 (8e-8;
// iteratively reweighted least squares), -1 / 2 in its coefficients.  So the negative side,
// where 1 + erf cancels, keeps its relative precision but for that of exp's argument
// (2^-20.6 to x = -3, 2^-18 to x = -9).
__device__ __forceinline__ float2 gelu_fast(float2 x) {
  const float2 a = make_float2(fabsf(x.x), fabsf(x.y));
  const float2 d = __ffma2_rn(a, both(0.23334524f), both(1.f));
  const float2 t = make_float2(rcp_fast(d.x), rcp_fast(d.y));
  float2 p = __ffma2_rn(t, both(0.0679643899f), both(-0.231344074f));
  p = __ffma2_rn(p, t, both(0.177719399f));
  p = __ffma2_rn(p, t, both(-0.206270739f));
  p = __ffma2_rn(p, t, both(-0.0225053579f));
  p = __ffma2_rn(p, t, both(-0.100961901f));
  p = __ffma2_rn(p, t, both(-0.0914186239f));
  p = __ffma2_rn(p, t, both(-0.0931830555f));
  const float2 q = __fmul2_rn(__fmul2_rn(a, both(-0.5f * kLog2e)), a);
  const float2 e = __fmul2_rn(__fmul2_rn(p, t), make_float2(exp2_fast(q.x), exp2_fast(q.y)));
  return __ffma2_rn(a, e, make_float2(fmaxf(x.x, 0.f), fmaxf(x.y, 0.f)));
}

// v[0 .. N) *= f; plus 0, which gives a product that is exactly 0 the positive sign.
template <int N>
__device__ __forceinline__ void scale_by(float* v, float f) {
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const float2 r = __ffma2_rn(make_float2(v[i], v[i + 1]), both(f), both(0.f));
    v[i] = r.x;
    v[i + 1] = r.y;
  }
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

// Largest absolute value, a NaN if one of them is.
__device__ __forceinline__ float absmax3(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Barrier of two warps (of its number's 64 threads).
__device__ __forceinline__ void pair_barrier(int id) {
  asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory");
}

// The same, and whether all of them had `ok`.
__device__ __forceinline__ bool pair_all(int id, bool ok) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %2, 0;\n\t"
      "barrier.cta.red.and.pred q, %1, 64, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"(id), "r"(static_cast<uint32_t>(ok))
      : "memory");
  return r != 0;
}

}  // namespace mx
}  // namespace clq
