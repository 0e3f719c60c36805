// Quantization of many swapped and rotated rows: 64 values a thread, b = 64 or 128.
//
// A block of 64 is rotated in one thread's registers (two values an instruction), its
// scales need no other lane, and rows arrive in shared memory by bulk copies, so that a
// swapped element costs one read of shared memory and few instructions besides.  b = 128
// adds one stage between neighbouring lanes, in which each gives away half of its registers.
// Every value passes through the operations of the loop with 16 values a thread
// (mx_quant.cu) and has its bits.  Bound by the reads of the swap (a random one meets some
// 3.5 to a bank) and the latencies that twelve warps a SM leave.  Measured, us, BLOCK32, a
// random swap, here / with 16 values a thread: 8192 x 1152, b = 64, 12.3 / 16.9, b = 128
// 12.9 / 18.0; 16384 x 4608 61 / 91 (3.1 TB/s) and 64 / 99, with neighbours left together
// 59 / 76.  Into eight rows each (8192 x 2048) 33.5 / 37.4: there the scales' stores count, so
// a thread's leave together (b = 128: a pair's; a byte each took 44.5), its codes in one
// store of 32 bytes (two of 16: 38.2).
#pragma once

#include "mx_device.cuh"
#include "mx_kernels.h"

namespace clq {
namespace mx {
namespace {

constexpr int WIDE = 64;           // values a thread
constexpr int WIDE_THREADS = 192;  // at most: 12288 values, 24 KB a stage, two blocks a SM
constexpr int WIDE_STAGES = 3;

// Butterflies of registers k and k + HP (float2 units) of v: sum and difference, or the other
// way round where p = -1 and m = 1.
template <int HP>
__device__ __forceinline__ void wide_stage(float2 (&v)[32], float p, float m) {
  const float2 pp = make_float2(p, p), mm = make_float2(m, m);
#pragma unroll
  for (int k = 0; k < 32; ++k)
    if ((k & HP) == 0) {
      const float2 a = v[k], b = v[k + HP];
      v[k] = __ffma2_rn(b, pp, a);
      v[k + HP] = __ffma2_rn(b, mm, a);
    }
}

template <typename T, int FMT, int LOGB>
__global__ void __launch_bounds__(WIDE_THREADS, 2) quantize_wide_kernel(QuantArgs a) {
  static_assert(LOGB == 6 || LOGB == 7, "");
  extern __shared__ __align__(128) uint8_t stages[];  // [WIDE_STAGES][R][K] of T
  __shared__ uint32_t row_max[3][WIDE_THREADS];
  __shared__ __align__(8) uint64_t full[WIDE_STAGES];
  __shared__ int32_t abort;
  constexpr int BLOCKS = FMT == CLQ_MX_BLOCK16 ? 4 : 2;  // scales of a thread
  const int per_row = a.K / WIDE, R = a.block_rows;
  const int lane = threadIdx.x & 31;
  const bool on = static_cast<int>(threadIdx.x) < R * per_row;
  const int y = on ? threadIdx.x / per_row : 0, x = on ? threadIdx.x - y * per_row : 0;
  const uint32_t row_bytes = static_cast<uint32_t>(a.K) * 2;
  const uint32_t stage_bytes = R * row_bytes;
  const int chunks = scale_chunks(a.K, FMT);
  const int tiles = (a.M + R - 1) / R;
  if (threadIdx.x == 0) {
    for (int s = 0; s < WIDE_STAGES; ++s) mbar_init(&full[s], 1);
    abort = 0;
    fence_mbarrier_init();
  }
  for (int i = threadIdx.x; i < 3 * WIDE_THREADS; i += blockDim.x) (&row_max[0][0])[i] = 0;
  __syncthreads();
  pdl_wait();
  pdl_launch_dependents();
  // The rows of tile blockIdx + i gridDim into stage i, by the first warp.
  auto load = [&](int i) {
    const int64_t t = blockIdx.x + static_cast<int64_t>(i) * gridDim.x;
    if (threadIdx.x >= 32 || t >= tiles) return;
    const int r0 = static_cast<int>(t) * R, n = min(R, a.M - r0), s = i % WIDE_STAGES;
    if (lane == 0) mbar_arrive_expect_tx(&full[s], n * row_bytes);
    __syncwarp();
    for (int r = lane; r < n; r += 32)
      bulk_load(stages + s * stage_bytes + r * row_bytes,
                static_cast<const uint16_t*>(a.X) + static_cast<size_t>(r0 + r) * a.ld, row_bytes,
                &full[s]);
  };
  for (int i = 0; i < WIDE_STAGES; ++i) load(i);
  // Where this thread's elements lie in a stage (bytes), two to a register.  Lanes 128
  // bytes apart would meet on one bank where a swap leaves neighbours together, so register
  // j takes element j ^ 2 order, order the lane's number (for b = 128 its pair's).  The
  // butterflies pair the same elements, and output j comes out as (-1)^popc(j & 2 order)
  // times the transform's, which the sign of its multiplier undoes.
  const int order = LOGB == 6 ? lane : lane & 30;
  const bool wide_perm = (reinterpret_cast<uintptr_t>(a.perm) & 15) == 0;
  uint32_t at[WIDE / 2];
#pragma unroll
  for (int c = 0; c < WIDE / 4; ++c) {
    int p[4] = {0, 0, 0, 0};
    if (on) {
      const int32_t* src = a.perm + x * WIDE + 4 * (c ^ (order >> 1));
      if (wide_perm) {
        const int4 q = __ldg(reinterpret_cast<const int4*>(src));
        p[0] = q.x, p[1] = q.y, p[2] = q.z, p[3] = q.w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = __ldg(src + j);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (p[j] < 0 || p[j] >= a.K) {
        record_status(a.status, CLQ_ERR_DEVICE_INDEX);
        p[j] = 0;
      }
      p[j] = y * row_bytes + 2 * p[j];
    }
    const uint32_t lo = p[0] | (p[1] << 16), hi = p[2] | (p[3] << 16);
    at[2 * c] = (order & 1) ? hi : lo;
    at[2 * c + 1] = (order & 1) ? lo : hi;
  }
  // sign bits to undo: of register 4 c + j, flip[j] with bit c of `turned` on top
  uint32_t flip[4], turned = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) flip[j] = static_cast<uint32_t>(__popc(j & order)) << 31;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const int k = LOGB == 6 ? 4 * c : 4 * (c & 3) | ((lane & 1) << 4);  // position / 2
    turned |= (static_cast<uint32_t>(__popc(k & order)) & 1u) << c;
  }
  const float odd = LOGB == 7 && (lane & 1) ? -1.f : 1.f;
  int slot = 0;
  for (int i = 0;; ++i) {
    const int64_t t = blockIdx.x + static_cast<int64_t>(i) * gridDim.x;
    if (t >= tiles) break;
    const int s = i % WIDE_STAGES;
    const int row = static_cast<int>(t) * R + y;
    const bool live = on && row < a.M;
    const bool ok = mbar_wait_bounded(&full[s], (i / WIDE_STAGES) & 1,
                                      static_cast<volatile int32_t*>(&abort), a.status, kWaitLimitNs);
    const uint8_t* base = stages + s * stage_bytes;
    // (lanes without a row of their own read what is there and store nothing)
    float2 v[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      uint32_t o = at[k];
      asm volatile("" : "+r"(o));  // unpacked here, not ahead of the loop in twice the registers
      const float p = Num<T>::to_f(*reinterpret_cast<const uint16_t*>(base + (o & 0xFFFFu)));
      const float q = Num<T>::to_f(*reinterpret_cast<const uint16_t*>(base + (o >> 16)));
      v[k] = make_float2(__fadd_rn(p, q), __fsub_rn(p, q));
    }
    wide_stage<1>(v, 1.f, -1.f);
    wide_stage<2>(v, 1.f, -1.f);
    wide_stage<4>(v, 1.f, -1.f);
    wide_stage<8>(v, 1.f, -1.f);
    // b = 128: an odd lane's two halves lie the other way round, so that each lane keeps in
    // registers 0 .. 15 the half that its partner's 16 .. 31 belong to
    wide_stage<16>(v, odd, -odd);
    if (LOGB == 7) {
      const float2 s2 = make_float2(odd, odd), n2 = make_float2(-odd, -odd);
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const float2 q = make_float2(__shfl_xor_sync(0xffffffffu, v[k + 16].x, 1),
                                     __shfl_xor_sync(0xffffffffu, v[k + 16].y, 1));
        const float2 own = v[k];
        v[k] = __fadd2_rn(own, q);
        v[k + 16] = __ffma2_rn(own, s2, __fmul2_rn(q, n2));  // even's less odd's
      }
    }
    uint32_t amax[BLOCKS];
#pragma unroll
    for (int q = 0; q < BLOCKS; ++q) {
      constexpr int N = 32 / BLOCKS;
      float most = fabsf(v[q * N].x);
      most = absmax3(most, v[q * N].y, v[q * N].y);
#pragma unroll
      for (int k = 1; k < N; ++k) most = absmax3(most, v[q * N + k].x, v[q * N + k].y);
      amax[q] = __float_as_uint(most);
    }
    if (FMT == CLQ_MX_BLOCK16) {
      uint32_t m = 0;
#pragma unroll
      for (int q = 0; q < BLOCKS; ++q) m = max(m, amax[q]);
      if (live && m != 0) atomicMax(&row_max[slot][y], m);
    }
    if (!__syncthreads_and(ok)) {
      // a copy is missing: those under way land before the block ends
      if (threadIdx.x == 0)
        for (int j = max(0, i - WIDE_STAGES + 1); j < i + WIDE_STAGES; ++j) {
          if (blockIdx.x + static_cast<int64_t>(j) * gridDim.x >= tiles) break;
          mbar_wait_bounded(&full[j % WIDE_STAGES], (j / WIDE_STAGES) & 1, nullptr, nullptr, 10000000ull);
        }
      return;
    }
    load(i + WIDE_STAGES);  // every thread has read this stage
    uint32_t rmax = 0;
    if (FMT == CLQ_MX_BLOCK16) {
      rmax = row_max[slot][y];
      slot = slot == 2 ? 0 : slot + 1;
      // used again in two tiles' time, behind the next tile's barrier
      if (on && x == 0) row_max[slot == 2 ? 0 : slot + 1][y] = 0;
    }
    float srow = 0.f;
    const bool bad_row = rmax >= 0x7F800000u;
    if (FMT == CLQ_MX_BLOCK16)
      srow = bad_row ? __uint_as_float(0x7FC00000u)
                     : fmaxf(__fmul_rn(__uint_as_float(rmax), 1.f / 2688.f), 0x1p-100f);
    uint32_t w[8], word = 0;
#pragma unroll
    for (int q = 0; q < BLOCKS; ++q) {
      uint32_t byte;
      float inv;
      bool bad = bad_row;
      if (FMT == CLQ_MX_BLOCK32) {
        bad = amax[q] >= 0x7F800000u;
        byte = e8m0_byte(amax[q]);
        inv = e8m0_inverse(byte);
      } else {
        byte = bad ? 0u : e4m3_byte(__fdiv_rn(__uint_as_float(amax[q]), __fmul_rn(6.f, srow)));
        inv = byte == 0 ? 0.f : __frcp_rn(__fmul_rn(e4m3_value(byte), srow));
      }
      constexpr int C = 8 / BLOCKS;  // chunks of a block
      word |= byte << (8 * q);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const uint32_t m = __float_as_uint(inv) ^ ((turned << (31 - q * C - c)) & 0x80000000u);
        float f[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float t = __uint_as_float(m ^ flip[j]);
          const float2 r = __ffma2_rn(v[4 * (q * C + c) + j], make_float2(t, t), make_float2(0.f, 0.f));
          f[2 * j] = r.x;
          f[2 * j + 1] = r.y;
        }
        w[q * C + c] = bad ? 0u : e2m1x8(f);
      }
    }
    if (LOGB == 7) {  // whole chunks of four scales: BLOCK32 the even lane's, BLOCK16 one each
      const uint32_t o = __shfl_xor_sync(0xffffffffu, word, 1);
      word = FMT == CLQ_MX_BLOCK32 ? __byte_perm(word, o, 0x5140)
             : (lane & 1)          ? __byte_perm(word, o, 0x3276)
                                   : __byte_perm(word, o, 0x5410);
    }
    if (!live) continue;
    // Registers 0 .. 15 hold 32 positions from `first`, the others those `apart` behind.
    const int first = LOGB == 6 ? x * WIDE : (x >> 1) * 128 + (x & 1) * 32;
    constexpr int apart = LOGB == 6 ? 32 : 64;
    const int n = a.out_rows == nullptr ? 1 : a.k;
    const bool whole = (reinterpret_cast<uintptr_t>(a.codes) & 31) == 0;  // one 32-byte store
    for (int j = 0; j < n; ++j) {
      const int to = a.out_rows == nullptr ? row : __ldg(a.out_rows + static_cast<size_t>(row) * a.k + j);
      if (to < 0) continue;
      if (to >= a.rows) {
        record_status(a.status, CLQ_ERR_DEVICE_INDEX);
        continue;
      }
      uint8_t* q = a.codes + static_cast<size_t>(to) * (a.K / 2) + first / 2;
      if (LOGB == 6 && whole) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(q), "r"(w[0]),
                     "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
      } else {
        *reinterpret_cast<uint4*>(q) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(q + apart / 2) = make_uint4(w[4], w[5], w[6], w[7]);
      }
      uint8_t* p = a.scales + static_cast<size_t>(to / kRowBlock) * chunks * 512 + (to & 31) * 16 +
                   ((to >> 5) & 3) * 4;
      if (LOGB == 6) {  // all of them neighbours
        if (FMT == CLQ_MX_BLOCK16) {
          *reinterpret_cast<uint32_t*>(p + x * 512) = word;
        } else {
          *reinterpret_cast<uint16_t*>(p + (x >> 1) * 512 + 2 * (x & 1)) = static_cast<uint16_t>(word);
          if (x == per_row - 1 && (x & 1) == 0)  // behind the last block: zeros
            *reinterpret_cast<uint16_t*>(p + (x >> 1) * 512 + 2) = 0;
        }
      } else if ((x & 1) == 0 || FMT == CLQ_MX_BLOCK16) {
        const int chunk = FMT == CLQ_MX_BLOCK16 ? x : x >> 1;
        *reinterpret_cast<uint32_t*>(p + chunk * 512) = word;
      }
      if (FMT == CLQ_MX_BLOCK16 && x == 0) a.row_scale[to] = srow;
    }
  }
}

}  // namespace
}  // namespace mx
}  // namespace clq
