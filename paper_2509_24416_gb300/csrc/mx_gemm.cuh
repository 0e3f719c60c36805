// Product of two arrays of microscaled E2M1 codes, dense or one matrix per expert.
//
// D[n][i] = sum_k w[n][k] x[i][k], each value a code times its block's scale:
// tcgen05.mma kind::mxf4 / kind::mxf4nvf4 multiplies codes and scales exactly and
// accumulates in fp32 in tensor memory.  The weights are the MMA's A operand (128
// output channels a CTA, the lanes of tensor memory) and the rows of X its B operand
// (NT columns), so that one kernel serves a single token (NT = 32) and long batches:
// with the rows as A, one token would cost the MMAs and operands of 128.
//
// Codes arrive by TMA in the 128-byte swizzle, 256 codes a row and K step; scales, 512
// bytes for 128 rows and four blocks as they lie in memory, go through shared memory
// into tensor memory by tcgen05.cp, which repeats them for the four groups of lanes.
//
// Roles: warp 4 copies, one lane of warp 5 issues tcgen05.cp and tcgen05.mma, warps
// 0-3 and 6-9 take a tile out of tensor memory (32 channels and a share of the
// columns each) while the next tile's MMAs run in the other accumulator.  Every wait is
// bounded.
#pragma once

#include "gemm_common.cuh"
#include "mx_device.cuh"
#include "mx_kernels.h"
#include "mx_tiles.h"

namespace clq {
namespace mx {

using gemm::EPI_BYTES;
using gemm::EPI_COLS;

constexpr int WARP_TMA = 4;
constexpr int WARP_MMA = 5;
// Eight: with sixteen the registers left to each spill (32768 x 4096 -> 8192 in blocks of 16
// 323 -> 351 us; the experts' GELU in the epilogue 88 -> 105).
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 32 * (EPI_WARPS + 2);
constexpr int MAX_STAGES = 8;

template <int FMT, int NT, int CG>
struct Cfg {
  static constexpr int SC = FMT == CLQ_MX_BLOCK16 ? 4 : 2;  // scale chunks of a K step
  static constexpr int XB = NT > 128 ? NT / 128 : 1;        // row blocks of X in a tile
  static constexpr int A = TN * 128;
  static constexpr int B = NT / CG * 128;
  static constexpr int SA = SC * 512;
  static constexpr int SB = XB * SC * 512;
  static constexpr int STAGE = A + B + SA + SB;
  static constexpr uint32_t TX = CG * STAGE;
  static constexpr int PARTS = NT >= 64 ? 2 : 1;  // column shares (four warps each)
  static constexpr int NCOL = NT / PARTS;
  static constexpr int FIXED = EPI_WARPS * 2 * EPI_BYTES;  // two staging buffers a warp
  static constexpr int S0 = (222 * 1024 - FIXED) / STAGE;
  static constexpr int S = S0 > MAX_STAGES ? MAX_STAGES : S0;
  static constexpr int OFF_A = 0;
  static constexpr int OFF_B = OFF_A + S * A;
  static constexpr int OFF_SA = OFF_B + S * B;
  static constexpr int OFF_SB = OFF_SA + S * SA;
  static constexpr int OFF_EPI = OFF_SB + S * SB;
  static constexpr int BYTES = OFF_EPI + FIXED;
  // Tensor memory: two accumulators of NT columns and the scales of NSF K steps (tcgen05
  // copies and MMAs of one thread run in the order of their issue; a second buffer beside
  // 256-column accumulators would make them share more columns than two blocks: 32768 x 4096
  // -> 8192 in blocks of 16 357 us, with one 327).
  static constexpr int SFA = 4 * SC;
  static constexpr int SFB = 4 * SC * XB;
  static constexpr int SF = SFA + SFB;
  static constexpr int NSF = NT == 256 ? 1 : 2;
  static constexpr int NEED = 2 * NT + NSF * SF;
  static constexpr int TMEM = NEED <= 128 ? 128 : NEED <= 256 ? 256 : 512;
  // Two accumulators of 256 columns and the scales do not fit: the second then starts
  // OV columns inside the first, and a tile's MMAs wait for those alone.
  static constexpr int OV = NEED > 512 ? (NEED - 512 + 31) / 32 * 32 : 0;
  static constexpr int OFF_SF = 2 * NT - OV;
  static_assert(OFF_SF + NSF * SF <= TMEM && OV <= NCOL, "tensor memory");
  static_assert(S >= 3 && STAGE % 1024 == 0, "stages");
};

struct __align__(8) Bars {
  uint64_t full[MAX_STAGES];
  uint64_t empty[MAX_STAGES];
  uint64_t acc_full[2];
  uint64_t acc_empty[2];
  uint64_t ov_empty;  // the overlapped columns have been taken out
  uint64_t drained;
  uint32_t tmem_slot;
  int32_t abort;
};

// Scales of 32 rows x 16 bytes, shared -> tensor memory, for each group of 32 lanes.
template <int CG>
__device__ __forceinline__ void cp_scales(uint32_t taddr, uint64_t desc) {
  if (CG == 2)
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc)
                 : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc)
                 : "memory");
}

// Descriptor of 512 contiguous bytes: four 8-row groups of 128 bytes, no swizzle.
__device__ __forceinline__ uint64_t scale_desc(uint32_t smem_byte_addr) {
  return static_cast<uint64_t>((smem_byte_addr >> 4) & 0x3FFFu) |
         (static_cast<uint64_t>(128u >> 4) << 32) | (static_cast<uint64_t>(1u) << 46);
}

template <int FMT, int CG>
__device__ __forceinline__ void mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc,
                                       uint32_t sfa, uint32_t sfb, uint32_t acc) {
#define CLQ_MX_MMA(G, KIND)                                                              \
  asm volatile(                                                                          \
      "{\n\t.reg .pred p;\n\t"                                                           \
      "setp.ne.b32 p, %4, 0;\n\t"                                                        \
      "tcgen05.mma.cta_group::" G "." KIND " [%0], %1, %2, %3, [%5], [%6], p;\n\t}" ::   \
          "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(sfa), "r"(sfb)               \
      : "memory")
  if (FMT == CLQ_MX_BLOCK32) {
    if (CG == 2)
      CLQ_MX_MMA("2", "kind::mxf4.block_scale.scale_vec::2X");
    else
      CLQ_MX_MMA("1", "kind::mxf4.block_scale.scale_vec::2X");
  } else {
    if (CG == 2)
      CLQ_MX_MMA("2", "kind::mxf4nvf4.block_scale.scale_vec::4X");
    else
      CLQ_MX_MMA("1", "kind::mxf4nvf4.block_scale.scale_vec::4X");
  }
#undef CLQ_MX_MMA
}

// Instruction descriptor of the block-scaled kinds: E2M1 operands, K-major, K = 64;
// scale format E8M0 or E4M3; sf: the byte pair of a scale word that the MMA takes.
__host__ __device__ constexpr uint32_t idesc_mx(int fmt, uint32_t M, uint32_t N, uint32_t sf) {
  return (sf << 4) | (1u << 7) | (1u << 10) | ((N >> 3) << 17) |
         ((fmt == CLQ_MX_BLOCK32 ? 1u : 0u) << 23) | ((M >> 4) << 24) | (sf << 29);
}

__device__ __forceinline__ void stmatrix4_trans(uint32_t addr, const uint32_t (&o)[4]) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr),
               "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3])
               : "memory");
}

// A tile of the output: `n0` its first channel within its matrix, `expert`'s.
struct Tile {
  int n0, row0, rows, expert;
  // Columns that its MMAs make: a tile that ends early takes only the time of those (the
  // pair's CTAs hold half of them each).
  __device__ __forceinline__ int columns(int nt) const { return min(nt, (rows + 63) / 64 * 64); }
};

__device__ __forceinline__ uint4 select(bool c, const uint4& a, const uint4& b) {
  return make_uint4(c ? a.x : b.x, c ? a.y : b.y, c ? a.z : b.z, c ? a.w : b.w);
}

// Scale `byte` of block `blk` (of `blocks`) of a row of the codes that the epilogue makes;
// the last block's warp also zeroes the bytes behind it.
__device__ __forceinline__ void store_scale(const GemmArgs& g, int row, int blk, int blocks,
                                            uint32_t byte) {
  uint8_t* s = g.Ys + (static_cast<size_t>(row / kRowBlock) * g.y_chunks + (blk >> 2)) * 512 +
               (row & 31) * 16 + ((row >> 5) & 3) * 4;
  s[blk & 3] = static_cast<uint8_t>(byte);
  if (blk == blocks - 1)
    for (int q = (blk & 3) + 1; q < 4; ++q) s[q] = 0;
}

// One tile of the list into L1.
__device__ __forceinline__ void fetch_line(const RowTile* p) {
  int4 e;
  asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(e.x), "=r"(e.y), "=r"(e.z), "=r"(e.w)
               : "l"(p)
               : "memory");
}

template <int NT, int CG, bool GROUPED>
__device__ __forceinline__ Tile tile_at(const GemmArgs& g, int t, int tiles_n) {
  const int m = t / tiles_n;
  Tile r;
  r.n0 = (t - m * tiles_n) * (TN * CG);
  if (GROUPED) {
    // (an ordinary load: the plan may be written while this CTA waits for it, which a
    // read-only one must not be used for)
    const int4 e = reinterpret_cast<const int4*>(g.tiles)[m];
    r.expert = e.x;
    r.row0 = e.y;
    r.rows = e.z;
  } else {
    r.expert = 0;
    r.row0 = m * NT;
    r.rows = min(NT, g.M - r.row0);
  }
  return r;
}

// What becomes of a tile: stored as OutT, or rounded to OutT, put through an activation and
// quantized to codes with block scales (blocks of 32).
constexpr int EPI_STORE = 0;
constexpr int EPI_ACT = 1;     // CLQ_MX_ACT_NONE or _GELU: a channel a code
constexpr int EPI_SWIGLU = 2;  // 8 channels of the gate, 8 of the up half, and so on

template <typename OutT, int FMT, int NT, int CG, bool GROUPED, int EPI>
__global__ void __launch_bounds__(THREADS, 1)
    mx_gemm_kernel(const __grid_constant__ CUtensorMap mapW,
                   const __grid_constant__ CUtensorMap mapX,
                   const __grid_constant__ CUtensorMap mapSW,
                   const __grid_constant__ CUtensorMap mapSX,
                   const __grid_constant__ CUtensorMap mapY, GemmArgs g, int use_tma_store) {
  using C = Cfg<FMT, NT, CG>;
  constexpr int S = C::S;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Bars bars;
  uint8_t* smem = reinterpret_cast<uint8_t*>(
      (reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&bars.full[s], 1);
      mbar_init(&bars.empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&bars.acc_full[s], 1);
      mbar_init(&bars.acc_empty[s], CG * 4 * C::PARTS);
    }
    mbar_init(&bars.ov_empty, CG * 4);
    mbar_init(&bars.drained, 1);
    bars.abort = 0;
    fence_mbarrier_init();
  }
  if (warp == WARP_MMA) {
    tmem_alloc<CG>(&bars.tmem_slot, C::TMEM);
  }
  if (warp == WARP_TMA) {
    if (elect_one()) {
      prefetch_tensor_map(&mapW);
      prefetch_tensor_map(&mapX);
      prefetch_tensor_map(&mapSW);
      prefetch_tensor_map(&mapSX);
      if (use_tma_store) prefetch_tensor_map(&mapY);
    }
  }
  __syncwarp();  // the cluster barrier counts whole warps: none may come to it in parts
  tc_fence_before();
  if (CG == 2)
    cluster_sync();
  else
    __syncthreads();
  tc_fence_after();
  // The permit to allocate belongs to the pair: given up by one CTA while the other's
  // allocation is still on its way, it leaves that allocation waiting for ever (seen once
  // in 10^4 to 10^5 launches), so both have allocated first.
  if (warp == WARP_MMA) tmem_relinquish<CG>();
  const uint32_t tmem = bars.tmem_slot;
  const int nk = (g.K + KC - 1) / KC;
  const int tiles_n = (g.N + TN * CG - 1) / (TN * CG);
  // While the previous kernel finishes, this CTA's first weights are on their way into L2:
  // few rows meet many experts' weights, whose bytes are the work (8 tokens through 6 of 64
  // experts: 30.1 us, with these 27.3; a dense layer's weights are often in L2 already, and
  // the hints cost 1 x 4096 -> 16384 a microsecond).  The plan's list may still be in the
  // writing: whatever it holds by now, a hint changes no value, and the relaxed load leaves no
  // old line behind for the loads after the wait.
  if (GROUPED && NT <= 128 && warp == WARP_TMA) {
    if (elect_one()) {
      const int t = static_cast<int>(blockIdx.x);
      const int expert = min(max(ld_relaxed(&g.tiles[min(t / tiles_n, g.max_tiles - 1)].expert), 0),
                             g.experts - 1);
      const int n0 = t % tiles_n * TN;
      for (int kb = 0; kb < nk; ++kb) {
        tma_prefetch_2d(&mapW, kb * 128, expert * g.N + n0);
        tma_prefetch_2d(&mapSW, 0, (expert * g.w_blocks + n0 / kRowBlock) * g.chunks + kb * C::SC);
      }
    }
    __syncwarp();
  }
  pdl_wait();
  pdl_launch_dependents();

  volatile int32_t* abort = &bars.abort;
  const int unit = static_cast<int>(blockIdx.x) / CG;
  // this CTA's first tile on its way beside the list's length (the list has room for it)
  if (GROUPED) fetch_line(g.tiles + unit / tiles_n);
  const int tiles = (GROUPED ? *g.tile_count : (g.M + NT - 1) / NT) * tiles_n;
  const int units = static_cast<int>(gridDim.x) / CG;
  const int rank = CG == 2 ? static_cast<int>(cluster_ctarank()) : 0;

  if (warp == WARP_TMA) {
    if (elect_one()) {
      int it = 0, s = 0;
      uint32_t phase = 1;
      bool ok = true;
      const uint32_t full0 = CG == 2 ? cluster_addr(&bars.full[0], 0) : 0;
      for (int t = unit; t < tiles && ok; t += units) {
        const Tile T = tile_at<NT, CG, GROUPED>(g, t, tiles_n);
        const int n0 = T.n0 + rank * TN;
        const int wrow = T.expert * g.N + n0;
        const int xrow = T.row0 + (CG == 2 && rank != 0 ? T.columns(NT) / 2 : 0);
        const int wchunk = (T.expert * g.w_blocks + n0 / kRowBlock) * g.chunks;
        const int xchunk = T.row0 / kRowBlock * g.chunks;
        for (int kb = 0; kb < nk; ++kb, ++it) {
          if (!mbar_wait_bounded(&bars.empty[s], phase, abort, g.status, kWaitLimitNs)) {
            ok = false;
            break;
          }
          uint64_t* full = &bars.full[s];
          if (CG == 1 || rank == 0) mbar_arrive_expect_tx(full, C::TX);
          auto load = [&](int off, const CUtensorMap* map, int x, int y) {
            if constexpr (CG == 2)
              tma_load_2d_pair(smem + off, map, x, y, full0 + 8u * s);
            else
              tma_load_2d(smem + off, map, x, y, full);
          };
          load(C::OFF_A + s * C::A, &mapW, kb * 128, wrow);
          load(C::OFF_B + s * C::B, &mapX, kb * 128, xrow);
          load(C::OFF_SA + s * C::SA, &mapSW, 0, wchunk + kb * C::SC);
#pragma unroll
          for (int j = 0; j < C::XB; ++j)
            load(C::OFF_SB + s * C::SB + j * C::SC * 512, &mapSX, 0,
                 xchunk + j * g.chunks + kb * C::SC);
          if (++s == S) {
            s = 0;
            phase ^= 1;
          }
        }
      }
      // On an abort the copies in flight land before exit (a pair's second CTA, whose
      // copies complete on the leader's barriers, allows them a millisecond).
      if (!ok && rank != 0) {
        const uint64_t t0 = global_timer_ns();
        while (global_timer_ns() - t0 < 1000000ull) __nanosleep(1000);
      } else if (!ok) {
        for (int j = max(0, it - S); j < it; ++j)
          mbar_wait_bounded(&bars.full[j % S], (j / S) & 1, nullptr, nullptr, 10000000ull);
      }
    }
    __syncwarp();
  } else if (warp == WARP_MMA) {
    if (rank == 0 && elect_one()) {
      const uint64_t adesc = sw128_desc(smem_addr(smem + C::OFF_A));
      const uint64_t bdesc = sw128_desc(smem_addr(smem + C::OFF_B));
      const uint64_t sadesc = scale_desc(smem_addr(smem + C::OFF_SA));
      const uint64_t sbdesc = scale_desc(smem_addr(smem + C::OFF_SB));
      int s = 0, tc = 0;
      uint32_t phase = 0, sfbuf = 0;
      bool ok = true;
      for (int t = unit; t < tiles && ok; t += units, ++tc) {
        const Tile T = tile_at<NT, CG, GROUPED>(g, t, tiles_n);
        // a 64-row tile may be the second half of its scale block
        const uint32_t xcol = NT == 64 ? static_cast<uint32_t>(T.row0 & 64) / 32u : 0u;
        const uint32_t columns = static_cast<uint32_t>(T.columns(NT));
        const int buf = tc & 1;
        if (!mbar_wait_bounded(&bars.acc_empty[buf], ((tc >> 1) & 1) ^ 1, abort, g.status,
                               kWaitLimitNs) ||
            (C::OV > 0 && tc > 0 &&
             !mbar_wait_bounded(&bars.ov_empty, (tc - 1) & 1, abort, g.status, kWaitLimitNs))) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t d = tmem + buf * (NT - C::OV);
        for (int kb = 0; kb < nk; ++kb) {
          if (!mbar_wait_bounded(&bars.full[s], phase, abort, g.status, kWaitLimitNs)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t sfa = tmem + C::OFF_SF + sfbuf * C::SF;
          const uint32_t sfb = sfa + C::SFA;
#pragma unroll
          for (int c = 0; c < C::SC; ++c) {
            cp_scales<CG>(sfa + 4 * c, sadesc + static_cast<uint32_t>((s * C::SA + c * 512) / 16));
#pragma unroll
            for (int j = 0; j < C::XB; ++j)
              cp_scales<CG>(sfb + 4 * (c * C::XB + j),
                            sbdesc + static_cast<uint32_t>((s * C::SB + (j * C::SC + c) * 512) / 16));
          }
          const uint64_t a0 = adesc + static_cast<uint32_t>(s * (C::A / 16));
          const uint64_t b0 = bdesc + static_cast<uint32_t>(s * (C::B / 16));
          // MMAs of 64 codes; past the end of a row there are codes of zero, but no scales
          const int steps = min(KC / 64, (g.K - kb * KC + 63) / 64);
#pragma unroll
          for (int k = 0; k < KC / 64; ++k) {
            if (k < steps) {
              const int c = FMT == CLQ_MX_BLOCK32 ? k >> 1 : k;
              const uint32_t sf = FMT == CLQ_MX_BLOCK32 ? (k & 1) * 2 : 0;
              mma_mx<FMT, CG>(d, a0 + k * 2, b0 + k * 2, idesc_mx(FMT, TN * CG, columns, sf),
                              sfa + 4 * c, sfb + 4 * C::XB * c + xcol, (kb | k) == 0 ? 0u : 1u);
            }
          }
          mma_commit<CG>(&bars.empty[s]);
          if (C::NSF == 2) sfbuf ^= 1;
          if (++s == S) {
            s = 0;
            phase ^= 1;
          }
        }
        if (ok) mma_commit<CG>(&bars.acc_full[buf]);
      }
      mma_commit<CG>(&bars.drained);
      mbar_wait_bounded(&bars.drained, 0, nullptr, nullptr, 10000000ull);
    } else if (CG == 2 && rank == 1 && elect_one()) {
      // The leader's commits signal this CTA's barriers too: it stays for the last one.
      mbar_wait_bounded(&bars.drained, 0, abort, nullptr, 2 * kWaitLimitNs);
    }
    __syncwarp();
  } else if (warp < 4 || C::PARTS == 2) {
    const int quarter = warp & 3;
    const int part = warp < 4 ? 0 : 1;
    uint8_t* staging = smem + C::OFF_EPI + (part * 4 + quarter) * 2 * EPI_BYTES;
    const uint32_t empty0 = CG == 2 ? cluster_addr(&bars.acc_empty[0], 0) : 0;
    const uint32_t ov0 = CG == 2 ? cluster_addr(&bars.ov_empty, 0) : 0;
    constexpr int NB = C::NCOL / EPI_COLS;  // blocks of 32 rows of X
    const int col0 = part * C::NCOL;        // this warp's tile columns
    // A tile's channel data (channels 8 k + lane / 4 of a thread's fragments) and row
    // scales (row 32 j + lane of the warp's columns), loaded a tile ahead.
    float next_w[4], next_b[4], next_x[NB];
    auto load_scales = [&](int t) {
      if (t >= tiles) return;
      const Tile T = tile_at<NT, CG, GROUPED>(g, t, tiles_n);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int n = T.n0 + rank * TN + quarter * 32 + 8 * k + (lane >> 2);
        const bool in = n < g.N;
        const size_t at = static_cast<size_t>(T.expert) * g.N + n;
        next_w[k] = FMT == CLQ_MX_BLOCK16 ? (in ? __ldg(g.s_w + at) : 0.f) : 1.f;
        next_b[k] = in && g.bias != nullptr
                        ? Num<OutT>::to_f(__ldg(static_cast<const uint16_t*>(g.bias) + at))
                        : 0.f;
      }
      if (FMT == CLQ_MX_BLOCK16) {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const int i = col0 + 32 * j + lane;
          next_x[j] = i < T.rows ? __ldg(g.s_x + T.row0 + i) : 0.f;
        }
      }
    };
    load_scales(unit);
    int tc = 0, turn = 0;
    for (int t = unit; t < tiles; t += units, ++tc) {
      const Tile T = tile_at<NT, CG, GROUPED>(g, t, tiles_n);
      const int n0 = T.n0 + rank * TN + quarter * 32;  // this warp's channels
      const int buf = tc & 1;
      float sw[4], bi[4], sx[NB];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        sw[k] = next_w[k] * g.inv_b;
        bi[k] = next_b[k];
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) sx[j] = FMT == CLQ_MX_BLOCK16 ? next_x[j] : 1.f;
      load_scales(t + units);
      bool ok = mbar_wait_bounded(&bars.acc_full[buf], (tc >> 1) & 1, abort, g.status,
                                  kWaitLimitNs);
      ok = __all_sync(0xffffffffu, ok);
      // both warps of a pair go on or neither does: one that gave up would leave the other
      // at its barrier (8192 tokens through gated experts: 282.3 us without this, 282.9 with)
      if (EPI == EPI_SWIGLU) ok = pair_all(1 + part * 2 + (quarter >> 1), ok);
      if (!ok) break;
      tc_fence_after();
      const uint32_t lane_base =
          tmem + buf * (NT - C::OV) + (static_cast<uint32_t>(quarter * 32) << 16);
      const int live = n0 < g.N ? max(0, min(NB, (T.rows - col0 + 31) / 32)) : 0;
      // Two blocks at a time leave tensor memory, and the accumulator goes back as soon as
      // the last ones have, before they are scaled or stored.  The columns that the two
      // accumulators share are the first buffer's last and the other's first: the warps that
      // hold them begin there and release them by themselves.
      const bool shares = C::OV > 0 && part == (buf == 0 ? 1 : 0);
      const bool down = shares && buf == 0;
      auto release = [&](uint64_t* bar, uint32_t remote) {
        tc_fence_before();
        __syncwarp();
        if (elect_one()) {
          if (CG == 2)
            mbar_arrive_cluster(remote);
          else
            mbar_arrive(bar);
        }
      };
      constexpr int STEP = NB >= 2 ? 2 : 1;
#pragma unroll
      for (int j0 = 0; j0 < NB; j0 += STEP) {
        uint32_t r[STEP][2][16];  // channels 0 .. 15 and 16 .. 31 of a block
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
          const int blk = down ? NB - 1 - j0 - i : j0 + i;
          if (blk < live) {
            const uint32_t at = lane_base + col0 + blk * EPI_COLS;
            gemm::tmem_ld_frag(at, r[i][0]);
            gemm::tmem_ld_frag(at + (16u << 16), r[i][1]);
          }
        }
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
          gemm::tmem_ld_wait_tie(r[i][0]);
          gemm::tmem_ld_wait_tie(r[i][1]);
        }
        if (C::OV > 0 && shares && 32 * j0 < C::OV && C::OV <= 32 * (j0 + STEP))
          release(&bars.ov_empty, ov0);
        if (j0 + STEP == NB) release(&bars.acc_empty[buf], empty0 + 8u * buf);
#pragma unroll
        for (int i = 0; i < STEP; ++i) {
          const int blk = down ? NB - 1 - j0 - i : j0 + i;
          if (blk >= live) continue;
          const float sxv = down ? sx[NB - 1 - j0 - i] : sx[j0 + i];
          uint8_t* stage = staging + turn * EPI_BYTES;
          const uint32_t stage_addr = smem_addr(stage);
          // the store before last has read this buffer
          if (EPI == EPI_STORE && use_tma_store && elect_one()) gemm::bulk_wait_read<1>();
          __syncwarp();
#pragma unroll
          for (int q = 0; q < 4; ++q) {  // rows 8 q + 2 (lane % 4), + 1
            float2 x2 = make_float2(1.f, 1.f);
            if (FMT == CLQ_MX_BLOCK16)
              x2 = make_float2(__shfl_sync(0xffffffffu, sxv, 8 * q + 2 * (lane & 3)),
                               __shfl_sync(0xffffffffu, sxv, 8 * q + 2 * (lane & 3) + 1));
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float2 acc =
                  make_float2(__uint_as_float(r[i][k >> 1][4 * q + 2 * (k & 1)]),
                              __uint_as_float(r[i][k >> 1][4 * q + 2 * (k & 1) + 1]));
              float2 s2 = make_float2(sw[k], sw[k]);
              if (FMT == CLQ_MX_BLOCK16) s2 = __fmul2_rn(s2, x2);
              const float2 v = __ffma2_rn(acc, s2, make_float2(bi[k], bi[k]));
              o[k] = Num<OutT>::pack2(v.x, v.y);
            }
            stmatrix4_trans(stage_addr + gemm::staged_chunk(8 * q + (lane & 7), lane >> 3), o);
          }
          const int row = T.row0 + col0 + 32 * blk, rows = T.rows - col0 - 32 * blk;
          if constexpr (EPI == EPI_STORE) {
            if (use_tma_store) {
              fence_proxy_async_smem();
              __syncwarp();
              if (elect_one()) {
                gemm::tma_store_2d(&mapY, stage, n0, row);
                gemm::bulk_commit();
              }
            } else {
              __syncwarp();
              gemm::store_block_direct(stage_addr, lane, row, row + rows, n0, g.N,
                                       static_cast<uint16_t*>(g.Y));
            }
          } else if constexpr (EPI == EPI_ACT) {
            __syncwarp();
            // a lane a row: its 32 channels are one block
            float v[32];
#pragma unroll
            for (int c = 0; c < 4; ++c)
              unpack8<OutT>(*reinterpret_cast<const uint4*>(stage + gemm::staged_chunk(lane, c)),
                            v + 8 * c);
            if (g.act == CLQ_MX_ACT_GELU) {
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const float2 y = gelu_fast(make_float2(v[i], v[i + 1]));
                v[i] = y.x;
                v[i + 1] = y.y;
              }
            }
            float most = fabsf(v[0]);
#pragma unroll
            for (int i = 1; i < 31; i += 2) most = absmax3(most, v[i], v[i + 1]);
            most = absmax3(most, v[31], v[31]);
            const uint32_t byte = e8m0_byte(__float_as_uint(most));
            const float inv = e8m0_inverse(byte);
            scale_by<32>(v, inv);
            uint32_t code[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) code[c] = byte == 255u ? 0u : e2m1x8(v + 8 * c);
            if (lane < rows) {
              *reinterpret_cast<uint4*>(g.Yq + static_cast<size_t>(row + lane) * (g.N / 2) + n0 / 2) =
                  make_uint4(code[0], code[1], code[2], code[3]);
              store_scale(g, row + lane, n0 / 32, g.N / 32, byte);
            }
          } else {
            // Two warps hold a block of 32 (64 channels).  Both have staged their half; each
            // then works on half of the rows, two lanes a row.  One barrier a block: the
            // buffers alternate.
            pair_barrier(1 + part * 2 + (quarter >> 1));
            const int half = lane & 1, m = 16 * (quarter & 1) + (lane >> 1);
            const uint8_t* from = smem + C::OFF_EPI +
                                  ((part * 4 + (quarter & 2) + half) * 2 + turn) * EPI_BYTES;
            uint4 p[4];
#pragma unroll
            for (int c = 0; c < 4; ++c)  // the two lanes' chunks on different banks
              p[c] = *reinterpret_cast<const uint4*>(from + gemm::staged_chunk(m, c ^ (2 * half)));
            float v[16];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float gate[8], up[8];
              unpack8<OutT>(select(half, p[(2 * h) ^ 2], p[2 * h]), gate);
              unpack8<OutT>(select(half, p[(2 * h + 1) ^ 2], p[2 * h + 1]), up);
#pragma unroll
              for (int i = 0; i < 8; i += 2) {
                const float2 y = swiglu_fast(make_float2(gate[i], gate[i + 1]),
                                             make_float2(up[i], up[i + 1]));
                v[8 * h + i] = y.x;
                v[8 * h + i + 1] = y.y;
              }
            }
            float most = fabsf(v[0]);
#pragma unroll
            for (int i = 1; i < 15; i += 2) most = absmax3(most, v[i], v[i + 1]);
            most = absmax3(most, v[15], __shfl_xor_sync(0xffffffffu, absmax3(most, v[15], v[15]), 1));
            const uint32_t byte = e8m0_byte(__float_as_uint(most));
            const float inv = e8m0_inverse(byte);
            scale_by<16>(v, inv);
            uint2 code = make_uint2(e2m1x8(v), e2m1x8(v + 8));
            if (byte == 255u) code = make_uint2(0, 0);
            if (m < rows) {
              const int f0 = (T.n0 + rank * TN + (quarter & 2) * 32) / 2;  // the block's first code
              *reinterpret_cast<uint2*>(g.Yq + static_cast<size_t>(row + m) * (g.N / 4) + f0 / 2 +
                                        8 * half) = code;
              if (half == 0) store_scale(g, row + m, f0 / 32, g.N / 64, byte);
            }
          }
          turn ^= 1;
        }
      }
    }
    if (EPI == EPI_STORE && elect_one()) gemm::bulk_wait_all();
    __syncwarp();
  }
  tc_fence_before();
  if (CG == 2)
    cluster_sync();
  else
    __syncthreads();
  if (warp == WARP_MMA) {
    tc_fence_after();
    tmem_dealloc<CG>(tmem, C::TMEM);
  }
}

struct GemmMaps {
  CUtensorMap W, X, SW, SX, Y;
};

template <typename OutT, int FMT, int NT, int CG, bool GROUPED, int EPI>
cudaError_t launch_gemm_t(const GemmMaps& m, const GemmArgs& g, int use_tma_store, int grid,
                          cudaStream_t st) {
  using C = Cfg<FMT, NT, CG>;
  auto k = mx_gemm_kernel<OutT, FMT, NT, CG, GROUPED, EPI>;
  constexpr size_t smem = C::BYTES + 1024;
  cudaError_t e = kernel_setup(reinterpret_cast<const void*>(k), smem, THREADS, nullptr);
  if (e != cudaSuccess) return e;
  return launch_cluster_pdl(k, grid, CG, THREADS, smem, st, m.W, m.X, m.SW, m.SX, m.Y, g,
                            use_tma_store);
}

// Instantiated for each output type and format in mx_gemm_*.cu.  A plan's tiles have up to
// 128 or 256 rows; the epilogues that quantize go with them in blocks of 32.
template <typename OutT, int FMT, int NT, int CG>
cudaError_t launch_grouped(const GemmMaps& m, const GemmArgs& g, int use_tma_store, int grid,
                           cudaStream_t st) {
  if constexpr (FMT == CLQ_MX_BLOCK32) {
    if (g.Yq != nullptr)
      return g.act == CLQ_MX_ACT_SWIGLU
                 ? launch_gemm_t<OutT, FMT, NT, CG, true, EPI_SWIGLU>(m, g, 0, grid, st)
                 : launch_gemm_t<OutT, FMT, NT, CG, true, EPI_ACT>(m, g, 0, grid, st);
  }
  return launch_gemm_t<OutT, FMT, NT, CG, true, EPI_STORE>(m, g, use_tma_store, grid, st);
}

template <typename OutT, int FMT>
cudaError_t launch_gemm_tiles(const GemmMaps& m, const GemmArgs& g, TileShape t, bool grouped,
                              int use_tma_store, int grid, cudaStream_t st) {
  if (grouped) {
    if (t.nt == 32) return launch_grouped<OutT, FMT, 32, 1>(m, g, use_tma_store, grid, st);
    if (t.nt == 128) return launch_grouped<OutT, FMT, 128, 1>(m, g, use_tma_store, grid, st);
    return launch_grouped<OutT, FMT, 256, 2>(m, g, use_tma_store, grid, st);
  }
#define CLQ_MX_GO(NT, CG) \
  return launch_gemm_t<OutT, FMT, NT, CG, false, EPI_STORE>(m, g, use_tma_store, grid, st)
  switch (t.nt) {
    case 32: CLQ_MX_GO(32, 1);
    case 64: CLQ_MX_GO(64, 1);
    case 128:
      if (t.cg == 1) CLQ_MX_GO(128, 1);
      CLQ_MX_GO(128, 2);
    default:
      if (t.cg == 1) CLQ_MX_GO(256, 1);
      CLQ_MX_GO(256, 2);
  }
#undef CLQ_MX_GO
}

using GemmFn = cudaError_t (*)(const GemmMaps&, const GemmArgs&, TileShape, bool, int, int, cudaStream_t);
cudaError_t gemm_block32_f16(const GemmMaps&, const GemmArgs&, TileShape, bool, int, int, cudaStream_t);
cudaError_t gemm_block32_bf16(const GemmMaps&, const GemmArgs&, TileShape, bool, int, int, cudaStream_t);
cudaError_t gemm_block16_f16(const GemmMaps&, const GemmArgs&, TileShape, bool, int, int, cudaStream_t);
cudaError_t gemm_block16_bf16(const GemmMaps&, const GemmArgs&, TileShape, bool, int, int, cudaStream_t);

}  // namespace mx
}  // namespace clq
