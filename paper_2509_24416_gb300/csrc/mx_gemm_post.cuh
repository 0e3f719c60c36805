// The product's epilogue with an activation and a residual (included by mx_gemm.cuh).
//
// Y = OutT(act(acc s + bias) + residual), in fp32 up to the one rounding: a warp takes 32 channels
// of 32 rows of X at a time out of tensor memory.  Their block of the residual, which the warp
// asked for a block ahead, lies by then in the staging buffer from which the result will leave, so
// that both travel in tensor copies and meet the accumulators' fragments by ldmatrix and stmatrix at
// the same places.  A tile's blocks are dealt to the warps of a quarter of its channels in turn, a
// tile's first block to another one each time, since three warps do not share eight blocks evenly.
//
// Few rows with few channels: up to eight CTAs, a cluster, share a tile's K steps (pick_row_tile has the
// rule and the times).  The first waits for the others' fp32 sums, which st.async writes where its
// operands were and counts on a barrier, and adds them up in the order of the shares, so that the bits
// are the same every time.
//
// What bounds it is the epilogue warps' instructions where K is short (a value costs 5 in the plain
// epilogue, 9 with a residual, 14 with GELU), the MMAs where it is long.  Measured, us, E4M3
// 8192 x 1152 -> 3456 with GELU / a residual / both, plain 28: 32 / 32 / 37.  With a shorter GELU (the
// logistic one named at gelu_post): twelve warps of 128 registers 31 / 32 / 34; eight, all blocks of a tile unrolled, 43 / 36 / 53 (fetching instructions); sixteen of
// 96 registers, with a stage less of operands, 33 / 36 / 37; sixteen, blocks of 16 rows, 36 / 36 /
// 42; with one staging buffer 37 / 45 / 51 (a store's read waits behind the operands' copies);
// residuals by loads of the lanes and results by their stores 46 / 50 / 61; residuals prefetched
// into L2 a tile ahead 33 / 39 / 38.
#pragma once

namespace clq {
namespace mx {

// Two 8 x 8 matrices: lanes 0 .. 15 give the addresses.
__device__ __forceinline__ void stmatrix2_trans(uint32_t addr, uint32_t o0, uint32_t o1) {
  asm volatile("stmatrix.sync.aligned.m8n8.x2.trans.shared.b16 [%0], {%1, %2};" ::"r"(addr), "r"(o0),
               "r"(o1)
               : "memory");
}

// What stmatrix4_trans / stmatrix2_trans would store from the same lanes.
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&o)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldmatrix2_trans(uint32_t addr, uint32_t& o0, uint32_t& o1) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0, %1}, [%2];"
               : "=r"(o0), "=r"(o1)
               : "r"(addr)
               : "memory");
}

// Byte offset of 16-byte chunk q (8 columns, 0 or 1) of row r in a staging buffer of 16 columns:
// the tensor map's 32-byte swizzle.
__device__ __forceinline__ int staged_chunk16(int r, int q) {
  return r * 32 + ((q ^ ((r >> 2) & 1)) << 4);
}

template <typename T>
__device__ __forceinline__ float2 add2(float2 v, uint32_t r) {
  return __fadd2_rn(v, make_float2(Num<T>::to_f(static_cast<uint16_t>(r)),
                                   Num<T>::to_f(static_cast<uint16_t>(r >> 16))));
}

__device__ __forceinline__ float max_nan(float x, float y) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
  return r;
}

// GELU of an accumulator, which may be anything, as max(x, 0) - |x| 2^N(-|x|): N, log2 of the normal
// distribution function, of degree 8 (iteratively reweighted least squares down to -13).  Within 2^-18 of
// itself and 2^-22 |x|, and, so that a 16-bit result has its digits far down the negative side too, within 2^-13
// of itself to x = -6 and 2^-10 to -12.9 (a quarter of half a step of fp16, which ends there, and of bf16) and
// 2^-122 behind that.  Infinity is its own value, minus infinity 0, NaN NaN.
// a = |x| / 16, at most 1 (two operations in one instruction of the multiply-add pipe; by minima 33.1 us, 72.3, for 32.5,
// 69.2), 16 in the exponential.  Eight instructions a value.  Measured, us, E4M3 8192 x 1152 -> 3456 / blocks of
// 32 16384 x 1152 -> 4608: this 32.5 / 69.2; gelu_fast with the same ends, 12 1/2 instructions, 37.4 / 84.7; a logistic form
// that is exact to 2^-22 |x| alone, five times too large at x = -5.5, 31.7 / 67.6.
__device__ __forceinline__ float2 gelu_post(float2 x) {
  const float2 a = make_float2(__saturatef(fabsf(x.x) * 0.0625f), __saturatef(fabsf(x.y) * 0.0625f));
  float2 p = __ffma2_rn(a, both(206.0473175048828f), both(-734.8352661132812f));
  p = __ffma2_rn(p, a, both(1125.03515625f));
  p = __ffma2_rn(p, a, both(-982.8634033203125f));
  p = __ffma2_rn(p, a, both(554.6920776367188f));
  p = __ffma2_rn(p, a, both(-220.39712524414062f));
  p = __ffma2_rn(p, a, both(-117.40802764892578f));
  p = __ffma2_rn(p, a, both(-18.419126510620117f));
  p = __ffma2_rn(p, a, both(3.0000009536743164f));
  const float2 h = make_float2(exp2_fast(p.x), exp2_fast(p.y));
  return make_float2(__fmaf_rn(-a.x, h.x, max_nan(x.x, 0.f)), __fmaf_rn(-a.y, h.y, max_nan(x.y, 0.f)));
}

// A block of the residual (`rows` of its rows from row0, columns col0 .. + W - 1) into a staging
// buffer where its rows or its address rule the tensor copy out: a lane a column, eight rows under
// way.
template <int W>
__device__ __forceinline__ void load_residual_direct(uint8_t* stage, int lane, const GemmArgs& g,
                                                     int row0, int rows, int col0, int columns) {
  const int c = W == 32 ? lane : lane & 15, r0 = W == 32 ? 0 : lane >> 4;
  constexpr int STEP = W == 32 ? 1 : 2;
  const bool in = col0 + c < columns;
  const uint16_t* src = static_cast<const uint16_t*>(g.residual) +
                        static_cast<size_t>(row0 + r0) * g.ldr + col0 + c;
#pragma unroll
  for (int i0 = 0; i0 < EPI_ROWS / STEP; i0 += 8) {
    uint16_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + (i0 + i) * STEP;
      v[i] = in && r < rows ? src[static_cast<size_t>((i0 + i) * STEP) * g.ldr] : 0;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = r0 + (i0 + i) * STEP;
      const int at = W == 32 ? gemm::staged_chunk(r, c >> 3) : staged_chunk16(r, c >> 3);
      *reinterpret_cast<uint16_t*>(stage + at + (c & 7) * 2) = v[i];
    }
  }
}

// Four values to another CTA of the cluster, counted there on its barrier.
__device__ __forceinline__ void send4(uint32_t addr, const uint32_t* v, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(addr),
               "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(bar)
               : "memory");
}

template <typename OutT, int FMT, int NT, int CG, int EPI>
__device__ __forceinline__ void post_tiles(Bars& bars, uint8_t* smem, const CUtensorMap& mapY,
                                           const CUtensorMap& mapR, const GemmArgs& g,
                                           int use_tma_store, uint32_t tmem, int unit, int units,
                                           int tiles, int tiles_n, int rank, int split, int share,
                                           int warp, int lane) {
  using C = Cfg<FMT, NT, CG, EPI>;
  constexpr int OUT = C::OUT, PARTS = C::PARTS;
  constexpr int BLOCKS = NT / EPI_ROWS;  // of 32 rows of X in a tile
  constexpr int OVB = C::OV / EPI_ROWS;  // of them in the columns that the accumulators share
  static_assert(POST_RING == 2, "buffers in turn");
  volatile int32_t* abort = &bars.abort;
  const int quarter = warp & 3;
  const int part = warp < 4 ? 0 : (warp - WARP_MMA - 1) / 4 + 1;
  const int channel0 = rank * TN + quarter * 32;  // this warp's within a tile
  const int columns = EPI == EPI_GATED ? g.N / 2 : g.N;
  uint8_t* staging = smem + C::OFF_EPI + (part * 4 + quarter) * POST_RING * C::SLOT;
  uint64_t* res_bar = bars.residual[part * 4 + quarter];
  const bool residual = g.residual != nullptr && share == 0, copied = residual && g.tma_residual;
  // A tile as this warp sees it: its rows (none without channels), the first column of Y, and the
  // order of its blocks: from the last one down where the columns that the two accumulators share
  // are its last, from the first one up where they are its first.  The warp's own are number
  // `first`, first + PARTS, ..
  struct Share {
    int row, rows, x, first, down;
    __device__ __forceinline__ int block(int o) const { return down ? BLOCKS - 1 - o : o; }
    // its next block with rows, from number o on
    __device__ __forceinline__ int from(int o) const {
      while (o < BLOCKS && EPI_ROWS * block(o) >= rows) o += PARTS;
      return o;
    }
  };
  auto release = [&](uint64_t* bar) {
    tc_fence_before();
    __syncwarp();
    if (elect_one()) {
      if (CG == 2)
        mbar_arrive_cluster(cluster_addr(bar, 0));
      else
        mbar_arrive(bar);
    }
  };
  // Block number o of the residual into staging buffer `slot`, and the row scales of its rows.
  float next_x = 0.f;
  bool asked = false;
  auto ask = [&](const Share& s, int o, int slot) {
    asked = o < BLOCKS;
    if (!asked) return;
    const int r = EPI_ROWS * s.block(o);
    if (FMT == CLQ_MX_BLOCK16) next_x = r + lane < s.rows ? __ldg(g.s_x + s.row + r + lane) : 0.f;
    if (copied) {
      if (elect_one()) {
        mbar_arrive_expect_tx(&res_bar[slot], C::SLOT);
        tma_load_2d(staging + slot * C::SLOT, &mapR, s.x, s.row + r, &res_bar[slot]);
      }
      __syncwarp();
    } else if (residual) {
      load_residual_direct<OUT>(staging + slot * C::SLOT, lane, g, s.row + r, s.rows - r, s.x, columns);
      __syncwarp();
    }
  };

  // A tile's channel data (channels 8 k + lane / 4 of a thread's fragments), loaded a tile ahead.
  float next_w[4], next_b[4];
  Share next{0, 0, 0, 0, 0};
  auto look = [&](int t, int tc) {
    next.rows = 0;
    if (t >= tiles) return;
    const Tile T = tile_at<NT, CG, false>(g, t, tiles_n);
    const int n0 = T.n0 + channel0;
    next.row = T.row0;
    next.rows = n0 < g.N ? T.rows : 0;
    next.x = first_column(n0, EPI == EPI_GATED);
    next.down = C::OV > 0 && (tc & 1) == 0;
    next.first = static_cast<unsigned>(part + tc) % PARTS;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int n = n0 + 8 * k + (lane >> 2);
      const bool in = n < g.N;
      next_w[k] = FMT == CLQ_MX_BLOCK16 ? (in ? __ldg(g.s_w + n) : 0.f) : 1.f;
      next_b[k] = in && g.bias != nullptr
                      ? Num<OutT>::to_f(__ldg(static_cast<const uint16_t*>(g.bias) + n))
                      : 0.f;
    }
  };
  look(unit, 0);
  int tc = 0, slot = 0;
  uint32_t phase = 0;
  for (int t = unit; t < tiles; t += units, ++tc) {
    const Share now = next;
    const int buf = tc & 1;
    float sw[4], bi[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      sw[k] = next_w[k] * g.inv_b;
      bi[k] = next_b[k];
    }
    look(t + units, tc + 1);
    if (!asked) {  // the first tile, or one behind a tile without rows here
      if (residual && use_tma_store && elect_one()) gemm::bulk_wait_read<0>();
      __syncwarp();
      ask(now, now.from(now.first), slot);
    }
    const bool ok = mbar_wait_bounded(&bars.acc_full[buf], (tc >> 1) & 1, abort, g.status, kWaitLimitNs);
    if (!__all_sync(0xffffffffu, ok)) break;
    tc_fence_after();
    const uint32_t acc = tmem + buf * (NT - C::OV) + (static_cast<uint32_t>(quarter * 32) << 16);
    // Of CTAs that share the tile, the first adds up what the others send it, in their order, and
    // goes on; its operands' buffers take it as soon as its own MMAs are done.  Both barriers hand
    // shared memory from one CTA to another, so both count at the cluster's scope.
    if (C::JOIN && split > 1) {
      if (share == 0 && warp == 0 && lane > 0 && lane < split)
        mbar_arrive_cluster_release(cluster_addr(&bars.go, lane));
      const bool there = mbar_wait_bounded<true>(share == 0 ? &bars.joined : &bars.go, 0, abort, g.status, kWaitLimitNs);
      if (!__all_sync(0xffffffffu, there)) break;
      if (share > 0) {
        const uint32_t bar = cluster_addr(&bars.joined, 0);
        const uint32_t to = cluster_addr(smem + (share - 1) * C::PARTIAL + quarter * 4096 + lane * 16, 0);
        for (int blk = part; blk < BLOCKS; blk += PARTS) {
          uint32_t r[2][16];
          gemm::tmem_ld_frag(acc + blk * EPI_ROWS, r[0]);
          gemm::tmem_ld_frag(acc + blk * EPI_ROWS + (16u << 16), r[1]);
          gemm::tmem_ld_wait_tie(r[0]);
          gemm::tmem_ld_wait_tie(r[1]);
#pragma unroll
          for (int i = 0; i < 8; ++i) send4(to + blk * 16384 + i * 512, &r[i >> 2][4 * (i & 3)], bar);
        }
        break;
      }
    }
#pragma unroll 1
    for (int o = now.first; o < BLOCKS; o += PARTS) {
      const int blk = now.block(o);
      const bool live = EPI_ROWS * blk < now.rows;
      uint32_t r[2][16];  // channels 0 .. 15 and 16 .. 31
      if (live) {
        gemm::tmem_ld_frag(acc + blk * EPI_ROWS, r[0]);
        gemm::tmem_ld_frag(acc + blk * EPI_ROWS + (16u << 16), r[1]);
      }
      gemm::tmem_ld_wait_tie(r[0]);
      gemm::tmem_ld_wait_tie(r[1]);
      if (C::JOIN && split > 1 && live) {
        const uint8_t* from = smem + blk * 16384 + quarter * 4096 + lane * 16;
#pragma unroll 1
        for (int q = 1; q < split; ++q, from += C::PARTIAL) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 p = *reinterpret_cast<const float4*>(from + i * 512);
            uint32_t* v = &r[i >> 2][4 * (i & 3)];
            v[0] = __float_as_uint(__fadd_rn(__uint_as_float(v[0]), p.x));
            v[1] = __float_as_uint(__fadd_rn(__uint_as_float(v[1]), p.y));
            v[2] = __float_as_uint(__fadd_rn(__uint_as_float(v[2]), p.z));
            v[3] = __float_as_uint(__fadd_rn(__uint_as_float(v[3]), p.w));
          }
        }
      }
      if (C::OV > 0 && o < OVB) release(&bars.ov_empty);
      if (o + PARTS >= BLOCKS) release(&bars.acc_empty[buf]);
      if (!live) continue;
      uint8_t* stage = staging + slot * C::SLOT;
      const uint32_t stage_addr = smem_addr(stage);
      const int row = now.row + EPI_ROWS * blk;
      const float sxv = next_x;
      if (use_tma_store) {
        // the other buffer's store has read it (the next block of the residual may go there), or
        // this one's last store has
        if (elect_one()) {
          if (residual)
            gemm::bulk_wait_read<0>();
          else
            gemm::bulk_wait_read<1>();
        }
        __syncwarp();
      }
      const int o2 = now.from(o + PARTS);
      if (o2 < BLOCKS)
        ask(now, o2, slot ^ 1);
      else
        ask(next, next.from(next.first), slot ^ 1);
      if (copied) mbar_wait_bounded(&res_bar[slot], phase, abort, g.status, kWaitLimitNs);
#pragma unroll
      for (int q = 0; q < 4; ++q) {  // rows 8 q + 2 (lane % 4), + 1
        float2 x2 = make_float2(1.f, 1.f);
        if (FMT == CLQ_MX_BLOCK16)
          x2 = make_float2(__shfl_sync(0xffffffffu, sxv, 8 * q + 2 * (lane & 3)),
                           __shfl_sync(0xffffffffu, sxv, 8 * q + 2 * (lane & 3) + 1));
        // The residual's fragments on their way before the activation; zeros where there is none, so that
        // they have a value on either path (4096 x 2048 -> 8192 in blocks of 16 with GELU and a residual 43.2
        // us for 44.5; the gated ones' so 33 for 32 without a residual).
        uint32_t at = 0, w[4] = {0u, 0u, 0u, 0u};
        if constexpr (EPI != EPI_GATED) {
          at = stage_addr + gemm::staged_chunk(8 * q + (lane & 7), lane >> 3);
          if (residual) ldmatrix4_trans(at, w);
        }
        float2 y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 a = make_float2(__uint_as_float(r[k >> 1][4 * q + 2 * (k & 1)]),
                                       __uint_as_float(r[k >> 1][4 * q + 2 * (k & 1) + 1]));
          float2 s2 = make_float2(sw[k], sw[k]);
          if (FMT == CLQ_MX_BLOCK16) s2 = __fmul2_rn(s2, x2);
          y[k] = __ffma2_rn(a, s2, make_float2(bi[k], bi[k]));
        }
        if constexpr (EPI == EPI_GATED) {
          // gate and up half of a column are two fragments of one thread
          at = stage_addr + staged_chunk16(8 * q + (lane & 7), (lane >> 3) & 1);
          float2 p0 = swiglu_fast(y[0], y[1]), p1 = swiglu_fast(y[2], y[3]);
          if (residual) {
            uint32_t o0, o1;
            ldmatrix2_trans(at, o0, o1);
            p0 = add2<OutT>(p0, o0);
            p1 = add2<OutT>(p1, o1);
          }
          stmatrix2_trans(at, Num<OutT>::pack2(p0.x, p0.y), Num<OutT>::pack2(p1.x, p1.y));
        } else {
          if (EPI == EPI_GELU) {
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = gelu_post(y[k]);
          }
          if (residual) {
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = add2<OutT>(y[k], w[k]);
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) w[k] = Num<OutT>::pack2(y[k].x, y[k].y);
          stmatrix4_trans(at, w);
        }
      }
      if (use_tma_store) {
        fence_proxy_async_smem();
        __syncwarp();
        if (elect_one()) {
          gemm::tma_store_2d(&mapY, stage, now.x, row);
          gemm::bulk_commit();
        }
      } else {
        __syncwarp();
        gemm::store_block_direct(stage_addr, lane, row, now.row + now.rows, now.x, g.N,
                                 static_cast<uint16_t*>(g.Y));
        __syncwarp();
      }
      slot ^= 1;
      if (slot == 0) phase ^= 1;
    }
  }
  // (on an abort, a block of the residual in flight lands before the CTA exits)
  if (copied && asked) mbar_wait_bounded(&res_bar[slot], phase, nullptr, nullptr, 10000000ull);
  if (elect_one()) gemm::bulk_wait_all();
  __syncwarp();
}

}  // namespace mx
}  // namespace clq
