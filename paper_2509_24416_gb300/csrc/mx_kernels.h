// Host-side launch interface of the microscaled kernels (mx_*.cu).
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>

#include "../../include/clq_mx.h"
#include "clq_kernels.h"

namespace clq {
namespace mx {

constexpr int kRowBlock = 128;  // rows of a scale block

__host__ __device__ inline int block_of(int fmt) { return fmt == CLQ_MX_BLOCK16 ? 16 : 32; }
// Groups of four scales of a row.
__host__ __device__ inline int scale_chunks(int K, int fmt) {
  return (K / block_of(fmt) + 3) / 4;
}

struct QuantArgs {
  const void* X;
  int32_t M, K, ld;
  const int32_t* perm;  // [K] or null
  int32_t b, act;
  uint8_t* codes;
  uint8_t* scales;
  float* row_scale;         // BLOCK16
  const int32_t* out_rows;  // [M][k] or null
  int32_t k, rows;
  int32_t block_rows;           // filled in by the launcher
  const struct RowTile* tiles;  // X holds the rows of a plan: its tiles of 128 rows, or null
  const int32_t* tile_count;
  int32_t* status;
};
cudaError_t launch_quantize(const QuantArgs& a, int dtype, int fmt, cudaStream_t st);
cudaError_t launch_dequantize(const uint8_t* codes, const uint8_t* scales, const float* row_scale,
                              int M, int K, int fmt, int dtype, void* out, cudaStream_t st);

// One tile of rows of the grouped product: `rows` rows of `expert` from row `row0`.
struct RowTile {
  int32_t expert, row0, rows, unused;
};

// What clq_mx_plan leaves for the product.  tiles128 / tiles256: tiles of up to
// 128 / 256 rows of one expert, counts[0] / counts[1] of them.
struct PlanLayout {
  size_t counts_off, tiles128_off, tiles256_off, start_off, hist_off, prefix_off, bytes;
  int max128, max256, chunks, pitch;
};
PlanLayout plan_layout(int T, int k, int E);
inline int plan_rows(int T, int k, int E) {
  const int64_t n = static_cast<int64_t>(T) * k;
  return static_cast<int>((n + 127 * std::min<int64_t>(E, n)) / kRowBlock * kRowBlock);
}

struct GemmArgs {
  const float* s_x;
  const float* s_w;
  const void* bias;
  void* Y;
  int32_t M, N, K;
  float inv_b;
  int32_t chunks;    // scale_chunks of a row
  int32_t w_blocks;  // scale row blocks of one weight matrix
  const RowTile* tiles;  // grouped: the tile list and its length, on the device
  const int32_t* tile_count;
  int32_t max_tiles;  // grouped: host bound of the list
  int32_t experts;    // weight matrices (1: dense)
  int32_t x_rows;     // rows of the X code array
  uint8_t* Yq;        // output as codes (act of the rounded product), or null
  uint8_t* Ys;
  int32_t act, y_chunks;
  int32_t* status;
};
cudaError_t launch_gemm(const uint8_t* Xq, const uint8_t* Xs, const uint8_t* Wq,
                        const uint8_t* Ws, const GemmArgs& g, int fmt, int dtype, const void* plan,
                        const PlanLayout* pl, int T, int k, cudaStream_t st);

struct RouteArgs {
  const void* logits;
  const float* balance;
  int32_t* experts;
  float* weights;
  int32_t T, E, ld, k, scoring, groups, top_groups, group_top, renormalize;
  float scale;
};
cudaError_t launch_route(const RouteArgs& a, int dtype, cudaStream_t st);
cudaError_t launch_plan(const int32_t* experts, int T, int k, int E, int32_t* out_rows, void* plan,
                        const PlanLayout& pl, cudaStream_t st);
cudaError_t launch_combine(const void* Y, int dtype, const int32_t* rows, const float* weights,
                           int T, int k, int D, int R, void* out, int32_t* status,
                           cudaStream_t st);

}  // namespace mx
}  // namespace clq
