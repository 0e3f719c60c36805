// Launch of the microscaled product (mx_gemm.cuh): tensor maps.
#include "mx_gemm.cuh"

namespace clq {
namespace mx {
namespace {

bool codes_map(CUtensorMap* m, const uint8_t* p, int64_t rows, int K, int box_rows) {
  return encode_tma_2d(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, p, static_cast<uint64_t>(K) / 2,
                       static_cast<uint64_t>(rows), 128, box_rows, CU_TENSOR_MAP_SWIZZLE_128B);
}

// A scale array as rows of 512 bytes, `sc` of them a copy.  Copies that reach past a
// row block's chunks bring bytes that no MMA uses.
bool scales_map(CUtensorMap* m, const uint8_t* p, int64_t chunks, int sc) {
  return encode_tma_2d(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, p, 128,
                       static_cast<uint64_t>(chunks), 128, sc, CU_TENSOR_MAP_SWIZZLE_NONE);
}

}  // namespace

cudaError_t launch_gemm(const uint8_t* Xq, const uint8_t* Xs, const uint8_t* Wq,
                        const uint8_t* Ws, const GemmArgs& args, int fmt, int dtype,
                        const void* plan, const PlanLayout* pl, int T, int k, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return cudaErrorInvalidDevice;
  GemmArgs g = args;
  const bool grouped = plan != nullptr;
  const int64_t blocks = (g.x_rows + kRowBlock - 1) / kRowBlock;
  const TileShape t = grouped ? pick_grouped_tile(T, k, g.experts, g.N, g.K, sms)
                              : pick_tile(g.M, 1, g.N, g.K, sms, false);
  const int nt = t.nt, cg = t.cg;
  if (grouped) {
    const uint8_t* p = static_cast<const uint8_t*>(plan);
    g.tiles = reinterpret_cast<const RowTile*>(p + (nt == 256 ? pl->tiles256_off : pl->tiles128_off));
    g.tile_count = reinterpret_cast<const int32_t*>(p + pl->counts_off) + (nt == 256 ? 1 : 0);
    g.max_tiles = nt == 256 ? pl->max256 : pl->max128;
  }
  const int sc = fmt == CLQ_MX_BLOCK16 ? 4 : 2;
  GemmMaps m;
  if (!codes_map(&m.W, Wq, static_cast<int64_t>(g.experts) * g.N, g.K, TN) ||
      !codes_map(&m.X, Xq, g.x_rows, g.K, nt / cg) ||
      !scales_map(&m.SW, Ws, static_cast<int64_t>(g.experts) * g.w_blocks * g.chunks, sc) ||
      !scales_map(&m.SX, Xs, blocks * g.chunks, sc))
    return cudaErrorInvalidValue;
  const int use_tma_store = g.Yq == nullptr && g.N % 8 == 0 ? 1 : 0;
  if (use_tma_store) {
    if (!encode_tma_out_tile(&m.Y, g.Y, g.x_rows, g.N)) return cudaErrorInvalidValue;
  } else {
    m.Y = m.W;  // unused
  }
  const int64_t row_tiles = grouped ? g.max_tiles : (g.M + nt - 1) / nt;
  const int64_t tiles = row_tiles * ((g.N + TN * cg - 1) / (TN * cg));
  const int grid = cg * static_cast<int>(std::min<int64_t>(tiles, sms / cg));
  GemmFn go = fmt == CLQ_MX_BLOCK32 ? (dtype == CLQ_F16 ? gemm_block32_f16 : gemm_block32_bf16)
                                    : (dtype == CLQ_F16 ? gemm_block16_f16 : gemm_block16_bf16);
  return go(m, g, t, grouped, use_tma_store, grid, st);
}

}  // namespace mx
}  // namespace clq
