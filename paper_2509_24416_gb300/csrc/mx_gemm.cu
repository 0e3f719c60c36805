// Launch of the microscaled product (mx_gemm.cuh): tensor maps and tile choice.
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

// The tile of a product whose rows are `rows` for each of `matrices` matrices: the CTAs or
// pairs go ceil(tiles / units) rounds; a round takes its K steps and the part of an epilogue
// that the next round's MMAs do not cover, and the last epilogue and the launch come on top.
// The times are fitted to 112 products of 33 .. 8192 rows (step: us for 256 codes; epilogue:
// us a tile); the rule is within 10 % of the best of the five on all but six of them (18 % off at most).  Examples,
// us at 64 / 128 / 128 in pairs / 256 / 256 in pairs: 64 x 1152 -> 3456 3.8 / 4.1 / 4.1 / 5.1 /
// 4.8, 2048 x 4608 -> 1152 10.4 / 7.4 / 10.3 / 11.0 / 9.8, 4096 x 4608 -> 1152 18.4 / 11.7 /
// 13.9 / 11.2 / 15.3, 8192 x 4096 -> 8192 190 / 114 / 91 / 110 / 83.
TileShape pick_tile(int rows, int matrices, int N, int K, int sms, bool grouped) {
  if (rows <= 32) return {32, 1};
  struct Option {
    TileShape t;
    double step, epilogue;
    bool plan;  // a plan has such tiles
  };
  const Option options[] = {{{64, 1}, 0.22, 0.75, false},
                            {{128, 1}, 0.26, 1.03, true},
                            {{128, 2}, 0.21, 1.03, false},
                            {{256, 1}, 0.48, 1.8, false},
                            {{256, 2}, 0.36, 1.8, true}};
  TileShape best{128, 1};
  double least = 1e300;
  for (const Option& o : options) {
    if (grouped && !o.plan) continue;
    const int64_t tiles = static_cast<int64_t>(matrices) * ((rows + o.t.nt - 1) / o.t.nt) *
                          ((N + TN * o.t.cg - 1) / (TN * o.t.cg));
    const int64_t units = sms / o.t.cg;
    const double cost = ((tiles + units - 1) / units) *
                            ((K + KC - 1) / KC * o.step + 0.35 * o.epilogue) +
                        o.epilogue;
    if (cost < least) {
      least = cost;
      best = o.t;
    }
  }
  return best;
}

}  // namespace

cudaError_t launch_gemm(const uint8_t* Xq, const uint8_t* Xs, const uint8_t* Wq,
                        const uint8_t* Ws, const GemmArgs& args, int fmt, int dtype,
                        const void* plan, const PlanLayout* pl, int T, int k, cudaStream_t st) {
  const int64_t picks = static_cast<int64_t>(T) * k;
  const int sms = sm_count();
  if (sms <= 0) return cudaErrorInvalidDevice;
  GemmArgs g = args;
  const bool grouped = plan != nullptr;
  const int64_t blocks = (g.x_rows + kRowBlock - 1) / kRowBlock;
  // A plan's rows are taken as evenly spread over the matrices that have any; T rows at most
  // meet one of them.
  const int64_t spread = std::max<int64_t>(1, std::min<int64_t>(g.experts, picks));
  const TileShape t =
      grouped ? (T <= 32 ? TileShape{32, 1}
                         : pick_tile(std::max(33, static_cast<int>((picks + spread - 1) / spread)),
                                     static_cast<int>(spread), g.N, g.K, sms, true))
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
