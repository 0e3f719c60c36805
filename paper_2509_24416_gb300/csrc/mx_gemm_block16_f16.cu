// Microscaled product, blocks of 16, f16 outputs.
#include "mx_gemm.cuh"

namespace clq {
namespace mx {
cudaError_t gemm_block16_f16(const GemmMaps& m, const GemmArgs& g, TileShape t, bool grouped,
                            int use_tma_store, int grid, cudaStream_t st) {
  return launch_gemm_tiles<__half, CLQ_MX_BLOCK16>(m, g, t, grouped, use_tma_store, grid, st);
}
}  // namespace mx
}  // namespace clq
