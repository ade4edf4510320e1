// gemm_loss.cu -- instances of the matrix product of gemm.cuh: the loss's logits.
#include "gemm.cuh"

namespace bds {

cudaError_t launch_gemm_loss(const GemmCfg& c, const GemmParams& p, const GemmMaps& m, cudaStream_t s) {
  if (c.epi == kEpiStats && c.cg == 2 && c.bn == 256 && c.pieces == 1)
    return gemm_t<2, 256, 1, false, false, kEpiStats, false>(p, m, s);
  if (c.epi == kEpiStats && c.cg == 1 && c.bn == 128 && c.pieces == 1)
    return gemm_t<1, 128, 1, false, false, kEpiStats, false>(p, m, s);
  if (c.epi == kEpiStats && c.cg == 2 && c.bn == 128 && c.pieces == 3)
    return gemm_t<2, 128, 3, false, false, kEpiStats, false>(p, m, s);
  if (c.epi == kEpiStats && c.cg == 1 && c.bn == 128 && c.pieces == 3)
    return gemm_t<1, 128, 3, false, false, kEpiStats, false>(p, m, s);
  if (c.epi == kEpiDz && c.cg == 2 && c.bn == 256 && c.pieces == 1)
    return gemm_t<2, 256, 1, false, false, kEpiDz, false>(p, m, s);
  if (c.epi == kEpiDz && c.cg == 1 && c.bn == 128 && c.pieces == 1)
    return gemm_t<1, 128, 1, false, false, kEpiDz, false>(p, m, s);
  if (c.epi == kEpiDz && c.cg == 2 && c.bn == 128 && c.pieces == 3)
    return gemm_t<2, 128, 3, false, false, kEpiDz, false>(p, m, s);
  if (c.epi == kEpiDz && c.cg == 1 && c.bn == 128 && c.pieces == 3)
    return gemm_t<1, 128, 3, false, false, kEpiDz, false>(p, m, s);
  return cudaErrorInvalidValue;
}

}  // namespace bds
