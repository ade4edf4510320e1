// gemm_tn.cu -- instances of the matrix product of gemm.cuh: both operands with rows along k, bf16.
#include "gemm.cuh"

namespace bds {

cudaError_t launch_gemm_tn(const GemmCfg& c, const GemmParams& p, const GemmMaps& m, cudaStream_t s) {
  if (c.epi == kEpiOut && c.cg == 2 && c.bn == 256 && c.pieces == 1 && c.out_f32 == false)
    return gemm_t<2, 256, 1, true, true, kEpiOut, false>(p, m, s);
  if (c.epi == kEpiOut && c.cg == 2 && c.bn == 256 && c.pieces == 1 && c.out_f32 == true)
    return gemm_t<2, 256, 1, true, true, kEpiOut, true>(p, m, s);
  if (c.epi == kEpiOut && c.cg == 1 && c.bn == 128 && c.pieces == 1 && c.out_f32 == false)
    return gemm_t<1, 128, 1, true, true, kEpiOut, false>(p, m, s);
  if (c.epi == kEpiOut && c.cg == 1 && c.bn == 128 && c.pieces == 1 && c.out_f32 == true)
    return gemm_t<1, 128, 1, true, true, kEpiOut, true>(p, m, s);
  if (c.epi == kEpiRows && c.cg == 2 && c.bn == 256 && c.pieces == 1 && c.out_f32 == false)
    return gemm_t<2, 256, 1, true, true, kEpiRows, false>(p, m, s);
  if (c.epi == kEpiRows && c.cg == 1 && c.bn == 128 && c.pieces == 1 && c.out_f32 == false)
    return gemm_t<1, 128, 1, true, true, kEpiRows, false>(p, m, s);
  if (c.epi == kEpiJoin && c.cg == 1 && c.bn == 128 && c.pieces == 1)
    return gemm_t<1, 128, 1, true, true, kEpiJoin, false>(p, m, s);
  return cudaErrorInvalidValue;
}

}  // namespace bds
