// gemm_tn3.cu -- instances of the matrix product of gemm.cuh: both operands with rows along k, fp32.
#include "gemm.cuh"

namespace bds {

cudaError_t launch_gemm_tn3(const GemmCfg& c, const GemmParams& p, const GemmMaps& m, cudaStream_t s) {
  if (c.epi == kEpiOut && c.cg == 2 && c.bn == 128 && c.pieces == 3 && c.out_f32 == true)
    return gemm_t<2, 128, 3, true, true, kEpiOut, true>(p, m, s);
  if (c.epi == kEpiOut && c.cg == 1 && c.bn == 128 && c.pieces == 3 && c.out_f32 == true)
    return gemm_t<1, 128, 3, true, true, kEpiOut, true>(p, m, s);
  if (c.epi == kEpiRows && c.cg == 2 && c.bn == 128 && c.pieces == 3 && c.out_f32 == true)
    return gemm_t<2, 128, 3, true, true, kEpiRows, true>(p, m, s);
  if (c.epi == kEpiRows && c.cg == 1 && c.bn == 128 && c.pieces == 3 && c.out_f32 == true)
    return gemm_t<1, 128, 3, true, true, kEpiRows, true>(p, m, s);
  return cudaErrorInvalidValue;
}

}  // namespace bds
