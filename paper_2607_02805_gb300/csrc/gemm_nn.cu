// gemm_nn.cu -- instances of the matrix product of gemm.cuh: A with rows along m, B with rows along k.
#include "gemm.cuh"

namespace bds {

cudaError_t launch_gemm_nn(const GemmCfg& c, const GemmParams& p, const GemmMaps& m, cudaStream_t s) {
  if (c.cg == 2 && c.bn == 256 && c.pieces == 1)
    return gemm_t<2, 256, 1, false, true, kEpiOut>(p, m, s);
  if (c.cg == 1 && c.bn == 128 && c.pieces == 1)
    return gemm_t<1, 128, 1, false, true, kEpiOut>(p, m, s);
  if (c.cg == 1 && c.bn == 64 && c.pieces == 1)
    return gemm_t<1, 64, 1, false, true, kEpiOut>(p, m, s);
  if (c.cg == 2 && c.bn == 128 && c.pieces == 3)
    return gemm_t<2, 128, 3, false, true, kEpiOut>(p, m, s);
  if (c.cg == 1 && c.bn == 128 && c.pieces == 3)
    return gemm_t<1, 128, 3, false, true, kEpiOut>(p, m, s);
  return cudaErrorInvalidValue;
}

}  // namespace bds
