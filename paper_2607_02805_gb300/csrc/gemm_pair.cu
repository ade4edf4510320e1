// gemm_pair.cu -- instances of the matrix product of gemm.cuh: the two
// products of a gradient in one launch, B with rows along k, A either way.
#include "gemm.cuh"

namespace bds {

cudaError_t launch_gemm_pair(const GemmCfg& c, const GemmCall<2>& call, cudaStream_t s) {
  if (c.cg == 2 && c.bn == 256 && c.pieces == 1) return gemm_pair_t<2, 256, 1>(call, s);
  if (c.cg == 1 && c.bn == 128 && c.pieces == 1) return gemm_pair_t<1, 128, 1>(call, s);
  if (c.cg == 2 && c.bn == 128 && c.pieces == 3) return gemm_pair_t<2, 128, 3>(call, s);
  if (c.cg == 1 && c.bn == 128 && c.pieces == 3) return gemm_pair_t<1, 128, 3>(call, s);
  return cudaErrorInvalidValue;
}

}  // namespace bds
