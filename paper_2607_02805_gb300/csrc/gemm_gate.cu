// gemm_gate.cu -- instances of the matrix product of gemm.cuh: the gated linear layer, forward and the gradients at
// its projections.
#include "gemm.cuh"

namespace bds {
namespace {

template <int EPI>
cudaError_t gate_cfg(const GemmCfg& c, const GemmParams& p, const GemmMaps& m, cudaStream_t s) {
  if (c.cg == 2 && c.bn == 256 && c.pieces == 1) return gemm_t<2, 256, 1, false, false, EPI, false>(p, m, s);
  if (c.cg == 1 && c.bn == 128 && c.pieces == 1) return gemm_t<1, 128, 1, false, false, EPI, false>(p, m, s);
  if (c.cg == 2 && c.bn == 128 && c.pieces == 3) return gemm_t<2, 128, 3, false, false, EPI, true>(p, m, s);
  if (c.cg == 1 && c.bn == 128 && c.pieces == 3) return gemm_t<1, 128, 3, false, false, EPI, true>(p, m, s);
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_gemm_gate(const GemmCfg& c, const GemmParams& p, const GemmMaps& m, cudaStream_t s) {
  switch (c.epi) {
    case kEpiGate: return gate_cfg<kEpiGate>(c, p, m, s);
    case kEpiGateRows: return gate_cfg<kEpiGateRows>(c, p, m, s);
    case kEpiGateDz: return gate_cfg<kEpiGateDz>(c, p, m, s);
    case kEpiGateDzRows: return gate_cfg<kEpiGateDzRows>(c, p, m, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace bds
