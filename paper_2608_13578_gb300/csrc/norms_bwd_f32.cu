// Backward of the norms around a block over fp32 rows, without a post norm (files of their own so that the
// kernels compile side by side).
#include "norms_bwd.cuh"

namespace bcmt {

cudaError_t norms_bwd_f32(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  return pl.mode == kGateRows ? bwd_typed<float, false, true>(lc, a, pl) : bwd_typed<float, false, false>(lc, a, pl);
}

}  // namespace bcmt
