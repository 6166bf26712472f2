// Backward of the norms around a block over bf16 rows, without a post norm (files of their own so that the
// kernels compile side by side).
#include "norms_bwd.cuh"

namespace bcmt {

cudaError_t norms_bwd_bf16(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  return pl.mode == kGateRows ? bwd_typed<bf16, false, true>(lc, a, pl) : bwd_typed<bf16, false, false>(lc, a, pl);
}

}  // namespace bcmt
