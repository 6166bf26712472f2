// Backward of the norms around a block over bf16 rows, with a post norm (files of
// their own so that the kernels compile side by side).
#include "norms_bwd.cuh"

namespace bcmt {

cudaError_t norms_bwd_bf16_post(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  return bwd_typed<bf16, true, false>(lc, a, pl);
}

}  // namespace bcmt
