// Backward of the norms around a block over fp32 rows, with a post norm (files of
// their own so that the kernels compile side by side).
#include "norms_bwd.cuh"

namespace bcmt {

cudaError_t norms_bwd_f32_post(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  return bwd_typed<float, true, false>(lc, a, pl);
}

}  // namespace bcmt
