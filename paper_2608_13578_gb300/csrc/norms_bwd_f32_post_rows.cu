// Backward of the norms around a block over fp32 rows, with a post norm and a gate per row (files of
// their own so that the kernels compile side by side).
#include "norms_bwd.cuh"

namespace bcmt {

cudaError_t norms_bwd_f32_post_rows(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  return bwd_typed<float, true, true>(lc, a, pl);
}

}  // namespace bcmt
