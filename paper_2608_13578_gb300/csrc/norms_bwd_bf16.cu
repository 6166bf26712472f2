// Backward of the norms around a block over bf16 rows (a file of its own so that the two
// types compile side by side).
#include "norms_bwd.cuh"

namespace bcmt {

cudaError_t norm_bwd_bf16(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  return a.post_weight ? bwd_typed<bf16, true>(lc, a, pl) : bwd_typed<bf16, false>(lc, a, pl);
}

}  // namespace bcmt
