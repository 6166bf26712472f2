// Host-side interface of the norms around a block (norms.cu).
#pragma once

#include "internal.h"

namespace bcmt {

struct NormFwd {
  long long rows;
  int D, layer, w_bf16;
  long long group_rows;   // consecutive rows that share a row of the gate
  float alpha, eps;
  const void *branch, *x, *weight, *bias, *post_weight, *post_bias, *gate;  // bias.. may be NULL
  void *h, *n;
};

struct NormBwd {
  int D, layer, w_bf16;
  long long group_rows;
  float alpha, eps;
  const void *dh, *dn, *branch, *h, *weight, *post_weight, *post_bias, *gate;  // dh may be NULL
  void *dbranch, *dx, *dgate;   // dx, dgate may be NULL
  int wanted;                   // bits: which of dw, db, dpw, dpb
  float *part, *gate_part;      // sums of each CTA [ctas, 4, D], of each segment [nseg, D]
  // from the plan
  int tpr, rows_per_cta, turns;
  long long seg_rows, segs_per_group, seg_group_rows, nseg;
};

// Sums of the parts: dw, db, dpw, dpb (NULL: not wanted) and the gates' gradient.
struct NormJoin {
  int D, w_bf16, t_bf16;
  void* out[4];
  void* dgate;
  const float *part, *gate_part;
  long long first, nparts, segs_per_group;
};

// How a backward call is cut: threads of a row, rows at a time in a CTA, CTAs, and the
// segments of rows that its workers walk.
struct NormPlan {
  int tpr, threads, rows_per_cta, ctas, turns;
  bool wide;
  long long seg_rows, segs_per_group, seg_group_rows, nseg;
  size_t part_bytes, gate_bytes;
};
constexpr int kNormMaxD = 8192;
NormPlan norm_plan(long long rows, int D, long long groups, bool post, int sms);
cudaError_t norm_bwd_f32(const Launch& lc, const NormBwd& a, const NormPlan& pl);
cudaError_t norm_bwd_bf16(const Launch& lc, const NormBwd& a, const NormPlan& pl);
cudaError_t norm_forward(const Launch& lc, int dtype, const NormFwd& a);
cudaError_t norm_backward(const Launch& lc, int dtype, const NormPlan& pl, NormBwd a,
                          const NormJoin& j);

}  // namespace bcmt
