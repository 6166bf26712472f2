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

// How a forward call walks its rows.
struct NormWalk {
  int tpr, threads, ctas, stages, smem;
};

// How rows share the gate: none, one for all, one for groups of rows, one per row.
enum NormMode { kGateNone, kGateOne, kGateGroups, kGateRows };

struct NormBwd {
  long long rows;
  int D, layer, w_bf16;
  float alpha, eps;
  const void *dh, *dn, *branch, *h, *weight, *post_weight, *post_bias, *gate;  // dh may be NULL
  void *dbranch, *dx, *dgate;   // dx, dgate may be NULL
  int wanted;                   // bits: which of dw, db, dpw, dpb
  float *part, *gate_part;      // sums of each CTA [ctas, 4, D], of each segment [nseg, D]
  // from the plan
  int tpr, stages, mode, ring16, ds_slots;
  bool gp_smem, tot_smem, pw_smem, one_seg;
  long long seg_rows, segs_per_group, seg_group_rows, nseg;
};

// Sums of the parts: dw, db, dpw, dpb (NULL: not wanted) and the gates' gradient (with one
// gate: from the last two, which it also scales).
struct NormJoin {
  int D, w_bf16, t_bf16, mode;
  void* out[4];
  void* dgate;
  const void *gate, *post_weight, *post_bias;
  const float *part, *gate_part;
  long long first, nparts, segs_per_group;
};

// How a backward call is cut: threads of a row with 8 J columns each, threads of a CTA,
// CTAs, its shared memory, and the segments of rows that its workers walk.
struct NormPlan {
  int tpr, J, threads, ctas, stages, mode, ring16, ds_slots, smem;
  bool gp_smem, tot_smem, pw_smem, one_seg;
  long long seg_rows, segs_per_group, seg_group_rows, nseg;
  size_t part_bytes, gate_bytes;
};
constexpr int kNormMaxD = 8192;
constexpr int kNormSmem = 227 * 1024 - 1024;   // of a CTA, beside the sums' buffers
// Warps of a CTA whose threads have 8 J columns, one warp a row or several: 96, 128, and for
// rows of 24 columns a lane of one warp 168 registers a thread (16384 x 768: 40 us, with 16 warps
// of 128 registers 42).
constexpr int norm_max_warps(int J, bool one) { return J == 1 ? 20 : one && J == 3 ? 12 : 16; }
NormPlan norm_plan(long long rows, int D, int es, long long groups, bool post, int sms);
cudaError_t norms_bwd_f32(const Launch& lc, const NormBwd& a, const NormPlan& pl);
cudaError_t norms_bwd_f32_post(const Launch& lc, const NormBwd& a, const NormPlan& pl);
cudaError_t norms_bwd_f32_post_rows(const Launch& lc, const NormBwd& a, const NormPlan& pl);
cudaError_t norms_bwd_bf16(const Launch& lc, const NormBwd& a, const NormPlan& pl);
cudaError_t norms_bwd_bf16_post(const Launch& lc, const NormBwd& a, const NormPlan& pl);
cudaError_t norms_bwd_bf16_post_rows(const Launch& lc, const NormBwd& a, const NormPlan& pl);
cudaError_t norm_forward(const Launch& lc, int dtype, const NormFwd& a, int sms);
cudaError_t norm_backward(const Launch& lc, int dtype, const NormPlan& pl, NormBwd a,
                          const NormJoin& j);

}  // namespace bcmt
