// Linear attention with a decay per head: the passes the kernels run.
//
// A pass computes, for one head of one sequence with n valid tokens,
//   S_t = a S_{t-1} + k_t v_t^T,   o_t = out_mul * S_t^T q_t     (t < n)
// forwards in time, or the same recurrence backwards in time (rev: S_t =
// a S_{t+1} + k_t v_t^T, the incoming state not decayed by the last valid
// token).  Rows t >= n of o are written as zeros.  The layer's forward is one
// pass; its backward is three:
//   dq = pass(do, v, k),  dv = rev pass(k, q, do),  dk = rev pass(v, do, q)
// with the transposed states in the first and the last.
#pragma once

#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"

namespace bcmt {

struct LinPass {
  const void *q, *k, *v;  // row of token (b, t): x + (b*T + t) * ld, head h at column h*dh
  long ldq, ldk, ldv;
  void* o;                // null: states only
  long ldo;
  const float* s_in;      // [B, H, dh, dh] or null (zero)
  int s_in_t;             // read transposed
  float s_in_mul;
  float* s_out;           // [B, H, dh, dh] or null; may be s_in (when not transposed)
  float s_out_mul;        // multiplies the outgoing state (rev: times a as well, when n > 0)
  float out_mul;
  int rev;
  float* seg;             // segment states [B*H, nseg, dh, dh] fp32 (nseg > 1)
};

struct LinArgs {
  LinPass pass[3];
  int npass;
  int B, T, H, dh;
  const float* decay;     // [H]
  const int* lengths;     // [B] or null
  int nseg, seg_len;      // the tokens in nseg segments of seg_len
  int joined;             // pass.seg holds the segments' incoming states, not their own
  // the tensor-core form's segment states: groups of 4 columns of all rows together,
  // and the join gives the outgoing state too
  int grouped;
  unsigned* status;       // the device status word
};

// A decay outside [0, 1] (or NaN) is reported by the walks and the single-token step;
// what its head then gives is not defined.
__device__ __forceinline__ void check_decay(float a, unsigned* status) {
  if (!(a >= 0.f && a <= 1.f)) atomicOr(status, kStatusBadDecay);
}

// How the passes are cut along the tokens (the same rule for the workspace
// size and the launch): `tc` tells which kernel runs.
struct LinPlan {
  bool tc;
  int nseg, seg_len;
};
LinPlan linattn_plan(int dtype, int B, int T, int H, int dh, int npass, int sms, bool allow_tc,
                     bool ragged);

// The recurrence on CUDA cores in fp32, any dtype and head width.
cudaError_t linattn_simt(const Launch& lc, int dtype, const LinArgs& a);
// T = 1, forward: the state is read once and written once.
cudaError_t linattn_step(const Launch& lc, int dtype, const LinArgs& a);
// The chunked form on the tensor cores: bf16, segments of whole 128-token chunks.
cudaError_t linattn_tc(const Launch& lc, const LinArgs& a);
// Local segment states (in pass.seg) -> each segment's incoming state, and with
// a.grouped the outgoing state.
cudaError_t linattn_combine(const Launch& lc, const LinArgs& a);

}  // namespace bcmt
