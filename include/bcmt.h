/*
 * bcmt.h -- C ABI of the GB300 (sm_103a) BCMT token mixer.
 *
 * BCMT ("Blockwise Causal Memory Transformer") replaces dense causal
 * self-attention with four steps, all computed on the GPU by this library:
 *
 *   1. dense causal multi-head attention inside each length-L block, then the
 *      output projection W_O                                       (Sec. 3.2-3.3)
 *   2. an adaptive softmax-pooled summary S_i of each block          (Sec. 3.4)
 *   3. the normalised exponential causal memory
 *        M_i = sum_{j<=i} a^(i-j) S_j / sum_{j<=i} a^(i-j),
 *      projected by W_m and shifted by one block                     (Sec. 3.5)
 *   4. broadcast of the memory to the block's tokens and gated injection
 *        Y = H + sigmoid(H W_g) * M_tokens                           (Sec. 3.7-3.8)
 *
 * and the matching backward pass (the paper trains the layer with autograd,
 * Sec. 4.1; the gradients are derived from the forward definition).
 *
 * Conventions common to every entry point
 * ---------------------------------------
 *  - All tensor pointers are DEVICE pointers owned by the caller.  The library
 *    allocates no device memory per call; the caller provides a forward
 *    workspace (bcmt_workspace_size) that carries the activations saved for
 *    the backward pass, and a backward scratch buffer (bcmt_scratch_size).
 *  - Tensors are dense, row-major, without padding: x, y, q, k, v, dy, dx ...
 *    are [B, T, D]; token (b, t) is row b*T + t.
 *  - Weights follow the paper's row-vector convention (Q = X W_Q): a weight is
 *    [D_in, D_out] row-major.  W_qkv = [W_Q | W_K | W_V] is [D, 3D].  Head i
 *    owns columns i*dh .. (i+1)*dh - 1 of Q, K, V and of Concat(heads).
 *  - dtype: every tensor except `decay` has the storage type p->dtype (fp32 or
 *    bf16); arithmetic accumulates in fp32.  `decay` is always fp32 [D], each
 *    entry in [0, 1); pass 0.8 in every entry for the paper's setting.
 *  - Pointers must be 16-byte aligned.  Requirements on shapes: B, T >= 1;
 *    H >= 1 and D % H == 0; dh = D / H a multiple of 8 and <= 128; D a
 *    multiple of 64; 1 <= L <= 1024.  Any T is accepted: the last block may be
 *    ragged (Sec. 3.2).  bf16 shapes with dh in {16, 32, 64} run the tcgen05
 *    tensor-core attention: L in {16, 32, 64, 128} on the single-tile kernels
 *    (a 128-token tile holds whole blocks), L a multiple of 128 from 256 to
 *    1024 on the key-tile-walking kernels (an online softmax over the block's
 *    128-token key tiles).  fp32 shapes, other head widths and the remaining
 *    block sizes run a SIMT attention kernel in fp32.
 *  - `stream` is a cudaStream_t (NULL = legacy default stream).  Calls are
 *    asynchronous: they validate their arguments, enqueue kernels and return.
 *    On invalid arguments nothing is launched and an error code is returned;
 *    bcmt_last_error() then describes it.
 *  - Device-side waits are bounded.  A wait that expires sets a device status
 *    word instead of hanging; it is read by bcmt_device_status(), and
 *    automatically at the end of each call when p->flags has BCMT_FLAG_CHECK
 *    (which synchronises the stream).
 */
#ifndef BCMT_H
#define BCMT_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  BCMT_OK = 0,
  BCMT_ERR_ARG = 1,         /* null pointer or out-of-range parameter value        */
  BCMT_ERR_SHAPE = 2,       /* shape violates the requirements above               */
  BCMT_ERR_ALIGN = 3,       /* a pointer is not 16-byte aligned                    */
  BCMT_ERR_CUDA = 4,        /* a CUDA runtime call or kernel launch failed         */
  BCMT_ERR_TIMEOUT = 5,     /* a bounded device-side wait expired                  */
  BCMT_ERR_UNSUPPORTED = 6  /* valid for the method, not implemented by the library */
} bcmt_status;

typedef enum { BCMT_F32 = 0, BCMT_BF16 = 1 } bcmt_dtype;

/* p->flags bits */
#define BCMT_FLAG_HONLY 1u    /* the paper's HOnly ablation (Sec. 4.5): Y = H, no summary/memory/gate */
#define BCMT_FLAG_CHECK 2u    /* synchronise at the end of the call and report device status        */
#define BCMT_FLAG_PROFILE 4u  /* record CUDA events around every kernel (bcmt_profile_read)          */

typedef struct {
  int B;           /* batch                                      */
  int T;           /* sequence length                            */
  int D;           /* model width d_model                        */
  int H;           /* attention heads h (head width dh = D / H)  */
  int L;           /* block size (Sec. 3.2)                      */
  int dtype;       /* bcmt_dtype of every tensor except decay    */
  int input_is_x;  /* 1: layer starts at x and W_qkv (Sec. 3.3); 0: at Q, K, V */
  unsigned flags;  /* BCMT_FLAG_* bits                           */
} bcmt_params;

/* Bytes of forward workspace: the activations bcmt_forward saves for
 * bcmt_backward (Q/K/V when input_is_x, attention log-sum-exp, Concat(heads),
 * H, pooling weights, summaries, memory, its projection, the gate).  Returns 0
 * for invalid parameters. */
size_t bcmt_workspace_size(const bcmt_params* p);

/* Bytes of backward scratch (temporaries of one backward call; free to reuse
 * between calls).  Returns 0 for invalid parameters. */
size_t bcmt_scratch_size(const bcmt_params* p);

/* Forward pass, Sec. 3.2-3.8.
 *   x      [B,T,D]   used iff input_is_x (else may be NULL)
 *   q,k,v  [B,T,D]   used iff !input_is_x (else may be NULL)
 *   w_qkv  [D,3D]    used iff input_is_x
 *   w_o    [D,D]     output projection W_O (Sec. 3.3)
 *   w_p    [D]       pooling score vector W_p (Sec. 3.4)
 *   w_m    [D,D]     memory projection W_m (Sec. 3.5)
 *   w_g    [D,D]     gate W_g (Sec. 3.8)
 *   decay  [D] fp32  exponential decay a per channel, each in [0,1)
 *   y      [B,T,D]   output, written
 *   workspace        bcmt_workspace_size(p) bytes, written; keep it unchanged
 *                    until the matching bcmt_backward has run
 * With BCMT_FLAG_HONLY, w_p, w_m, w_g and decay are unused and Y = H. */
bcmt_status bcmt_forward(const bcmt_params* p, const void* x, const void* q, const void* k,
                         const void* v, const void* w_qkv, const void* w_o, const void* w_p,
                         const void* w_m, const void* w_g, const float* decay, void* y,
                         void* workspace, void* stream);

/* Backward pass: gradients of sum(dy * Y) with respect to the layer inputs
 * and weights, given the workspace of the matching bcmt_forward (same p and
 * same inputs).  The paper keeps the decay fixed (Sec. 3.5); its gradient,
 * for a learned per-channel decay (named as future work in Sec. 5), is
 * returned only when d_decay is non-NULL.
 *   dy       [B,T,D]
 *   x_or_q   the forward's x when input_is_x, else its q
 *   k, v     the forward's k and v iff !input_is_x (else may be NULL)
 *   w_qkv, w_o, w_p, w_m, w_g, decay: the forward's weights (w_qkv iff
 *            input_is_x)
 *   workspace  the forward's workspace (read only)
 *   scratch    bcmt_scratch_size(p) bytes
 *   dx_or_dq [B,T,D]  dx when input_is_x, else dq
 *   dk, dv   [B,T,D]  used iff !input_is_x
 *   dw_qkv   [D,3D]   used iff input_is_x
 *   dw_o [D,D], dw_p [D], dw_m [D,D], dw_g [D,D]
 *   d_decay  [D] fp32, optional (NULL: not computed)
 * Every output is overwritten (not accumulated).  With BCMT_FLAG_HONLY,
 * dw_p, dw_m, dw_g and d_decay are set to zero. */
bcmt_status bcmt_backward(const bcmt_params* p, const void* dy, const void* x_or_q,
                          const void* k, const void* v, const void* w_qkv, const void* w_o,
                          const void* w_p, const void* w_m, const void* w_g,
                          const float* decay, const void* workspace,
                          void* scratch, void* dx_or_dq, void* dk, void* dv, void* dw_qkv,
                          void* dw_o, void* dw_p, void* dw_m, void* dw_g, float* d_decay,
                          void* stream);

/* Incremental decoding (one new token per sequence per call).  The paper
 * trains only; decoding follows from the causal structure of Sec. 3.3-3.8:
 * token t of block i = t / L attends to the earlier tokens of its block, and
 * Y_t = H_t + sigmoid(H_t W_g) * C_i with C_i = M_{i-1} W_m (zero in block 0).
 * The state carries the current block's K/V cache, the block summary
 * accumulated online (Sec. 3.4), the memory recurrence N_i = a N_{i-1} + S_i,
 * Z_i = a Z_{i-1} + 1 (Sec. 3.5) and the current memory row.  Decoding the
 * tokens 0..T-1 of a sequence in order gives the rows of bcmt_forward's Y.
 *
 * p: B sequences decoded in lockstep, D, H, L, dtype and flags as for the
 * forward (BCMT_FLAG_HONLY: Y = H); input_is_x must be 1; p->T is ignored.
 *   state  bcmt_decode_state_size(p) bytes of device memory, caller-owned;
 *          bcmt_decode_reset zeroes it to start new sequences
 *   pos    position t of the token being decoded (0, 1, 2, ... in order; the
 *          state assumes the previous call decoded pos - 1)
 *   x_t    [B, D] the token's input row per sequence
 *   weights and decay as for bcmt_forward (x-entry: w_qkv [D, 3D])
 *   y_t    [B, D] output row, written
 * Calls are asynchronous on `stream`; consecutive steps of one state must be
 * issued in order on one stream. */
size_t bcmt_decode_state_size(const bcmt_params* p);
bcmt_status bcmt_decode_reset(const bcmt_params* p, void* state, void* stream);
bcmt_status bcmt_decode_step(const bcmt_params* p, void* state, long pos, const void* x_t,
                             const void* w_qkv, const void* w_o, const void* w_p,
                             const void* w_m, const void* w_g, const float* decay, void* y_t,
                             void* stream);

/* Allocation-free backward of the intra-block attention alone (the SIMT
 * kernels of the layer's backward; the paper has no counterpart -- it is an
 * interface for callers that cannot call cudaMalloc, such as a host framework
 * that owns all device memory and hands this library only input and output
 * buffers, or a latency-critical path where an allocation's implicit device
 * synchronisation is not acceptable).  It computes dq, dk, dv from the
 * forward's q, k, v (row stride ld, head h at column h*D/H), its output o
 * [B*T, D] and log-sum-exp lse [B,H,T] fp32, and the upstream gradient dO
 * [B*T, D]; dq, dk, dv are written with row stride ld_d.  Shapes as in *p
 * (B, T, D, H, L, dtype; input_is_x and flags other than BCMT_FLAG_CHECK are
 * ignored).
 *
 * Its one scratch buffer (one fp32 per batch, head and token) is a device
 * array inside the library: 4 MiB, allocated on every GPU that loads the
 * library and held until the process exits.  B*H*T must not exceed 1048576;
 * larger shapes are rejected with BCMT_ERR_SHAPE before anything is launched.
 * The first call on a device looks up that array's device address (once per
 * device, with that device current); make that first call before any stream
 * capture.  All calls share the array and it keeps the last call's contents:
 * calls that overlap on the GPU (other streams, other threads) race on it, so
 * serialise them.  Nothing is allocated: no cudaMalloc, cudaFree or
 * allocating library routine is called. */
bcmt_status bcmt_attention_backward_noalloc(const bcmt_params* p, const void* q, const void* k,
                                            const void* v, long ld, const void* o,
                                            const float* lse, const void* dO, void* dq, void* dk,
                                            void* dv, long ld_d, void* stream);

/* ------------------------------------------------------------------------
 * Operators of the language model around the mixer.
 *
 * Linear attention with a decay per head: BCMT's exponential memory (Sec. 3.5)
 * taken per token instead of per block summary, as a token mixer of its own.
 * Per sequence b and head h, with a = decay[h] and n = lengths[b] (T when
 * lengths is NULL; values are clamped to [0, T]):
 *     S_t = a S_{t-1} + k_t v_t^T,    o_t = scale * S_t^T q_t      for t < n,
 * S_{-1} = state_in (zero when NULL), o_t = 0 for t >= n and state_out =
 * S_{n-1} (state_in when n = 0).  Rows t >= n of q, k, v are never used,
 * whatever they hold.  T = 1 is the step of incremental decoding.
 *
 *   q, k, v, o ... rows of token (b, t) start at x + (b*T + t)*ld elements, head
 *            h at column h*dh (dh channels); each row stride ld >= H*dh is a
 *            multiple of 8, so q, k, v may be slices of one projection's rows
 *   decay    [H] fp32, each in [0, 1] (a^0 = 1 for a = 0 too); a constant: no
 *            gradient is computed for it.  One outside, or NaN, is reported as
 *            BCMT_ERR_ARG by the next bcmt_device_status (BCMT_FLAG_CHECK: by the
 *            call); what its head gives then is not defined, the others are right
 *   lengths  [B] int32 device memory, or NULL
 *   state    [B, H, dh, dh] fp32, row = channel of k, column = channel of v
 *   Requirements: B, T, H >= 1; dh a multiple of 8, 8 <= dh <= 128; scale
 *   finite and not 0; B*T <= 2^30; B*H*dh <= 2^26.  flags: BCMT_FLAG_CHECK only.
 *   Arithmetic and states are fp32; with bf16 tensors the tensor-core form
 *   rounds the decayed scores and the state to bf16 where they enter a product
 *   with bf16 rows.  The running state is an fp32 sum whose decayed keys carry 16
 *   bits, in the states that a call returns 24.  An infinity or NaN of a valid
 *   entry reaches the rows that the definition lets it reach and no other: of o
 *   and dq no row of an earlier token, of dk and dv none of a later one.  No
 *   output may overlap an input, but for the states as stated below. */
typedef struct {
  int B, T, H, dh;
  int dtype;       /* bcmt_dtype of q, k, v, o and their gradients */
  unsigned flags;
  float scale;     /* usually 1 / sqrt(dh) */
} bcmt_linattn_params;

/* Bytes of workspace of one forward (backward = 0) or backward (1) call; free
 * to reuse between calls.  256 means that the call uses none, and then NULL may
 * be passed.  Returns 0 for invalid parameters. */
size_t bcmt_linattn_workspace_size(const bcmt_linattn_params* p, int backward);

/* state_in and state_out may each be NULL, and may be the same buffer. */
bcmt_status bcmt_linattn_forward(const bcmt_linattn_params* p, const void* q, long ld_q,
                                 const void* k, long ld_k, const void* v, long ld_v,
                                 const float* decay, const int* lengths, const float* state_in,
                                 void* o, long ld_o, float* state_out, void* workspace,
                                 void* stream);

/* Gradients of sum(d_o * o) + sum(d_state_out * state_out) with respect to q, k,
 * v and state_in, from the forward's inputs (nothing else is kept).
 * d_state_out NULL: zero; d_state_in NULL: not computed (it must not be
 * d_state_out's or state_in's buffer).  Rows t >= n of dq, dk, dv are zero.
 * d_state_out / scale must stay within fp32: with d_state_out, a scale whose
 * reciprocal does not is refused. */
bcmt_status bcmt_linattn_backward(const bcmt_linattn_params* p, const void* d_o, long ld_do,
                                  const void* q, long ld_q, const void* k, long ld_k,
                                  const void* v, long ld_v, const float* decay,
                                  const int* lengths, const float* state_in,
                                  const float* d_state_out, void* dq, long ld_dq, void* dk,
                                  long ld_dk, void* dv, long ld_dv, float* d_state_in,
                                  void* workspace, void* stream);

/* Scaled embedding lookup out[i] = scale * weight[ids[i]] and its gradient
 * d_weight[v] = scale * (sum of d_out[i] over the i with ids[i] = v), the sum in
 * fp32 in an order that ids alone decide (runs of up to 32 in the order of i, then
 * their sums): the same bits at every run.  weight, d_weight [V, D];
 * out, d_out [N, D]; ids [N] int32 (id_bytes 4) or int64 (8).  An id outside
 * [0, V) gives a zero row and no gradient, and is reported as BCMT_ERR_ARG by
 * the next bcmt_device_status (BCMT_FLAG_CHECK: by the call).  Every row of
 * d_weight is written.  Requirements: N >= 0 (0: an empty batch), N <= 2^30,
 * 1 <= V < 2^24, D a positive multiple of 8, scale finite.  flags:
 * BCMT_FLAG_CHECK only. */
typedef struct {
  long long N;
  int V, D;
  int dtype;
  int id_bytes;
  unsigned flags;
  float scale;
} bcmt_embedding_params;

/* Bytes of workspace of bcmt_embedding_backward; 0 for invalid parameters. */
size_t bcmt_embedding_workspace_size(const bcmt_embedding_params* p);
bcmt_status bcmt_embedding_forward(const bcmt_embedding_params* p, const void* ids,
                                   const void* weight, void* out, void* stream);
bcmt_status bcmt_embedding_backward(const bcmt_embedding_params* p, const void* ids,
                                    const void* d_out, void* d_weight, void* workspace,
                                    void* stream);

/* Dropout of n elements: y_i = [residual_i +] keep_i * x_i / (1 - p), the mask
 * recomputed from (seed, offset, i) wherever it is needed and never stored: the
 * backward pass is the same call on dy (residual NULL) with the same seed and
 * offset.  Element i takes 16-bit draw i % 8 of Philox4x32-10 with key `seed`
 * and counter (i / 8, offset) -- word (i % 8) / 2, its low half first -- and is
 * kept iff the draw is at least t = round(65536 p), at most 65535 for p < 1; a
 * dropped element contributes exactly 0 even where x is infinite or NaN.  The
 * mask's rate r = 1 - t / 65536 is up to 2^-17 off 1 - p: where 1 / (1 - p) is
 * further than 2^-15 from 1 / r (for some p above 0.75), 1 / r takes its place, so
 * that the expectation of y is x to within 2^-15 for every p < 1.  Use another offset for each place
 * and step.  `step` (device memory, or NULL) is added to offset when the kernel
 * runs, so a captured graph can draw a new mask at each replay.  y may be x or
 * residual.  Requirements: n >= 0, 0 <= p <= 1.  flags: BCMT_FLAG_CHECK only. */
typedef struct {
  long long n;
  int dtype;
  unsigned flags;
  double p;
  unsigned long long seed, offset;
  const unsigned long long* step;
} bcmt_dropout_params;

bcmt_status bcmt_dropout(const bcmt_dropout_params* p, const void* x, const void* residual,
                         void* y, void* stream);

/* The end of a block and the norm before the next, over rows of D channels:
 *     z = post(branch), or branch;   h = alpha * x + gate * z;   n = pre(h),
 * post and pre both layer norms, (v - mean) / sqrt(var + eps) * weight [+ bias], or
 * both root-mean-square norms, v / sqrt(mean v^2 + eps) * weight [+ bias].
 *
 *   branch, x, h, n .. [rows, D] of dtype, dense
 *   weight, bias .. [D] of wtype: the pre norm; bias may be NULL (0)
 *   post_weight, post_bias .. [D] of wtype: the post norm; post_weight NULL: none
 *   gate     [gates, D] of dtype, row i for rows i * rows / gates and on (gates
 *            divides rows: 1 for all rows, the number of sequences, rows); NULL: 1
 *
 * Statistics and everything between the loads and the stores are fp32; n is the
 * norm of h before its rounding.  Requirements: 0 <= rows <= 2^30, 1 <= D <= 8192,
 * alpha finite, eps >= 0 and finite.  flags: BCMT_FLAG_CHECK
 * only.  h may be x or branch; no other output may overlap an input. */
typedef struct {
  long long rows;
  int D;
  int dtype, wtype; /* bcmt_dtype */
  int rms;          /* 0: layer norms, 1: root-mean-square norms */
  long long gates;  /* rows of the gate (0 where gate is NULL) */
  unsigned flags;
  float alpha, eps;
} bcmt_norm_params;

bcmt_status bcmt_residual_norm_forward(const bcmt_norm_params* p, const void* branch,
                                       const void* x, const void* weight, const void* bias,
                                       const void* post_weight, const void* post_bias,
                                       const void* gate, void* h, void* n, void* stream);

/* Bytes of workspace of the backward call (post: with a post norm), free to
 * reuse between calls; 0 for invalid parameters. */
size_t bcmt_residual_norm_workspace_size(const bcmt_norm_params* p, int post);
/* Gradients of sum(dh * h) + sum(dn * n) from the forward's branch, weights and
 * gate and its h; dh NULL: zero.  The outputs have the shape and type of what
 * they belong to; each but dbranch may be NULL (not computed).  Column sums
 * are fp32 in an order that the sizes alone decide. */
bcmt_status bcmt_residual_norm_backward(const bcmt_norm_params* p, const void* dh, const void* dn,
                                        const void* branch, const void* h, const void* weight,
                                        const void* post_weight, const void* post_bias,
                                        const void* gate, void* dbranch, void* dx, void* dweight,
                                        void* dbias, void* dpost_weight, void* dpost_bias,
                                        void* dgate, void* workspace, void* stream);

/* One AdamW step over `count` tensors in one launch (384 tensors a launch):
 *     m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,   g times *grad_scale,
 *     p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps),
 * p taken from, and written to, the float32 master too where there is one (dtype
 * bf16, all tensors or none).  bits 32: m and v are float32.  bits 8: signed and
 * unsigned bytes with one float32 scale per 256 consecutive elements of the
 * tensor (the last block may be shorter): m = c |c| s with c in -127 .. 127 and
 * s = max |m| / 127^2, sqrt(v) = c^2 r with c in 0 .. 255 and r = sqrt(max v) /
 * 255^2 of the block, each c the nearest in c (rounded up at the middle; at least
 * 1 where v > 0); a block with s < 2^-100, r < 2^-60 is held as zeros there.  What
 * decides a code is rounded to fp32 at each operation.  All zeros are states of 0.
 * A gradient that is not finite makes its element's state, in 8 bits its block's
 * scales, not finite.  step_ptr and lr_ptr (device memory, or NULL) take the
 * place of step (>= 1 there too) and lr when the kernel runs, for captured graphs.
 * Requirements: buffers of a tensor and of different tensors do not overlap;
 * 0 <= beta < 1; lr, eps, weight_decay >= 0 and finite; step >= 1.  flags:
 * BCMT_FLAG_CHECK only.  `tensors` is read during the call (host memory). */
typedef struct {
  int count;
  int dtype; /* bcmt_dtype of p and g */
  int bits;  /* 32 or 8 */
  unsigned flags;
  long long step;
  double lr, beta1, beta2, eps, weight_decay;
  const float* grad_scale; /* device memory, or NULL: 1 */
  const long long* step_ptr;
  const float* lr_ptr;
} bcmt_adamw_params;

typedef struct {
  void* p;
  const void* g;
  void* m;
  void* v;
  float* master;  /* or NULL */
  float* m_scale; /* bits 8: [ceil(n / 256)] */
  float* v_scale;
  long long n;
} bcmt_adamw_tensor;

bcmt_status bcmt_adamw_step(const bcmt_adamw_params* p, const bcmt_adamw_tensor* tensors,
                            void* stream);
/* The float32 values m, v [n] that 8-bit states of n elements stand for. */
bcmt_status bcmt_adamw_values(const void* m_codes, const float* m_scale, const void* v_codes,
                              const float* v_scale, float* m, float* v, long long n, void* stream);

/* A step of beam search.  For each of N searches, over its K beams k and the V
 * tokens v, cand[k, v] = scores[k] + logits[k, v] - log sum_u exp(logits[k, u]); a
 * beam that has ended has one candidate, token `eos` at scores[k].  The K largest
 * candidates, equal ones by the lower k V + v, become the beams: their scores,
 * parents (k), tokens (v) and whether they have ended (the parent had, or v is
 * eos).  Logits of -inf are tokens ruled out and scores of -inf beams that are not
 * there: their candidates, -inf too, come last, in the order of k V + v.
 * Candidates of one beam go by their logits.  Those of different beams are compared
 * in 64 bits, with log-sums of which only the largest terms (K of every 4096 at least)
 * are added with more than 32 bits; the others are fp32 exponentials and sums, so that a
 * log-sum is off by at most (3 ln V + 25) 2^-24, and candidates of different beams that
 * are nearer than twice that may change places.  A beam with a logit or score that is NaN or +inf
 * counts as not there and is reported as BCMT_ERR_ARG by the next
 * bcmt_device_status (BCMT_FLAG_CHECK: by the call); the logits of beams that have
 * ended, or have a score of -inf, are not read.
 *
 *   logits   [N, K, V] of dtype, rows of a stride ld >= V elements
 *   scores, scores_out [N, K] fp32;   finished [N, K] bytes, or NULL: none has
 *   parents, tokens [N, K] 64-bit;    finished_out [N, K] bytes
 *   Requirements: N >= 0, 1 <= K <= 32, 1 <= V < 2^24, N * K <= 2^22; eos < V, negative
 *   for none (not with finished).  flags: BCMT_FLAG_CHECK only.  scores_out may
 *   be scores and finished_out finished. */
typedef struct {
  int N, K, V;
  int dtype;
  int eos;
  unsigned flags;
  long long ld;
} bcmt_beam_params;

/* Bytes of workspace of bcmt_beam_select; 0 for invalid parameters. */
size_t bcmt_beam_workspace_size(const bcmt_beam_params* p);
bcmt_status bcmt_beam_select(const bcmt_beam_params* p, const void* logits, const float* scores,
                             const void* finished, float* scores_out, long long* parents,
                             long long* tokens, void* finished_out, void* workspace, void* stream);

/* dst[n, k] = src[n, parents[n, k]] for `count` tensors of N x K rows of
 * row_bytes bytes each (dense; no dst overlaps a src, parents or another dst), one launch for
 * up to 128.  A parent outside [0, K) gives a row of zeros and is reported as
 * BCMT_ERR_ARG by the next bcmt_device_status.  N * K <= 2^22, K <= 32. */
typedef struct {
  const void* src;
  void* dst;
  long long row_bytes;
} bcmt_beam_tensor;
bcmt_status bcmt_beam_reorder(const long long* parents, int N, int K,
                              const bcmt_beam_tensor* tensors, int count, unsigned flags,
                              void* stream);

/* Reads and clears the device status word of the current device after
 * synchronising `stream`: BCMT_OK, BCMT_ERR_TIMEOUT if any bounded device-side
 * wait has expired, or BCMT_ERR_ARG if an embedding id was outside its table,
 * a decay of linear attention outside [0, 1], a logit or score of beam search NaN
 * or +inf, or a parent outside its beams, since the last read. */
bcmt_status bcmt_device_status(void* stream);

/* Message describing the last error of the calling thread ("" if none). */
const char* bcmt_last_error(void);

/* Profiling (BCMT_FLAG_PROFILE): per kernel name, the number of launches and
 * the summed CUDA-event time in milliseconds recorded since the last reset.
 * Synchronises the device.  Writes up to `cap` entries; returns the number of
 * distinct kernels recorded, or -1 on error.  names[i] point to static
 * strings. */
int bcmt_profile_read(const char** names, int* launches, double* ms, int cap);
void bcmt_profile_reset(void);

#ifdef __cplusplus
}
#endif

#endif /* BCMT_H */
