// Host-side interface of the AdamW step over many tensors (adamw.cu).
#pragma once

#include <stdint.h>

#include "internal.h"

namespace bcmt {

struct AdamwTensor {
  void* p;
  const void* g;
  void *m, *v;                            // float, or codes of 8 bits
  float *master, *m_scale, *v_scale;      // NULL where there is none
  long long n;
};

// Hyperparameters as the kernel uses them; step_ptr and lr_ptr replace step and lr by
// values that are read when the kernel runs.
struct AdamwHyper {
  float b1, omb1, b2, omb2, eps, lr, decay, rate, keep, ib2;
  double log_b1, log_b2;
  long long step;
  const long long* step_ptr;
  const float *lr_ptr, *grad_scale;
};

struct AdamwEntry {
  void* p;
  const void* g;
  void *m, *v;
  float *master, *m_scale, *v_scale;
  long long n;
  unsigned first;   // the tensor's first CTA
  int vec;          // every buffer starts at a multiple of 16 bytes
};
template <int CAP>
struct AdamwTable {
  AdamwEntry e[CAP];
  AdamwHyper h;
  int count, chunk;   // tensors; elements of a CTA
};

cudaError_t adamw_step(const Launch& lc, int dtype, int bits, bool master, const AdamwHyper& h,
                       const AdamwTensor* t, int count);
cudaError_t adamw_values(const Launch& lc, const uint8_t* mc, const float* ms, const uint8_t* vc,
                         const float* vs, float* m, float* v, long long n);

}  // namespace bcmt
