// Host-side interface of beam search's step (beam.cu).
#pragma once

#include <stdint.h>

#include "internal.h"

namespace bcmt {

constexpr int kBeamMaxK = 32;

struct BeamArgs {
  int N, K, V, eos;              // eos < 0: no token ends a beam
  const void* logits;
  long long ld;                  // elements between rows
  const float* scores;
  const uint8_t* finished;       // or NULL
  float* scores_out;
  long long *parents, *tokens;
  uint8_t* finished_out;
  void* ws;
};
size_t beam_workspace(int N, int K, int V, int sms);
cudaError_t beam_select(const Launch& lc, int dtype, int sms, const BeamArgs& a);

struct ReorderTensor {
  const void* src;
  void* dst;
  long long row_bytes;
};
cudaError_t beam_reorder(const Launch& lc, const long long* parents, int N, int K,
                         const ReorderTensor* t, int count);

}  // namespace bcmt
