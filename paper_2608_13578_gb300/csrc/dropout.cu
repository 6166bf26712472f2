// Dropout from a counter-based generator: y_i = [residual_i +] keep_i x_i / (1 - p),
// the mask recomputed from (seed, offset, i) wherever it is needed and never
// stored.  The generator is Philox4x32 with 10 rounds (Salmon, Moraes, Dror and
// Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): one counter
// value gives four 32-bit words, used as eight 16-bit draws for eight
// consecutive elements.
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace bcmt {

namespace {

// Words of counter (j, offset) under key `seed`.
__device__ __forceinline__ uint4 philox(unsigned long long j, unsigned long long offset,
                                        unsigned long long seed) {
  uint32_t c0 = (uint32_t)j, c1 = (uint32_t)(j >> 32), c2 = (uint32_t)offset,
           c3 = (uint32_t)(offset >> 32);
  uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const unsigned long long a = (unsigned long long)0xD2511F53u * c0;
    const unsigned long long b = (unsigned long long)0xCD9E8D57u * c2;
    c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)b;
    c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// Draw e (0..7) of a counter's words: 16 bits, low half of a word first.
__device__ __forceinline__ uint32_t draw16(const uint4& w, int e) {
  const uint32_t x = e < 2 ? w.x : e < 4 ? w.y : e < 6 ? w.z : w.w;
  return (e & 1) ? x >> 16 : x & 0xffffu;
}

}  // namespace

// A thread takes 8 consecutive elements (one counter); the generator is about
// 10 integer instructions per element, below what a bf16 element's bytes take:
// bandwidth-bound: 32767 x 1001 fp32 take 39.0 us (6.7 TB/s), 8192 x 512 bf16 with
// a residual 5.2.  A dropped element contributes exactly 0, whatever x holds.  y may be x
// or res (no __restrict__): a thread reads its elements before it writes them, and
// nobody else's.
template <class T, bool RES>
__global__ void __launch_bounds__(256)
    dropout_kernel(const T* x, const T* res, T* y, long long n, uint32_t threshold, float mul,
                   unsigned long long seed, unsigned long long offset,
                   const unsigned long long* __restrict__ step) {
  pdl_enter();
  if (step) offset += *step;
  const long long groups = (n + 7) / 8, stride = (long long)gridDim.x * 256;
  for (long long j = blockIdx.x * 256ll + threadIdx.x; j < groups; j += stride) {
    const long long i0 = j * 8;
    const uint4 w = philox((unsigned long long)j, offset, seed);
    if (i0 + 8 <= n) {
      float v[8], r[8];
      load8(x + i0, v);
      if (RES) load8(res + i0, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = draw16(w, e) >= threshold ? v[e] * mul : 0.f;
        v[e] = RES ? d + r[e] : d;
      }
      store8(y + i0, v);
    } else {
      for (int e = 0; i0 + e < n; ++e) {
        const float d = draw16(w, e) >= threshold ? to_f(x[i0 + e]) * mul : 0.f;
        y[i0 + e] = from_f<T>(RES ? d + to_f(res[i0 + e]) : d);
      }
    }
  }
}

namespace {
template <class T>
cudaError_t typed(const Launch& lc, const void* x, const void* res, void* y, long long n,
                  uint32_t thr, float mul, unsigned long long seed, unsigned long long offset,
                  const unsigned long long* step) {
  const long long groups = (n + 7) / 8;
  const unsigned blocks = (unsigned)std::min<long long>((groups + 255) / 256, 1ll << 20);
  cudaError_t e =
      res ? launch_k(dropout_kernel<T, true>, dim3(blocks), dim3(256), 0, lc.stream, (const T*)x,
                     (const T*)res, (T*)y, n, thr, mul, seed, offset, step)
          : launch_k(dropout_kernel<T, false>, dim3(blocks), dim3(256), 0, lc.stream, (const T*)x,
                     (const T*)nullptr, (T*)y, n, thr, mul, seed, offset, step);
  return e != cudaSuccess ? e : cudaGetLastError();
}
}  // namespace

cudaError_t dropout(const Launch& lc, int dtype, const void* x, const void* res, void* y,
                    long long n, double p, unsigned long long seed, unsigned long long offset,
                    const unsigned long long* step) {
  if (n == 0) return cudaSuccess;
  // kept iff the 16-bit draw is at least round(65536 p); p = 1 keeps nothing, and
  // nothing else does
  const uint32_t thr = p < 1.0 ? std::min((uint32_t)lrint(p * 65536.0), 65535u) : 65536u;
  // The mask keeps (65536 - thr) / 65536, up to 2^-17 off 1 - p.  The scale is 1 / (1 - p)
  // as long as the expectation is x to within 2^-15 with it (always up to p = 0.75), and
  // the mask's own beyond: 1 / (1 - p) would be 1.5 times that at p = 0.99999.
  const double kept = (65536u - thr) / 65536.0;
  const bool near = fabs(kept - (1.0 - p)) <= (1.0 - p) / 32768.0;
  const float mul = p < 1.0 ? (float)(1.0 / (near ? 1.0 - p : kept)) : 0.f;
  return dtype == 0 ? typed<float>(lc, x, res, y, n, thr, mul, seed, offset, step)
                    : typed<bf16>(lc, x, res, y, n, thr, mul, seed, offset, step);
}

}  // namespace bcmt
