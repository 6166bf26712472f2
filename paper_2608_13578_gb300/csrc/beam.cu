// A step of beam search.  For every search n of N, over its K beams k and the V tokens v,
//   cand[k, v] = score[k] + x[k, v] - log sum_u exp x[k, u],
// a beam that has ended having one candidate only, its end token at the score that it
// has; the K largest, equal ones by the lower k V + v, become the beams.  Candidates of
// -inf (tokens ruled out, beams without a score) come after all others, in the order of
// their places.  The states of the beams are then copied from each new beam's parent.
//
// Selection takes two launches.  A CTA of the first reads one chunk of one row into
// registers and leaves its largest K entries, its maximum and its sum of exponentials;
// the second merges the chunks of a search.  Scores are compared in 64 bits and rounded to
// fp32 at the end.  Of a row's sum only the few large terms (those selected) are added as
// exponentials of more than 32 bits; the others are fp32: one at a distance d below the
// maximum is off by 3 d 2^-24 of itself by its argument (the difference, the factor log2 e and
// their product are rounded once each), 2^-22 by ex2.approx and 20 * 2^-24 by additions.  A
// row's terms are at ln V at most in their weighted mean, so the logarithm is off by at most
// (3 ln V + 25) 2^-24; 64-bit exponentials for all would take the chip's slow units.
#include <math.h>

#include <algorithm>

#include "beam.h"
#include "common.cuh"
#include "internal.h"

namespace bcmt {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// Sums of exponentials are integers in units of 2^-48: exact, whatever the order of the
// additions (a chunk's is below 2^62).
constexpr float kUnit = 281474976710656.f;   // 2^48
struct ChunkHead {
  unsigned long long sum;   // of exp(x - max) over the chunk
  float max;                // -inf: no entry above it; NaN: a logit is NaN or +inf
  int n;                    // entries in the list
};
struct Entry {
  float x;
  int v;
};

// The sum a + b as a float and what it lacks (Knuth's two-sum).
__device__ __forceinline__ float two_sum(float a, float b, float& rest) {
  const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
  rest = __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t));
  return s;
}
// exp(x - ref), x - ref from -86 to 0, as 2^n (h + l) to within 2^-32: the 64-bit units of
// this chip are too slow for it (a fp64 exponential took most of the merge's time).
// x - ref = n ln 2 + r with r in two floats (as Cody and Waite reduce, ln 2 split in
// three), and exp(r) = 1 + r + r^2/2 + r^3/6 + ..., the first four terms in two floats,
// Taylor's next seven in one.
__device__ __forceinline__ void exp_wide(float x, float ref, float& h, float& l, int& n) {
  float lo, t;
  const float hi = two_sum(x, -ref, lo);
  const float fn = rintf(__fmul_rn(hi, 1.44269504f));
  n = (int)fn;
  // ln 2 = 90852 / 2^17 + kLn2b, the first exact in every product with n
  constexpr double kLn2 = 0.693147180559945309417;
  constexpr float kLn2a = 90852.f / 131072.f, kLn2b = (float)(kLn2 - 90852.0 / 131072.0),
                  kLn2c = (float)(kLn2 - 90852.0 / 131072.0 - (double)kLn2b);
  const float r1 = __fmaf_rn(-fn, kLn2a, hi);
  const float p = __fmul_rn(fn, kLn2b), pe = __fmaf_rn(fn, kLn2b, -p);
  float u;
  const float s0 = two_sum(r1, -p, u), s = two_sum(s0, u + (lo - pe - fn * kLn2c), t);
  // r^2 and r^3 / 6 as two floats
  const float a = __fmul_rn(s, s), ae = __fmaf_rn(s, s, -a) + 2.f * s * t;
  const float b = __fmul_rn(a, s), be = __fmaf_rn(a, s, -b) + ae * s + a * t;
  constexpr float kSixth = (float)(1.0 / 6.0), kSixthRest = (float)(1.0 / 6.0 - (double)kSixth);
  const float m = __fmul_rn(b, kSixth), me = __fmaf_rn(b, kSixth, -m) + b * kSixthRest + be * kSixth;
  float q = 1.f / 3628800.f;
  q = fmaf(q, s, 1.f / 362880.f);
  q = fmaf(q, s, 1.f / 40320.f);
  q = fmaf(q, s, 1.f / 5040.f);
  q = fmaf(q, s, 1.f / 720.f);
  q = fmaf(q, s, 1.f / 120.f);
  q = fmaf(q, s, 1.f / 24.f);
  float e0, e1, e2, e3;
  h = two_sum(1.f, s, e0);
  h = two_sum(h, 0.5f * a, e1);
  h = two_sum(h, m, e2);
  h = two_sum(h, a * a * q, e3);
  l = ((e0 + e1) + (e2 + e3)) + (t + (0.5f * ae + me));
}
__device__ __forceinline__ unsigned long long exp_units(float x, float ref) {
  if (!(x - ref > -34.f)) return 0;   // below half a unit
  float h, l;
  int n;
  exp_wide(x, ref, h, l, n);
  const float scale = __int_as_float((n + 48 + 127) << 23);
  return (unsigned long long)(__float2ll_rn(h * scale) + __float2ll_rn(l * scale));
}
__device__ __forceinline__ double exp_double(float x, float ref) {
  if (!(x - ref > -86.f)) return 0.0;
  float h, l;
  int n;
  exp_wide(x, ref, h, l, n);
  const float scale = __int_as_float((n + 127) << 23);
  return (double)(h * scale) + (double)(l * scale);
}

template <class T, int E, bool VEC>
__device__ __forceinline__ int column(int j, int e) {   // of element e of group j, in the chunk
  return VEC ? (j * kThreads + (int)threadIdx.x) * 8 + e : (j * 8 + e) * kThreads + (int)threadIdx.x;
}

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Sorted over the lanes, the largest first.
__device__ __forceinline__ float warp_sort(float v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1) {
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) {
      const float o = __shfl_xor_sync(0xffffffffu, v, j);
      const bool low = (lane & j) == 0, down = (lane & k) == 0;
      v = low == down ? fmaxf(v, o) : fminf(v, o);
    }
  }
  return v;
}
// The largest 32 of two such lists, sorted again.
__device__ __forceinline__ float warp_merge(float a, float b) {
  const int lane = threadIdx.x & 31;
  float v = fmaxf(a, __shfl_sync(0xffffffffu, b, 31 - lane));
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    const float o = __shfl_xor_sync(0xffffffffu, v, j);
    v = (lane & j) == 0 ? fmaxf(v, o) : fminf(v, o);
  }
  return v;
}

}  // namespace

// One chunk of one row.  The threshold is the K-th largest of the threads' maxima: at
// least K elements reach it, and those above it belong to fewer than K threads.  Elements
// equal to it are taken too; where they are too many (rows of one value), those up to the
// K-th lowest place among the threads' first ones, which are in K threads.  Up to kCoarseK
// beams the maxima of every eight threads give a threshold that is found in one sort, and
// lets few more elements through (K = 8: 9 of 4096); where they are too many, the other
// follows.  What every chunk pays whatever passes its threshold (a sort, a ranking, four
// barriers) and issue slots (53%) decide: 64 x 8 x 32000 bf16 30 us (5 at the copy's rate; 32 with
// the fine threshold), 40 x 5 x 50257 fp32 16 us.  Element by element 16 take 36 bytes of spills.
constexpr int kCoarseK = 16;
template <class T, int E, bool VEC>
__global__ void __launch_bounds__(kThreads, E == 16 ? 4 : 5) beam_chunk_kernel(const BeamArgs a, int nchunk) {
  constexpr int J = E / 8, kCap = 2 * kBeamMaxK * E;
  __shared__ float tops[kWarps][32];
  __shared__ Entry list[kCap];
  __shared__ unsigned long long total;
  __shared__ int bad;
  __shared__ float thr, most;
  __shared__ int cnt;
  pdl_enter();
  const long long row = blockIdx.x / nchunk;
  const int chunk = blockIdx.x - (int)(row * nchunk);
  // a beam that has ended or has no score takes nothing from its row
  const float score = a.scores[row];
  if ((a.finished && a.finished[row]) || !(score > -INFINITY && score < INFINITY)) return;
  const int base = chunk * E * kThreads, V = a.V, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld + base;
  const int left = V - base;
  float v[E], top = -INFINITY;
  if (VEC) {
    if (sizeof(T) == 2) {
      uint4 raw[J];
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int c = column<T, E, VEC>(j, 0);
        if (c < left) load8_raw(reinterpret_cast<const bf16*>(x) + c, raw[j]);
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if (column<T, E, VEC>(j, 0) < left) unpack8(raw[j], v + 8 * j);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) v[8 * j + e] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int c = column<T, E, VEC>(j, 0);
        if (c < left) load8(x + c, v + 8 * j);
        else
#pragma unroll
          for (int e = 0; e < 8; ++e) v[8 * j + e] = -INFINITY;
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = column<T, E, VEC>(j, e);
        v[8 * j + e] = c < left ? to_f(x[c]) : -INFINITY;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < E; ++i) top = fmaxf(top, v[i]);
  if (threadIdx.x == 0) {
    cnt = 0;
    total = 0;
    bad = 0;
  }
  // the K-th largest of the threads' values, in every thread; top: the largest
  auto kth = [&](float value, float& largest) {
    tops[warp][lane] = warp_sort(value);
    __syncthreads();
    if (warp == 0) {
      float p[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) p[w] = tops[w][lane];
#pragma unroll
      for (int m = kWarps / 2; m > 0; m >>= 1)
#pragma unroll
        for (int w = 0; w < m; ++w) p[w] = warp_merge(p[w], p[w + m]);
      if (lane == a.K - 1) thr = p[0];
      if (lane == 0) most = p[0];
    }
    __syncthreads();
    largest = most;
    return thr;
  };
  float limit, mx;
  const bool coarse = a.K <= kCoarseK;
  if (coarse) {   // of the largest of every eight threads
    float g = top;
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, o));
    if ((lane & 7) == 0) tops[0][warp * 4 + lane / 8] = g;
    __syncthreads();
    if (warp == 0) {
      g = warp_sort(tops[0][lane]);
      if (lane == a.K - 1) thr = g;
      if (lane == 0) most = g;
    }
    __syncthreads();
    limit = thr;
    mx = most;
  } else {
    limit = kth(top, mx);
  }
  // exp(x - max) = 2^(x log2 e - max log2 e); where nothing is finite, 0 or NaN
  constexpr float kLog2e = 1.4426950408889634f;
  const float ref = mx == -INFINITY ? 0.f : mx;
  // elements from the threshold up go into the list (a thread's one after another, a place in it
  // for a warp by one atomic addition), the others into the sum
  float s;
  auto collect = [&] {
    int mine = 0;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const bool hit = v[i] >= limit && v[i] > -INFINITY;
      mine += hit;
      const float e = exp2_fast((v[i] - ref) * kLog2e);
      s += hit ? 0.f : e;
    }
    if (__any_sync(0xffffffffu, mine)) {
      int before = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += up;
      }
      int from = 0;
      if (lane == 31) from = atomicAdd(&cnt, before);
      from = __shfl_sync(0xffffffffu, from, 31) + before - mine;
      if (mine) {
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (v[i] >= limit && v[i] > -INFINITY) {
            if (from < kCap) list[from] = Entry{v[i], column<T, E, VEC>(i / 8, i % 8)};
            ++from;
          }
      }
    }
    __syncthreads();
    return cnt;
  };
  int n = collect();
  unsigned long long part = 0;
  auto empty = [&] {
    __syncthreads();
    if (threadIdx.x == 0) cnt = 0;
    __syncthreads();
  };
  if (n > kCap && coarse) {
    empty();
    limit = kth(top, mx);
    n = collect();
  }
  if (n > kCap) {
    // many elements equal to the threshold: the lowest places among them, up to the K-th
    // lowest of the threads' first places (as floats: below 2^24)
    int first = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (v[i] == limit) first = min(first, column<T, E, VEC>(i / 8, i % 8));
    empty();
    float lowest;
    const float place = kth(first == 0x7fffffff ? -INFINITY : -(float)first, lowest);
    const int limit_at = place == -INFINITY ? 0x7fffffff : (int)-place;
    const unsigned long long one = exp_units(limit, ref);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int c = column<T, E, VEC>(i / 8, i % 8);
      if (v[i] > limit || (v[i] == limit && c <= limit_at)) {
        const int at = atomicAdd(&cnt, 1);
        if (at < kCap) list[at] = Entry{v[i], c};
      } else if (v[i] == limit) {
        part += one;
      }
    }
    __syncthreads();
    n = min(cnt, kCap);
  }
  // the list in order, and its exponentials
  Entry* out = reinterpret_cast<Entry*>(static_cast<char*>(a.ws) +
                                        (size_t)a.N * a.K * nchunk * sizeof(ChunkHead)) +
               (row * nchunk + chunk) * a.K;
  // eight threads find an entry's rank
  for (int i0 = 0; i0 < n; i0 += kThreads / 8) {
    const int i = i0 + threadIdx.x / 8;
    const Entry m = i < n ? list[i] : Entry{0.f, 0};
    int rank = 0;
    for (int k = threadIdx.x & 7; k < n; k += 8) {
      const Entry o = list[k];
      rank += o.x > m.x || (o.x == m.x && o.v < m.v);
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
    if ((threadIdx.x & 7) == 0 && i < n && rank < a.K) out[rank] = Entry{m.x, base + m.v};
  }
  for (int i = threadIdx.x; i < n; i += kThreads) part += exp_units(list[i].x, ref);
  // the others' sum of this warp; not finite where a logit is NaN or +inf
  s = warp_sum(s);
  if (lane == 0) {
    if (s < 1e9f) part += (unsigned long long)__float2ll_rn(s * kUnit);
    else bad = 1;
  }
  if (part) atomicAdd(&total, part);
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool ok = !bad && mx < INFINITY;
    static_cast<ChunkHead*>(a.ws)[row * nchunk + chunk] =
        ChunkHead{total, ok ? mx : __int_as_float(0x7fffffff), min(n, a.K)};
  }
}

namespace {

// A candidate: a 64-bit key that orders as its value, the larger the better, and its
// place, the lower the better.  Comparisons are of integers.
struct Cand {
  long long key;
  int at;
};
constexpr int kNoPlace = 0x7fffffff;
constexpr long long kNoKey = -0x7fffffffffffffffll - 1;

__device__ __forceinline__ bool before(const Cand& a, const Cand& b) {
  return a.key > b.key || (a.key == b.key && a.at < b.at);
}
__device__ __forceinline__ Cand shfl(const Cand& a, int from) {
  return Cand{__shfl_sync(0xffffffffu, a.key, from), __shfl_sync(0xffffffffu, a.at, from)};
}
__device__ __forceinline__ Cand settle(Cand v) {   // a bitonic sequence over the lanes, sorted
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    const Cand o = shfl(v, lane ^ j);
    if (before(o, v) == ((lane & j) == 0)) v = o;
  }
  return v;
}
// The best 32 of two lists that are sorted over the lanes, sorted again.
__device__ __forceinline__ Cand merge(const Cand& a, const Cand& b) {
  Cand v = shfl(b, 31 - (threadIdx.x & 31));
  if (before(a, v)) v = a;
  return settle(v);
}
// Entries of one beam: the logit's order above, the lower place the better below.
typedef unsigned long long Packed;
__device__ __forceinline__ Packed settle(Packed v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    const Packed o = __shfl_xor_sync(0xffffffffu, v, j);
    if ((o > v) == ((lane & j) == 0)) v = o;
  }
  return v;
}
__device__ __forceinline__ Packed sorted(Packed v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 2; k <= 32; k <<= 1) {
#pragma unroll
    for (int j = k >> 1; j > 0; j >>= 1) {
      const Packed o = __shfl_xor_sync(0xffffffffu, v, j);
      if ((o > v) == (((lane & j) == 0) == ((lane & k) == 0))) v = o;
    }
  }
  return v;
}
__device__ __forceinline__ Packed merge(Packed a, Packed b) {
  const Packed v = __shfl_sync(0xffffffffu, b, 31 - (threadIdx.x & 31));
  return settle(a > v ? a : v);
}
// Floats and doubles (no NaN, no -0) as integers of the same order.
__device__ __forceinline__ int ordered(float x) {
  const int b = __float_as_int(x + 0.f);
  return b < 0 ? b ^ 0x7fffffff : b;
}
__device__ __forceinline__ long long ordered(double x) {
  const long long b = __double_as_longlong(x);
  return b < 0 ? b ^ 0x7fffffffffffffffll : b;
}
__device__ __forceinline__ double value(long long key) {
  return __longlong_as_double(key < 0 ? key ^ 0x7fffffffffffffffll : key);
}

}  // namespace

// One search, one warp a beam: the sum of its row and the best K of its chunks' lists,
// then the beams' lists in pairs.  Latency decides: 9 us for 64 x 8 beams, 20 for 4 x 32.
__global__ void __launch_bounds__(32 * kBeamMaxK) beam_merge_kernel(const BeamArgs a, int nchunk,
                                                                    unsigned* status) {
  __shared__ Cand lists[kBeamMaxK][32];
  pdl_enter();
  const int n = blockIdx.x, K = a.K, lane = threadIdx.x & 31, k = threadIdx.x >> 5;
  const size_t row = (size_t)n * K + k;
  const ChunkHead* heads = static_cast<const ChunkHead*>(a.ws) + row * nchunk;
  const Entry* entries = reinterpret_cast<const Entry*>(static_cast<const char*>(a.ws) +
                                                        (size_t)a.N * K * nchunk * sizeof(ChunkHead)) +
                         row * nchunk * K;
  const float score = a.scores[row];
  const bool ended = a.finished && a.finished[row];
  const bool there = score > -INFINITY && score < INFINITY;
  if (lane == 0 && !(score < INFINITY)) atomicOr(status, kStatusBadLogit);
  Cand best{kNoKey, kNoPlace};
  if (there && ended) {
    if (lane == 0) best = Cand{ordered((double)score), k * a.V + a.eos};
  } else if (there) {
    // the best of the lists by logit; the first 32 heads stay for the sum
    ChunkHead h{0, -INFINITY, 0};
    if (lane < nchunk) h = heads[lane];
    // (the lists' first entries, then their second ones and so on: up to 32 lists, where no entry
    // of a turn is among the best, none that follows is)
    const int total = nchunk * K;
    Packed found = 0, last = 0;
    for (int i = 0; i < total; i += 32) {
      const int rank = (i + lane) / nchunk, l = i + lane - rank * nchunk;
      Packed c = 0;
      if (i + lane < total && rank < heads[l].n) {
        const Entry e = entries[l * K + rank];
        c = (Packed)((uint32_t)ordered(e.x) ^ 0x80000000u) << 32 | ~(uint32_t)e.v;
      }
      if (!__any_sync(0xffffffffu, c > last)) {
        if (nchunk <= 32) break;
        continue;
      }
      found = i == 0 ? sorted(c) : merge(found, sorted(c));
      last = __shfl_sync(0xffffffffu, found, K - 1);
    }
    float m = h.max;
    bool ok = m == m;
    for (int c = lane + 32; c < nchunk; c += 32) {
      ok = ok && heads[c].max == heads[c].max;
      m = fmaxf(m, heads[c].max);
    }
    ok = __all_sync(0xffffffffu, ok);
    if (!ok && lane == 0) atomicOr(status, kStatusBadLogit);
    m = warp_max(m);
    if (ok && m > -INFINITY) {
      double s = (double)h.sum * exp_double(h.max, m);
      for (int c = lane + 32; c < nchunk; c += 32) s += (double)heads[c].sum * exp_double(heads[c].max, m);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      s *= 0x1p-48;
      // log s: a float y near it, and log(s exp(-y)) from its series
      const float y = logf((float)s);
      const double z = s * exp_double(-y, 0.f) - 1.0;
      const double log_s = (double)y + (z - 0.5 * z * z);
      if (found) {
        const int o = (int)((uint32_t)(found >> 32) ^ 0x80000000u);
        const float x = __int_as_float(o < 0 ? o ^ 0x7fffffff : o);
        best = Cand{ordered((double)score + (((double)x - (double)m) - log_s)),
                    k * a.V + (int)~(uint32_t)found};
      }
    }
  }
  lists[k][lane] = best;
  for (int m = 1; m < K; m *= 2) {
    __syncthreads();
    if (k % (2 * m) == 0 && k + m < K) {
      best = merge(best, lists[k + m][lane]);
      lists[k][lane] = best;
    }
  }
  if (k != 0) return;
  // places of -inf fill what is left, the lowest first: those that are not among the selected
  const int have = __popc(__ballot_sync(0xffffffffu, lane < K && best.at != kNoPlace));
  int place = best.at;
  for (int at = 0, filled = 0; filled < K - have; ++at) {
    if (__any_sync(0xffffffffu, lane < have && place == at)) continue;
    if (lane == have + filled) place = at;
    ++filled;
  }
  if (lane < K) {
    const size_t o = (size_t)n * K + lane;
    const int parent = place / a.V, v = place - parent * a.V;
    const bool was = a.finished && a.finished[(size_t)n * K + parent];
    a.scores_out[o] = lane < have ? (float)value(best.key) : -INFINITY;
    a.parents[o] = parent;
    a.tokens[o] = v;
    lists[0][lane].at = was || v == a.eos;
  }
  // finished_out may be finished: written after all of it has been read
  __syncwarp();
  if (lane < K) a.finished_out[(size_t)n * K + lane] = (uint8_t)lists[0][lane].at;
}

namespace {

struct ReorderTable {
  static constexpr int kMax = 128;
  ReorderTensor t[kMax];
  int first[kMax + 1];   // pieces before each tensor's
  int count, N, K;
  const long long* parents;
  unsigned* status;
};
constexpr int kPiece = 4096;   // bytes of a row that a CTA copies

}  // namespace

// A CTA copies one piece of the rows of one search: beams with a parent in common read
// it while it is in the caches (64 x 8 beams of 6 layers of 8 x 64 x 64: 96 us, 6.9 TB/s).
// Rows of 16-byte multiples in 16-byte steps, others in single bytes.
__global__ void __launch_bounds__(256) beam_reorder_kernel(const __grid_constant__ ReorderTable a) {
  pdl_enter();
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.first[mid] <= (int)blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const ReorderTensor t = a.t[lo];
  const long long pieces = (t.row_bytes + kPiece - 1) / kPiece;
  const long long id = (int)blockIdx.x - a.first[lo], n = id / pieces, at = (id - n * pieces) * kPiece;
  const char* src = static_cast<const char*>(t.src) + n * a.K * t.row_bytes + at;
  char* dst = static_cast<char*>(t.dst) + n * a.K * t.row_bytes + at;
  const long long left = t.row_bytes - at;
  const bool wide = ((reinterpret_cast<uintptr_t>(t.src) | reinterpret_cast<uintptr_t>(t.dst) |
                      (uintptr_t)t.row_bytes) & 15) == 0;
  const int off = threadIdx.x * 16;
#pragma unroll 4
  for (int k = 0; k < a.K; ++k) {
    const long long parent = a.parents[n * a.K + k];
    const bool ok = parent >= 0 && parent < a.K;
    if (!ok && threadIdx.x == 0 && at == 0) atomicOr(a.status, kStatusBadParent);
    const char* s = src + (ok ? parent : 0) * t.row_bytes;
    char* d = dst + k * t.row_bytes;
    if (wide) {
      if (off < left) {
        uint4 v = *reinterpret_cast<const uint4*>(s + off);
        if (!ok) v = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(d + off) = v;
      }
    } else {
      for (int i = threadIdx.x; i < kPiece && i < left; i += 256) d[i] = ok ? s[i] : 0;
    }
  }
}

namespace {

// Elements per thread of a chunk: 16 where that gives every SM work, else 8, for more
// CTAs on few rows.
int chunk_elements(int N, int K, int V, int sms) {
  const long long big = (V + 16 * kThreads - 1) / (16 * kThreads);
  return (long long)N * K * big >= sms ? 16 : 8;
}

template <class T, int E>
cudaError_t chunks(const Launch& lc, const BeamArgs& a, int nchunk) {
  const dim3 grid((unsigned)((long long)a.N * a.K * nchunk));
  const bool vec = a.V % 8 == 0 && a.ld % 8 == 0 && (uintptr_t)a.logits % 16 == 0;
  return vec ? launch_k(beam_chunk_kernel<T, E, true>, grid, dim3(kThreads), 0, lc.stream, a, nchunk)
             : launch_k(beam_chunk_kernel<T, E, false>, grid, dim3(kThreads), 0, lc.stream, a, nchunk);
}

}  // namespace

size_t beam_workspace(int N, int K, int V, int sms) {
  const int chunk = chunk_elements(N, K, V, sms) * kThreads, nchunk = (V + chunk - 1) / chunk;
  return (size_t)N * K * nchunk * (sizeof(ChunkHead) + K * sizeof(Entry));
}

cudaError_t beam_select(const Launch& lc, int dtype, int sms, const BeamArgs& a) {
  if (a.N == 0) return cudaSuccess;
  const int e = chunk_elements(a.N, a.K, a.V, sms);
  const int nchunk = (a.V + e * kThreads - 1) / (e * kThreads);
  cudaError_t err = dtype == 0 ? e == 16 ? chunks<float, 16>(lc, a, nchunk) : chunks<float, 8>(lc, a, nchunk)
                    : e == 16  ? chunks<bf16, 16>(lc, a, nchunk)
                               : chunks<bf16, 8>(lc, a, nchunk);
  if (err != cudaSuccess) return err;
  return launch_k(beam_merge_kernel, dim3(a.N), dim3(a.K * 32), 0, lc.stream, a, nchunk, lc.status);
}

cudaError_t beam_reorder(const Launch& lc, const long long* parents, int N, int K,
                         const ReorderTensor* t, int count) {
  ReorderTable a;
  a.N = N;
  a.K = K;
  a.parents = parents;
  a.status = lc.status;
  a.count = 0;
  long long blocks = 0;
  cudaError_t err = cudaSuccess;
  auto flush = [&] {
    if (a.count > 0)
      err = launch_k(beam_reorder_kernel, dim3((unsigned)blocks), dim3(256), 0, lc.stream, a);
    a.count = 0;
    blocks = 0;
  };
  for (int i = 0; i < count && err == cudaSuccess; ++i) {
    if (t[i].row_bytes == 0 || N == 0) continue;
    const long long need = N * ((t[i].row_bytes + kPiece - 1) / kPiece);
    if (need > 0x7fffffffll) return cudaErrorInvalidValue;
    if (a.count == ReorderTable::kMax || blocks + need > 0x7fffffffll) flush();
    a.t[a.count] = t[i];
    a.first[a.count++] = (int)blocks;
    blocks += need;
  }
  if (err == cudaSuccess) flush();
  return err;
}

}  // namespace bcmt
