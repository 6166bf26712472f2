// A step of beam search.  For every search n of N, over its K beams k and the V tokens v,
//   cand[k, v] = score[k] + x[k, v] - log sum_u exp x[k, u],
// a beam that has ended having one candidate only, its end token at the score that it
// has; the K largest, equal ones by the lower k V + v, become the beams.  Candidates of
// -inf (tokens ruled out, beams without a score) come after all others, in the order of
// their places.  The states of the beams are then copied from each new beam's parent.
//
// Selection takes two launches.  A CTA of the first reads one chunk of one row into
// registers and leaves its largest K entries, its maximum and its sum of exponentials;
// the second merges the chunks of a search.  What decides between beams is held in 64
// bits: a sum's few large terms (those selected) are added as 64-bit exponentials, the
// others in fp32, and scores are rounded to fp32 at the end.
#include <math.h>

#include <algorithm>

#include "beam.h"
#include "common.cuh"
#include "internal.h"

namespace bcmt {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

struct ChunkHead {
  double sum;   // of exp(x - max) over the chunk
  float max;    // -inf: no entry above it
  int n;        // entries in the list
};
struct Entry {
  float x;
  int v;
};

template <class T, int E, bool VEC>
__device__ __forceinline__ int column(int j, int e) {   // of element e of group j, in the chunk
  return VEC ? (j * kThreads + (int)threadIdx.x) * 8 + e : (j * 8 + e) * kThreads + (int)threadIdx.x;
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
// K-th lowest place among the threads' first ones, which are in K threads.
template <class T, int E, bool VEC>
__global__ void __launch_bounds__(kThreads) beam_chunk_kernel(const BeamArgs a, int nchunk) {
  constexpr int J = E / 8, kCap = 2 * kBeamMaxK * E;
  __shared__ float tops[kWarps][32];
  __shared__ Entry list[kCap];
  __shared__ double sums[kWarps];
  __shared__ unsigned long long listed;
  __shared__ float thr;
  __shared__ int cnt, tie;
  pdl_enter();
  const long long row = blockIdx.x / nchunk;
  const int chunk = blockIdx.x - (int)(row * nchunk);
  // a beam that has ended or has no score takes nothing from its row
  const float score = a.scores[row];
  if ((a.finished && a.finished[row]) || !(score > -INFINITY && score < INFINITY)) return;
  const int base = chunk * E * kThreads, V = a.V, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld + base;
  const int left = V - base;
  float v[E], gmax[J], top = -INFINITY;
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
  for (int j = 0; j < J; ++j) {
    gmax[j] = v[8 * j];
#pragma unroll
    for (int e = 1; e < 8; ++e) gmax[j] = fmaxf(gmax[j], v[8 * j + e]);
    top = fmaxf(top, gmax[j]);
  }
  if (threadIdx.x == 0) {
    cnt = 0;
    listed = 0;
  }
  tops[warp][lane] = warp_sort(top);
  __syncthreads();
  if (warp == 0) {
    float s[kWarps];
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s[w] = tops[w][lane];
#pragma unroll
    for (int n = kWarps / 2; n > 0; n >>= 1)
#pragma unroll
      for (int w = 0; w < n; ++w) s[w] = warp_merge(s[w], s[w + n]);
    if (lane == a.K - 1) thr = s[0];
    if (lane == 0) tops[0][0] = s[0];
  }
  __syncthreads();
  const float limit = thr, mx = tops[0][0];
  // exp(x - max) = 2^(x log2 e - max log2 e); where nothing is finite, 0 or NaN
  constexpr float kLog2e = 1.4426950408889634f;
  const bool none = mx == -INFINITY;
  const float ref = none ? 0.f : mx;
  float s = 0.f;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    if (!(gmax[j] >= limit) || none) {
#pragma unroll
      for (int e = 0; e < 8; ++e) s += exp2f((v[8 * j + e] - ref) * kLog2e);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = v[8 * j + e];
        if (u >= limit && u > -INFINITY) {
          const int at = atomicAdd(&cnt, 1);
          if (at < kCap) list[at] = Entry{u, column<T, E, VEC>(j, e)};
        } else {
          s += exp2f((u - ref) * kLog2e);
        }
      }
    }
  }
  __syncthreads();
  int n = cnt;
  double d = s;
  if (n > kCap) {
    // many elements equal to the threshold: the lowest places among them
    __syncthreads();
    int first = 0x7fffffff;
#pragma unroll
    for (int i = 0; i < E; ++i)
      if (v[i] == limit) first = min(first, column<T, E, VEC>(i / 8, i % 8));
    // the K-th smallest of the threads' first places (as floats: below 2^24)
    tops[warp][lane] = warp_sort(first == 0x7fffffff ? -INFINITY : -(float)first);
    if (threadIdx.x == 0) cnt = 0;
    __syncthreads();
    if (warp == 0) {
      float p[kWarps];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) p[w] = tops[w][lane];
#pragma unroll
      for (int m = kWarps / 2; m > 0; m >>= 1)
#pragma unroll
        for (int w = 0; w < m; ++w) p[w] = warp_merge(p[w], p[w + m]);
      if (lane == a.K - 1) tie = p[0] == -INFINITY ? 0x7fffffff : (int)-p[0];
    }
    __syncthreads();
    const int limit_at = tie;
    const double one = exp((double)limit - (double)ref);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int c = column<T, E, VEC>(i / 8, i % 8);
      if (v[i] > limit || (v[i] == limit && c <= limit_at)) {
        const int at = atomicAdd(&cnt, 1);
        if (at < kCap) list[at] = Entry{v[i], c};
      } else if (v[i] == limit) {
        d += one;
      }
    }
    __syncthreads();
    n = min(cnt, kCap);
  }
  // the list's part of the sum in units of 2^-52: an integer, whatever the order in which
  // the entries came here
  Entry* out = reinterpret_cast<Entry*>(static_cast<char*>(a.ws) +
                                        (size_t)a.N * a.K * nchunk * sizeof(ChunkHead)) +
               (row * nchunk + chunk) * a.K;
  unsigned long long part = 0;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const Entry m = list[i];
    int rank = 0;
    for (int k = 0; k < n; ++k) {
      const Entry o = list[k];
      rank += o.x > m.x || (o.x == m.x && o.v < m.v);
    }
    part += (unsigned long long)(exp((double)m.x - (double)ref) * 0x1p52);
    if (rank < a.K) out[rank] = Entry{m.x, base + m.v};
  }
  if (part) atomicAdd(&listed, part);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
  if (lane == 0) sums[warp] = d;
  __syncthreads();
  if (threadIdx.x == 0) {
    d = (double)listed * 0x1p-52;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) d += sums[w];
    static_cast<ChunkHead*>(a.ws)[row * nchunk + chunk] = ChunkHead{d, mx, min(n, a.K)};
  }
}

namespace {

// A candidate: the value in 64 bits and its place k V + v.  Places are below 2^31.
struct Cand {
  double c;
  int at;
};
__device__ __forceinline__ bool before(const Cand& a, const Cand& b) {
  return a.c > b.c || (a.c == b.c && a.at < b.at);
}
__device__ __forceinline__ Cand shfl(const Cand& a, int from) {
  return Cand{__shfl_sync(0xffffffffu, a.c, from), __shfl_sync(0xffffffffu, a.at, from)};
}
// The best 32 of two lists that are sorted over the lanes, sorted again.
__device__ __forceinline__ Cand merge(const Cand& a, const Cand& b) {
  const int lane = threadIdx.x & 31;
  Cand v = shfl(b, 31 - lane);
  if (before(a, v)) v = a;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    const Cand o = shfl(v, lane ^ j);
    if (before(o, v) == ((lane & j) == 0)) v = o;
  }
  return v;
}
constexpr int kNoPlace = 0x7fffffff;

}  // namespace

// One search: the sums of its beams, then the lists of its chunks, each warp a part of
// them, then the warps' lists in pairs.
__global__ void __launch_bounds__(1024) beam_merge_kernel(const BeamArgs a, int nchunk,
                                                          unsigned* status) {
  __shared__ double tops[kBeamMaxK], logs[kBeamMaxK], base[kBeamMaxK];
  __shared__ int kind[kBeamMaxK];   // 0: candidates in the lists, 1: ended, 2: none
  __shared__ Cand lists[32][32];
  pdl_enter();
  const int n = blockIdx.x, K = a.K, lane = threadIdx.x & 31, warp = threadIdx.x >> 5,
            warps = blockDim.x >> 5;
  const ChunkHead* heads = static_cast<const ChunkHead*>(a.ws) + (size_t)n * K * nchunk;
  const Entry* entries = reinterpret_cast<const Entry*>(
                             static_cast<const char*>(a.ws) +
                             (size_t)a.N * K * nchunk * sizeof(ChunkHead)) +
                         (size_t)n * K * nchunk * K;
  for (int k = warp; k < K; k += warps) {
    const float score = a.scores[(size_t)n * K + k];
    const bool ended = a.finished && a.finished[(size_t)n * K + k];
    int what = !(score > -INFINITY && score < INFINITY) ? 2 : ended ? 1 : 0;
    double top = 0.0, total = 1.0;
    if (what == 0) {
      float m = -INFINITY;
      for (int c = lane; c < nchunk; c += 32) m = fmaxf(m, heads[k * nchunk + c].max);
      m = warp_max(m);
      double s = 0.0;
      for (int c = lane; c < nchunk; c += 32) {
        const ChunkHead h = heads[k * nchunk + c];
        // a chunk without a finite element adds its 0, or the NaN that it holds
        s += h.max == -INFINITY ? h.sum : h.sum * exp((double)h.max - (double)m);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (!(s < INFINITY) || !(m < INFINITY)) {
        what = 2;   // a logit is NaN or +inf
        if (lane == 0) atomicOr(status, kStatusBadLogit);
      } else if (m == -INFINITY) {
        what = 2;
      } else {
        top = m;
        total = s;
      }
    }
    if (lane == 0) {
      if (!(score < INFINITY)) atomicOr(status, kStatusBadLogit);
      kind[k] = what;
      tops[k] = top;
      logs[k] = log(total);
      base[k] = score;
    }
  }
  __syncthreads();
  Cand best{-INFINITY, kNoPlace};
  if (warp == 0) {   // ended beams: one candidate each
    Cand c{-INFINITY, kNoPlace};
    if (lane < K && kind[lane] == 1) c = Cand{base[lane], lane * a.V + a.eos};
    // in order: each lane to the number of those before it
    int rank = 0;
    for (int i = 0; i < 32; ++i) {
      const Cand o = shfl(c, i);
      rank += before(o, c) || (o.c == c.c && o.at == c.at && i < lane);
    }
    for (int i = 0; i < 32; ++i) {
      const int r = __shfl_sync(0xffffffffu, rank, i);
      const Cand o = shfl(c, i);
      if (lane == r) best = o;
    }
  }
  Cand last = shfl(best, K - 1);
  for (int l = warp; l < K * nchunk; l += warps) {
    const int k = l / nchunk;
    if (kind[k] != 0) continue;
    const int cnt = heads[l].n;
    Cand c{-INFINITY, kNoPlace};
    if (lane < cnt) {
      const Entry e = entries[(size_t)l * K + lane];
      c = Cand{base[k] + (((double)e.x - tops[k]) - logs[k]), k * a.V + e.v};
    }
    // the list's first is its best: nothing to do where that is past the K-th so far
    if (!before(shfl(c, 0), last)) continue;
    best = merge(best, c);
    last = shfl(best, K - 1);
  }
  lists[warp][lane] = best;
  for (int m = 1; m < warps; m *= 2) {
    __syncthreads();
    if (warp % (2 * m) == 0 && warp + m < warps) {
      best = merge(best, lists[warp + m][lane]);
      lists[warp][lane] = best;
    }
  }
  if (warp != 0) return;
  // places of -inf fill what is left, the lowest first: the places below 2 K that are not
  // among the selected, in order
  const int have = __popc(__ballot_sync(0xffffffffu, lane < K && best.at != kNoPlace));
  int place = best.at;
  if (have < K) {
    int filled = 0;
    for (int at = 0; filled < K - have; ++at) {
      const bool taken = __ballot_sync(0xffffffffu, lane < have && place == at) != 0;
      if (taken) continue;
      if (lane == have + filled) place = at;
      ++filled;
    }
  }
  if (lane < K) {
    const size_t o = (size_t)n * K + lane;
    const int k = place / a.V, v = place - k * a.V;
    a.scores_out[o] = (float)best.c;
    a.parents[o] = k;
    a.tokens[o] = v;
    a.finished_out[o] = (a.finished && a.finished[(size_t)n * K + k]) || v == a.eos;
  }
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
// it while it is in the caches.  Rows of 16-byte multiples in 16-byte steps, others in
// single bytes.
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

// Elements per thread of a chunk: 32 where that gives every SM work, else 8, for more
// CTAs on few rows.
int chunk_elements(int N, int K, int V, int sms) {
  const long long big = (V + 32 * kThreads - 1) / (32 * kThreads);
  return (long long)N * K * big >= sms ? 32 : 8;
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
  cudaError_t err = dtype == 0 ? e == 32 ? chunks<float, 32>(lc, a, nchunk) : chunks<float, 8>(lc, a, nchunk)
                    : e == 32  ? chunks<bf16, 32>(lc, a, nchunk)
                               : chunks<bf16, 8>(lc, a, nchunk);
  if (err != cudaSuccess) return err;
  const int warps = std::min(32, std::max(1, a.K * nchunk > 64 ? 32 : std::min(8, a.K * nchunk)));
  return launch_k(beam_merge_kernel, dim3(a.N), dim3(warps * 32), 0, lc.stream, a, nchunk, lc.status);
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
