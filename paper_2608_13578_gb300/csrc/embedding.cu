// Scaled embedding lookup out_i = s W[id_i], and its gradient by sorted tokens
// dW[v] = s sum_{i: id_i = v} dy_i, summed in fp32 in an order that the ids alone decide
// (position order in runs of up to 32, then the runs; no floating-point atomics: the
// result does not change from run to run) and rounded once.
#include <algorithm>

#include "common.cuh"
#include "internal.h"

namespace bcmt {

namespace {

constexpr int kSortThreads = 256;
// ids sorted by one CTA of a radix pass: a CTA's scattered stores take a cycle
// each, so small batches are cut finer; large ones are not, for their counts' sake
inline int sort_tile(long long N) { return N <= (1 << 17) ? 1024 : 4096; }
// More tiles than this, and the counts are scanned by a kernel before each pass
// (embed_scan_kernel); up to it, every CTA of a pass adds up every tile's counts, which
// saves the launch and grows with the tiles' square.  Into a table of 40000 x 8, us
// scanned and not: 16384 ids 27 and 25, 49152 28 and 28, 65536 30 and 35, 262144 53 and
// 65, 16777216 1538 and 9988.
constexpr int kScanTiles = 48;
constexpr int kChunk = 32;       // sorted positions summed by one warp

// The id at i, or -1 where it is outside [0, V).
__device__ __forceinline__ int id_at(const void* ids, int is64, long long i, int V) {
  const long long v = is64 ? static_cast<const long long*>(ids)[i] : static_cast<const int*>(ids)[i];
  return v >= 0 && v < V ? (int)v : -1;
}

// 16 bytes of T as fp32 and back.
template <class T>
constexpr int vec_n() { return 16 / (int)sizeof(T); }
template <class T>
__device__ __forceinline__ void unpack16(const uint4& r, float* v) {
  if constexpr (sizeof(T) == 2) {
    unpack8(r, v);
  } else {
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y);
    v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
  }
}
template <class T>
__device__ __forceinline__ void store16(T* p, const float* v) {
  if constexpr (sizeof(T) == 2) store8(p, v);
  else store4(p, v);
}

}  // namespace

// ---------------------------------------------------------------------- lookup
// One thread per 16 bytes of output, four in flight.  Bandwidth-bound: the
// output is written once and a row is read once from HBM (repeated tokens hit
// L2).  An id outside [0, V) gives a zero row and sets kStatusBadIndex.  8192 rows of
// 512 bf16 from a table of 32000: 4.4 us, the launch and two dependent reads (the id,
// then its row) above the 1.8 us that the bytes take.
template <class T>
__global__ void __launch_bounds__(256)
    embed_fwd_kernel(const void* __restrict__ ids, int is64, long long N, int V, int D,
                     const T* __restrict__ W, float scale, T* __restrict__ out, unsigned* status) {
  pdl_enter();
  constexpr int VN = vec_n<T>();
  const int rv = D / VN;
  const long long total = N * rv, stride = (long long)gridDim.x * 256;
  for (long long i0 = blockIdx.x * 256ll + threadIdx.x; i0 < total; i0 += 4 * stride) {
    uint4 raw[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = i0 + u * stride;
      raw[u] = make_uint4(0, 0, 0, 0);
      if (i < total) {
        const long long r = i / rv;
        const int c = (int)(i - r * rv);
        const int id = id_at(ids, is64, r, V);
        if (id >= 0) raw[u] = *reinterpret_cast<const uint4*>(W + (long long)id * D + c * VN);
        else if (c == 0) atomicOr(status, kStatusBadIndex);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = i0 + u * stride;
      if (i >= total) continue;
      float v[VN];
      unpack16<T>(raw[u], v);
#pragma unroll
      for (int e = 0; e < VN; ++e) v[e] *= scale;
      store16<T>(out + i * VN, v);
    }
  }
}

// ------------------------------------------------------------------- gradient
// A stable least-significant-digit radix sort of the ids (8 bits a pass, ids
// outside [0, V) as key V, at the end), then a segmented sum over the sorted
// positions.  The sort's launches occupy few SMs, so the CTAs beyond its tiles
// clear the table's gradient meanwhile (rows that no token names stay zero).
// 65536 tokens of width 768 over 32000 rows: 55 us (fp32 81), where the bytes alone take 22
// (44): the sum 24 (4.4 TB/s of rows), the rest the keys, two scans and passes and the
// join of runs across chunks, each a chain of latencies over few keys an SM.  Atomics into fp32 would need no
// sort, but their order, and with it the result, would change from run to run.
struct SortArgs {
  const void* ids;
  int is64;
  int N, V, tiles;
  int* key;      // [N] the ids
  int2* pair[2]; // [N] (key, position), sorted by the digits so far
  int* cnt[3];   // [tiles][256] per pass
  int* total;    // [256], of the pass whose counts have been scanned; null: none are
  int passes;
  uint4* zero;   // the gradient, cleared by parts over the sort's launches
  long long zero_n;
  unsigned* status;
};

namespace {
// CTAs from `first` on clear the part `part` of `parts`, eight stores a thread.
__device__ __forceinline__ void clear_part(const SortArgs& a, int first, int part, int parts) {
  const long long lo = a.zero_n * part / parts, hi = a.zero_n * (part + 1) / parts;
  const uint4 z = make_uint4(0, 0, 0, 0);
  const long long step = 8ll * kSortThreads;
  for (long long i0 = lo + (blockIdx.x - first) * step + threadIdx.x; i0 < hi;
       i0 += (gridDim.x - first) * step) {
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i0 + u * kSortThreads < hi) a.zero[i0 + u * kSortThreads] = z;
  }
}
}  // namespace

// Keys and digit counts of the first pass.
template <int PER>
__global__ void __launch_bounds__(kSortThreads) embed_keys_kernel(const __grid_constant__ SortArgs a) {
  constexpr int kTile = PER * kSortThreads;
  __shared__ int hist[256];
  pdl_enter();
  if ((int)blockIdx.x >= a.tiles) {
    clear_part(a, a.tiles, 0, a.passes + 1);
    return;
  }
  const int tid = threadIdx.x;
  hist[tid] = 0;
  __syncthreads();
  const int base = blockIdx.x * kTile;
  int id[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = base + j * kSortThreads + tid;
    id[j] = i < a.N ? id_at(a.ids, a.is64, i, a.V) : 0;
  }
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = base + j * kSortThreads + tid;
    if (i >= a.N) continue;
    if (id[j] < 0) {
      id[j] = a.V;
      atomicOr(a.status, kStatusBadIndex);
    }
    a.key[i] = id[j];
    atomicAdd(&hist[id[j] & 255], 1);
  }
  __syncthreads();
  a.cnt[0][blockIdx.x * 256 + tid] = hist[tid];
  for (int p = 1; p < a.passes; ++p) a.cnt[p][blockIdx.x * 256 + tid] = 0;
}

namespace {
// The lanes of `among` whose 8-bit digit is this lane's, by a ballot per bit (a
// match instruction takes a step per distinct value, hundreds of cycles here).
__device__ __forceinline__ unsigned equal_lanes(int d, unsigned among) {
  unsigned m = among;
#pragma unroll
  for (int b = 0; b < 8; ++b) {
    const unsigned v = __ballot_sync(0xffffffffu, (d >> b) & 1);
    m &= ((d >> b) & 1) ? v : ~v;
  }
  return m;
}
}  // namespace

// Before pass p, for many tiles: each tile's counts become, digit by digit, the keys
// with that digit in the tiles before it, and total[] the keys of all tiles.  In
// place; a CTA takes 8 digits (a sector of every tile's counts), a thread one digit of
// a run of consecutive tiles, twice: its sum, then the sums up to each tile.  Without
// it a pass reads tiles^2 KB: a second and more at the most ids a call takes.
constexpr int kScanThreads = 1024, kScanDigits = 8;
__global__ void __launch_bounds__(kScanThreads)
    embed_scan_kernel(const __grid_constant__ SortArgs a, int p) {
  constexpr int kRuns = kScanThreads / kScanDigits;
  __shared__ int sums[kRuns][kScanDigits];
  pdl_enter();
  const int d = threadIdx.x % kScanDigits, run = threadIdx.x / kScanDigits;
  const int digit = blockIdx.x * kScanDigits + d, per = (a.tiles + kRuns - 1) / kRuns;
  const int lo = min(run * per, a.tiles), hi = min(lo + per, a.tiles);
  int* c = a.cnt[p] + digit;
  int sum = 0;
#pragma unroll 8
  for (int t = lo; t < hi; ++t) sum += c[(long long)t * 256];
  sums[run][d] = sum;
  __syncthreads();
  if (run == 0) {
    int before = 0;
    for (int r = 0; r < kRuns; ++r) {
      const int x = sums[r][d];
      sums[r][d] = before;
      before += x;
    }
    a.total[digit] = before;
  }
  __syncthreads();
  int before = sums[run][d];
  for (int t0 = lo; t0 < hi; t0 += 8) {  // eight loads in flight
    int x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = t0 + u < hi ? c[(long long)(t0 + u) * 256] : 0;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (t0 + u < hi) c[(long long)(t0 + u) * 256] = before;
      before += x[u];
    }
  }
}

// One stable pass: digit `p` of the keys.  Ranks: each warp takes 256
// consecutive keys, 32 at a time, and ranks equal digits by lane order; the
// warps' counts are then scanned in warp order and the tiles' in tile order.
// The next pass's digit counts (integers: order does not matter) are taken on
// the way, at the tiles where the keys land.
template <int PER>
__global__ void __launch_bounds__(kSortThreads)
    embed_sort_kernel(const __grid_constant__ SortArgs a, int p) {
  constexpr int NW = kSortThreads / 32, kTile = PER * kSortThreads;
  __shared__ int wcnt[NW][256];
  __shared__ int wsum[NW];
  pdl_enter();
  if ((int)blockIdx.x >= a.tiles) {
    clear_part(a, a.tiles, p + 1, a.passes + 1);
    return;
  }
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int base = blockIdx.x * kTile;
  const int2* in = a.pair[(p + 1) & 1];
#pragma unroll
  for (int w = 0; w < NW; ++w) wcnt[w][tid] = 0;
  __syncthreads();
  int key[PER], pos[PER], rank[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = base + warp * (PER * 32) + j * 32 + lane;
    const int2 x = i >= a.N ? make_int2(-1, 0) : p == 0 ? make_int2(a.key[i], i) : in[i];
    key[j] = x.x;
    pos[j] = x.y;
  }
  unsigned same[PER];  // the warp's lanes with an equal digit
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int d = (key[j] >> (8 * p)) & 255;
    same[j] = equal_lanes(d, __ballot_sync(0xffffffffu, key[j] >= 0));
    const unsigned before = same[j] & ((1u << lane) - 1u);
    const int start = wcnt[warp][d];
    __syncwarp();
    if (key[j] >= 0 && before == 0) wcnt[warp][d] = start + __popc(same[j]);
    __syncwarp();
    rank[j] = start + __popc(before);
  }
  // digit tid: keys before this tile's, over all digits and the earlier tiles
  int total = 0, mine = 0;
  if (a.total) {
    total = a.total[tid];
    mine = a.cnt[p][(long long)blockIdx.x * 256 + tid];
  } else {
    for (int t0 = 0; t0 < a.tiles; t0 += 32) {  // 32 loads in flight
      int c[32];
#pragma unroll
      for (int u = 0; u < 32; ++u) c[u] = t0 + u < a.tiles ? a.cnt[p][(t0 + u) * 256 + tid] : 0;
#pragma unroll
      for (int u = 0; u < 32; ++u) {
        total += c[u];
        if (t0 + u < (int)blockIdx.x) mine += c[u];
      }
    }
  }
  int incl = total;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 31) wsum[warp] = incl;
  __syncthreads();
  int off = incl - total + mine;
  for (int w = 0; w < warp; ++w) off += wsum[w];
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    const int c = wcnt[w][tid];
    wcnt[w][tid] = off;
    off += c;
  }
  __syncthreads();
  int2* out = a.pair[p & 1];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (key[j] < 0) continue;
    const int dst = wcnt[warp][(key[j] >> (8 * p)) & 255] + rank[j];
    out[dst] = make_int2(key[j], pos[j]);
    rank[j] = dst / kTile;
  }
  if (p + 1 < a.passes) {
    // one addition for the warp's keys with equal digits that land in one tile: a
    // frequent token's keys would all add to one counter
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      const int d = (key[j] >> (8 * (p + 1))) & 255;
      const unsigned eq = equal_lanes(d, same[j]);
      const int first = __ffs(eq) - 1;
      const int t = __shfl_sync(0xffffffffu, rank[j], first < 0 ? 0 : first);
      const bool lead = key[j] >= 0 && lane == first;
      const unsigned near = eq & __ballot_sync(0xffffffffu, key[j] >= 0 && rank[j] == t);
      if (lead) atomicAdd(&a.cnt[p + 1][t * 256 + d], __popc(near));
      else if (key[j] >= 0 && rank[j] != t) atomicAdd(&a.cnt[p + 1][rank[j] * 256 + d], 1);
    }
  }
}

// The segmented sum: a warp takes kChunk sorted positions and 32 vectors of
// columns, adding the rows of equal keys in order.  A run inside the chunk is
// finished here; what a run has in a chunk that it shares with a neighbour goes
// to part[chunk][0] (the chunk's first run, when it began earlier) or
// part[chunk][1] (its last run, when it goes on).
struct SumArgs {
  const int2* pair;  // (key, position), sorted
  int N, V, D, chunks, cblocks;
  float scale;
  float* part;  // [chunks][2][D]
};

// Four rows in flight a warp and 48 registers a thread, so that 40 warps share an
// SM (80 KB in flight): the additions of a warp are a chain, which only other warps
// can fill (eight rows and half the warps: 4 us slower at 65536 x 768; rows
// streamed through shared memory by 12 warps: 8 us slower).
template <class T>
__global__ void __launch_bounds__(256, 5)
    embed_sum_kernel(const __grid_constant__ SumArgs a, const T* __restrict__ dy,
                     T* __restrict__ dw) {
  constexpr int VN = vec_n<T>();
  constexpr int U = 4;  // rows in flight
  pdl_enter();
  const int lane = threadIdx.x & 31;
  const int unit = blockIdx.x * 8 + (threadIdx.x >> 5);
  if (unit >= a.chunks * a.cblocks) return;
  const int chunk = unit / a.cblocks, col = ((unit - chunk * a.cblocks) * 32 + lane) * VN;
  const int p0 = chunk * kChunk, cnt = min(kChunk, a.N - p0);
  const int2 my = lane < cnt ? a.pair[p0 + lane] : make_int2(-1, 0);
  const int prev = p0 > 0 ? a.pair[p0 - 1].x : -1;
  const int next = p0 + cnt < a.N ? a.pair[p0 + cnt].x : -1;
  const bool ok = col < a.D;
  // keys past V are ids outside the table, sorted to the end
  const int used = __popc(__ballot_sync(0xffffffffu, lane < cnt && my.x < a.V));
  // where a run of equal keys ends in the chunk (the last position always does)
  const int nxt = __shfl_down_sync(0xffffffffu, my.x, 1);
  const unsigned ends = __ballot_sync(0xffffffffu, lane == cnt - 1 || nxt != my.x);
  bool from_prev = __shfl_sync(0xffffffffu, my.x, 0) == prev;
  float acc[VN];
#pragma unroll
  for (int e = 0; e < VN; ++e) acc[e] = 0.f;
#pragma unroll 1
  for (int j0 = 0; j0 < used; j0 += U) {
    uint4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long long row = __shfl_sync(0xffffffffu, my.y, j0 + u);
      raw[u] = make_uint4(0, 0, 0, 0);
      if (j0 + u < used && ok) raw[u] = *reinterpret_cast<const uint4*>(dy + row * a.D + col);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u;
      float v[VN];
      unpack16<T>(raw[u], v);
#pragma unroll
      for (int e = 0; e < VN; ++e) acc[e] += v[e];
      if (j >= used || !((ends >> j) & 1u)) continue;
      const int key = __shfl_sync(0xffffffffu, my.x, j);
      const bool goes_on = j == cnt - 1 && next == key;
      if (ok) {
        if (from_prev || goes_on) {
          float* d = a.part + ((long long)chunk * 2 + (from_prev ? 0 : 1)) * a.D + col;
#pragma unroll
          for (int e = 0; e < VN; e += 4) store4(d + e, acc + e);
        } else {
#pragma unroll
          for (int e = 0; e < VN; ++e) acc[e] *= a.scale;
          store16<T>(dw + (long long)key * a.D + col, acc);
        }
      }
#pragma unroll
      for (int e = 0; e < VN; ++e) acc[e] = 0.f;
      from_prev = false;
    }
  }
}

// Joins the runs that cross chunks, in chunk order: the chunk in which such a
// run begins owns it, and its warp adds part[chunk][1], part[chunk + 1][0], ...
// A run of more than kLong chunks is cut among the CTA's warps and their sums
// added in warp order.
constexpr int kLong = 16;
template <class T>
__global__ void __launch_bounds__(256)
    embed_join_kernel(const __grid_constant__ SumArgs a, T* __restrict__ dw) {
  constexpr int VN = vec_n<T>();
  __shared__ int run_len[8], run_key[8];
  __shared__ float sums[8][32 * 8 + 4];
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int chunk0 = blockIdx.x / a.cblocks * 8, cb = blockIdx.x % a.cblocks;
  const int col = (cb * 32 + lane) * VN;
  const bool ok = col < a.D;
  auto add = [&](int lo, int hi, int chunk, float* acc) {  // parts lo .. hi-1 of the run
    for (int m0 = lo; m0 < hi; m0 += 4) {  // four loads in flight
      float v[4][VN];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int m = m0 + u;
#pragma unroll
        for (int e = 0; e < VN; ++e) v[u][e] = 0.f;
        if (m < hi && ok) {
          const float* s = a.part + ((long long)(chunk + m) * 2 + (m == 0 ? 1 : 0)) * a.D + col;
#pragma unroll
          for (int e = 0; e < VN; e += 4) load4(s + e, v[u] + e);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < VN; ++e) acc[e] += v[u][e];
    }
  };
  auto finish = [&](int key, float* acc) {
#pragma unroll
    for (int e = 0; e < VN; ++e) acc[e] *= a.scale;
    store16<T>(dw + (long long)key * a.D + col, acc);
  };
  {
    const int chunk = chunk0 + warp;
    int len = 0, key = -1;
    const int end = (chunk + 1) * kChunk;  // first position of the next chunk
    if (chunk < a.chunks && end < a.N) {
      key = a.pair[end - 1].x;
      const int first = a.pair[chunk * kChunk].x, after = a.pair[end].x;
      const int before = chunk > 0 ? a.pair[chunk * kChunk - 1].x : -1;
      if (key < a.V && after == key && (first != key || before != key)) {
        // the last chunk that begins with key: 32 probes at a time, at strides of
        // 1, 32, 1024, ... chunks until one misses, then back down
        int lo = chunk + 1, stride = 1, hits = 32;
        auto probe = [&]() {
          const long long c = lo + (lane + 1ll) * stride;
          hits = __popc(__ballot_sync(0xffffffffu, c < a.chunks && a.pair[c * kChunk].x == key));
          lo += hits * stride;
        };
        for (probe(); hits == 32; probe()) stride *= 32;
        while (stride > 1) {
          stride /= 32;
          probe();
        }
        len = lo - chunk + 1;
      }
    }
    if (lane == 0) {
      run_len[warp] = len;
      run_key[warp] = key;
    }
    if (len > 0 && len <= kLong) {
      float acc[VN];
#pragma unroll
      for (int e = 0; e < VN; ++e) acc[e] = 0.f;
      add(0, len, chunk, acc);
      if (ok) finish(key, acc);
    }
  }
  __syncthreads();
  for (int w = 0; w < 8; ++w) {
    const int len = run_len[w];
    if (len <= kLong) continue;
    float acc[VN];
#pragma unroll
    for (int e = 0; e < VN; ++e) acc[e] = 0.f;
    const int per = (len + 7) / 8, lo = warp * per;
    add(min(lo, len), min(lo + per, len), chunk0 + w, acc);
#pragma unroll
    for (int e = 0; e < VN; ++e) sums[warp][lane * VN + e] = acc[e];
    __syncthreads();
    if (warp == 0 && ok) {
#pragma unroll
      for (int e = 0; e < VN; ++e) acc[e] = sums[0][lane * VN + e];
      for (int q = 1; q < 8; ++q)
#pragma unroll
        for (int e = 0; e < VN; ++e) acc[e] += sums[q][lane * VN + e];
      finish(run_key[w], acc);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- host side
namespace {
struct BwdLayout {
  size_t key, pair[2], cnt[3], total, part, bytes;
  int tiles, passes, chunks;
  bool scan;
};
BwdLayout bwd_layout(long long N, int V, int D) {
  BwdLayout l{};
  l.tiles = (int)((N + sort_tile(N) - 1) / sort_tile(N));
  l.chunks = (int)((N + kChunk - 1) / kChunk);
  l.passes = V < (1 << 8) ? 1 : V < (1 << 16) ? 2 : 3;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t r = off;
    off += (bytes + 255) & ~size_t(255);
    return r;
  };
  l.key = take((size_t)N * 4);
  for (int i = 0; i < 2; ++i) l.pair[i] = take((size_t)N * 8);
  for (int i = 0; i < l.passes; ++i) l.cnt[i] = take((size_t)l.tiles * 256 * 4);
  l.scan = l.tiles > kScanTiles;
  if (l.scan) l.total = take(256 * 4);
  l.part = take((size_t)l.chunks * 2 * D * 4);
  l.bytes = off;
  return l;
}

template <class T>
cudaError_t fwd_typed(const Launch& lc, const EmbedArgs& a, const void* W, void* out) {
  const long long vecs = a.N * (a.D / vec_n<T>());
  const long long blocks = std::min<long long>((vecs + 1023) / 1024, 152ll * 64);
  cudaError_t e = launch_k(embed_fwd_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, lc.stream,
                           a.ids, a.is64, a.N, a.V, a.D, (const T*)W, a.scale, (T*)out, lc.status);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <class T>
cudaError_t bwd_typed(const Launch& lc, const EmbedArgs& a, const void* dy, void* dw, void* ws) {
  const BwdLayout l = bwd_layout(a.N, a.V, a.D);
  char* w = static_cast<char*>(ws);
  SortArgs s{};
  s.ids = a.ids;
  s.is64 = a.is64;
  s.N = (int)a.N;
  s.V = a.V;
  s.tiles = l.tiles;
  s.passes = a.N > 0 ? l.passes : 0;  // an empty batch only clears
  s.key = reinterpret_cast<int*>(w + l.key);
  for (int i = 0; i < 2; ++i) s.pair[i] = reinterpret_cast<int2*>(w + l.pair[i]);
  for (int i = 0; i < l.passes; ++i) s.cnt[i] = reinterpret_cast<int*>(w + l.cnt[i]);
  s.total = l.scan ? reinterpret_cast<int*>(w + l.total) : nullptr;
  s.zero = static_cast<uint4*>(dw);
  s.zero_n = (long long)a.V * (a.D / vec_n<T>());
  s.status = lc.status;
  const unsigned clear = (unsigned)std::min<long long>((s.zero_n + 2047) / 2048, 152 * 4);
  const dim3 grid(l.tiles + clear);
  const bool fine = sort_tile(a.N) == 1024;
  cudaError_t e = fine ? launch_k(embed_keys_kernel<4>, grid, dim3(kSortThreads), 0, lc.stream, s)
                       : launch_k(embed_keys_kernel<16>, grid, dim3(kSortThreads), 0, lc.stream, s);
  if (e != cudaSuccess) return e;
  if (a.N == 0) return cudaGetLastError();
  for (int p = 0; p < l.passes; ++p) {
    if (l.scan) {
      e = launch_k(embed_scan_kernel, dim3(256 / kScanDigits), dim3(kScanThreads), 0, lc.stream, s, p);
      if (e != cudaSuccess) return e;
    }
    e = fine ? launch_k(embed_sort_kernel<4>, grid, dim3(kSortThreads), 0, lc.stream, s, p)
             : launch_k(embed_sort_kernel<16>, grid, dim3(kSortThreads), 0, lc.stream, s, p);
    if (e != cudaSuccess) return e;
  }
  SumArgs m{};
  m.pair = s.pair[(l.passes - 1) & 1];
  m.N = (int)a.N;
  m.V = a.V;
  m.D = a.D;
  m.chunks = l.chunks;
  m.cblocks = (a.D / vec_n<T>() + 31) / 32;
  m.scale = a.scale;
  m.part = reinterpret_cast<float*>(w + l.part);
  const long long units = (long long)m.chunks * m.cblocks;
  e = launch_k(embed_sum_kernel<T>, dim3((unsigned)((units + 7) / 8)), dim3(256), 0, lc.stream, m,
               (const T*)dy, (T*)dw);
  if (e != cudaSuccess) return e;
  if (m.chunks > 1)
    e = launch_k(embed_join_kernel<T>, dim3((unsigned)((m.chunks + 7) / 8 * m.cblocks)), dim3(256),
                 0, lc.stream, m, (T*)dw);
  return e != cudaSuccess ? e : cudaGetLastError();
}
}  // namespace

size_t embed_bwd_workspace(long long N, int V, int D) { return bwd_layout(N, V, D).bytes; }

cudaError_t embed_fwd(const Launch& lc, int dtype, const EmbedArgs& a, const void* W, void* out) {
  if (a.N == 0) return cudaSuccess;
  return dtype == 0 ? fwd_typed<float>(lc, a, W, out) : fwd_typed<bf16>(lc, a, W, out);
}

cudaError_t embed_bwd(const Launch& lc, int dtype, const EmbedArgs& a, const void* dy, void* dw,
                      void* ws) {
  return dtype == 0 ? bwd_typed<float>(lc, a, dy, dw, ws) : bwd_typed<bf16>(lc, a, dy, dw, ws);
}

}  // namespace bcmt
