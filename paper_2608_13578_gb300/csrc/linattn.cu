// Linear attention with a decay per head, on CUDA cores in fp32: the recurrent
// form for float32 tensors and short sequences, the single-token step, and the
// join of segment states that the tensor-core form shares.
#include <algorithm>

#include "common.cuh"
#include "linattn.h"

namespace bcmt {

namespace {

// Valid tokens of sequence b.
__device__ __forceinline__ int valid_tokens(const LinArgs& a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
}

// 16-byte vectors of T as fp32.
template <class T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(const uint4& r, float* v) {
    v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y);
    v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
  }
};
template <>
struct Vec<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(const uint4& r, float* v) { unpack8(r, v); }
};

// V consecutive floats of shared memory (8- or 16-byte aligned).
template <int V>
__device__ __forceinline__ void load_run(const float* p, float* v) {
  if constexpr (V == 4) {
    load4(p, v);
  } else {
    const float2 t = *reinterpret_cast<const float2*>(p);
    v[0] = t.x;
    v[1] = t.y;
  }
}

}  // namespace

// ------------------------------------------------------------- recurrent form
// One CTA walks the tokens of a segment of one head for NW*16 of the state's
// columns.  The state stays in registers: a warp owns 16 columns, lane = (row
// group g = lane % 8, column quad lane / 8), and a lane holds the DK/8 rows
// g*V + 8*V*i + e of its four columns (V rows in a run, so that a warp's q and k
// reads are conflict-free 16-byte broadcasts).  Tokens come in stages of TS
// rows through shared memory, converted to fp32 and zero-padded to DK
// channels; the next stage's rows are loaded into registers under this one's
// arithmetic.  Per token and lane: DK/8 * 4 * (multiply, two fused
// multiply-adds), and the sum over the 8 row groups as a reduce-scatter of the
// four columns (4 shuffles).  Rows are taken in pairs by the packed fp32
// instructions: 1.5 instructions per state element and token.  Bound by those and
// the latency of the sums: 4 x 4096 tokens of 8 heads of width 64 take 154 us (183
// without pairs; their backward 453), 2 x 2048 of width 128 take 142 us (167).
// `local`: states only, from zero, into pass.seg (the first launch of a
// segmented walk).
template <class T, int DK, int NW>
__global__ void __launch_bounds__(NW * 32)
    linattn_simt_kernel(const __grid_constant__ LinArgs a, int local) {
  constexpr int TS = DK == 128 ? 8 : 16;
  constexpr int NT = NW * 32, DVS = NW * 16, R = DK / 8;
  constexpr int V = R < 4 ? R : 4;  // rows in a run (2 or 4)
  constexpr int VN = Vec<T>::N;
  constexpr int QV = TS * (DK / VN), VV = TS * (DVS / VN);  // vectors per stage
  constexpr int QPT = (QV + NT - 1) / NT, VPT = (VV + NT - 1) / NT;
  __shared__ __align__(16) float sq[2][TS][DK], sk[2][TS][DK], sv[2][TS][DVS], so[2][TS][DVS];
  pdl_enter();
  const LinPass& p = a.pass[blockIdx.y];
  const int nslice = (a.dh + DVS - 1) / DVS;
  const int slice = blockIdx.x % nslice, rest = blockIdx.x / nslice;
  const int seg = rest % a.nseg, bh = rest / a.nseg, b = bh / a.H, h = bh - b * a.H;
  // nobody needs the last segment's own contribution
  if (local && seg == (p.rev ? 0 : a.nseg - 1)) return;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane & 7, cq = lane >> 3;
  const int c0 = slice * DVS;              // first column of the CTA
  const int col = warp * 16 + cq * 4;      // the lane's first column, within the CTA's
  const int n = valid_tokens(a, b);
  const int seg_lo = seg * a.seg_len, seg_hi = min(a.T, seg_lo + a.seg_len);
  const int t_lo = min(seg_lo, n), t_hi = min(seg_hi, n);
  const float dec = a.decay[h];
  if (tid == 0) check_decay(dec, a.status);
  const int dh = a.dh;
  const long long tok0 = (long long)b * a.T;
  const T* gq = (const T*)p.q + tok0 * p.ldq + h * dh;
  const T* gk = (const T*)p.k + tok0 * p.ldk + h * dh;
  const T* gv = (const T*)p.v + tok0 * p.ldv + h * dh + c0;
  const long long st = (long long)dh * dh;

  float2 S[R / 2][4];  // pairs of rows, for the packed fp32 arithmetic
#pragma unroll
  for (int r = 0; r < R / 2; ++r)
#pragma unroll
    for (int c = 0; c < 4; ++c) S[r][c] = make_float2(0.f, 0.f);
  auto row_of = [&](int r) { return (r / V) * 8 * V + g * V + (r % V); };
  const bool col_ok = c0 + col < dh;  // dh is a multiple of 8: the quad is whole or absent
  if (!local && col_ok) {
    const float* src = nullptr;
    long si = dh, sj = 1;
    float mul = 1.f;
    if (a.nseg > 1) {
      src = p.seg + ((long long)bh * a.nseg + seg) * st;
    } else if (p.s_in) {
      src = p.s_in + (long long)bh * st;
      mul = n > 0 ? p.s_in_mul : 1.f;  // an empty sequence passes its state on as it is
      if (p.s_in_t) { si = 1; sj = dh; }
    }
    if (src) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int row = row_of(r);
        if (row >= dh) continue;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          (r & 1 ? S[r / 2][c].y : S[r / 2][c].x) = mul * src[row * si + (c0 + col + c) * sj];
      }
    }
  }

  uint4 rq[QPT], rk[QPT], rv[VPT];
  const int cnt_all = t_hi - t_lo;
  const uint4 z4 = make_uint4(0, 0, 0, 0);
  auto token = [&](int i) { return p.rev ? t_hi - 1 - i : t_lo + i; };  // i-th of the walk
  auto load = [&](int s0) {
#pragma unroll
    for (int u = 0; u < QPT; ++u) {
      const int i = tid + u * NT, r = i / (DK / VN), e = (i % (DK / VN)) * VN;
      const bool ok = i < QV && s0 + r < cnt_all && e < dh;
      const long long t = ok ? token(s0 + r) : 0;
      rk[u] = ok ? *reinterpret_cast<const uint4*>(gk + t * p.ldk + e) : z4;
      rq[u] = ok && !local ? *reinterpret_cast<const uint4*>(gq + t * p.ldq + e) : z4;
    }
#pragma unroll
    for (int u = 0; u < VPT; ++u) {
      const int i = tid + u * NT, r = i / (DVS / VN), e = (i % (DVS / VN)) * VN;
      const bool ok = i < VV && s0 + r < cnt_all && c0 + e < dh;
      const long long t = ok ? token(s0 + r) : 0;
      rv[u] = ok ? *reinterpret_cast<const uint4*>(gv + t * p.ldv + e) : z4;
    }
  };
  auto put = [&](float* dst, const uint4& raw) {
    float v[VN];
    Vec<T>::unpack(raw, v);
#pragma unroll
    for (int e = 0; e < VN; e += 4) store4(dst + e, v + e);
  };
  // the finished rows of stage `buf` (its first token number s0) to global memory
  auto flush = [&](int buf, int s0) {
    const int cnt = min(TS, cnt_all - s0);
    for (int i = tid; i < cnt * (DVS / 4); i += NT) {
      const int r = i / (DVS / 4), e = (i % (DVS / 4)) * 4;
      if (c0 + e >= dh) continue;
      float v[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = so[buf][r][e + c] * p.out_mul;
      store4((T*)p.o + (tok0 + token(s0 + r)) * p.ldo + h * dh + c0 + e, v);
    }
  };

  load(0);
  int buf = 0;
  for (int s0 = 0; s0 < cnt_all; s0 += TS, buf ^= 1) {
#pragma unroll
    for (int u = 0; u < QPT; ++u) {
      const int i = tid + u * NT;
      if (i < QV) {
        put(&sk[buf][i / (DK / VN)][(i % (DK / VN)) * VN], rk[u]);
        if (!local) put(&sq[buf][i / (DK / VN)][(i % (DK / VN)) * VN], rq[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < VPT; ++u) {
      const int i = tid + u * NT;
      if (i < VV) put(&sv[buf][i / (DVS / VN)][(i % (DVS / VN)) * VN], rv[u]);
    }
    __syncthreads();
    if (s0 + TS < cnt_all) load(s0 + TS);
    if (!local && s0 > 0) flush(buf ^ 1, s0 - TS);
    const int cnt = min(TS, cnt_all - s0);
#pragma unroll(DK <= 32 ? 2 : 1)  // two tokens' sums overlap: 29.5 -> 22.7 us at 2 x 999, width 32
    for (int i = 0; i < cnt; ++i) {
      // the incoming state of a reverse walk is not decayed by its first token
      const float f = (p.rev && token(s0 + i) == n - 1) ? 1.f : dec;
      const float2 f2 = make_float2(f, f);
      float vv[4];
      load4(&sv[buf][i][col], vv);
      float kk[R], qq[R];
#pragma unroll
      for (int r = 0; r < R; r += V) load_run<V>(&sk[buf][i][row_of(r)], kk + r);
      if (local) {
#pragma unroll
        for (int r = 0; r < R / 2; ++r)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            S[r][c] = __ffma2_rn(make_float2(kk[2 * r], kk[2 * r + 1]), make_float2(vv[c], vv[c]),
                                 __fmul2_rn(f2, S[r][c]));
        continue;
      }
#pragma unroll
      for (int r = 0; r < R; r += V) load_run<V>(&sq[buf][i][row_of(r)], qq + r);
      float2 acc2[4];
#pragma unroll
      for (int r = 0; r < R / 2; ++r) {
        const float2 q2 = make_float2(qq[2 * r], qq[2 * r + 1]);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          S[r][c] = __ffma2_rn(make_float2(kk[2 * r], kk[2 * r + 1]), make_float2(vv[c], vv[c]),
                               __fmul2_rn(f2, S[r][c]));
          acc2[c] = r == 0 ? __fmul2_rn(q2, S[r][c]) : __ffma2_rn(q2, S[r][c], acc2[c]);
        }
      }
      float acc[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] = acc2[c].x + acc2[c].y;
      // reduce-scatter over the 8 row groups: lane bits 0 and 1 pick the column
      const bool hi0 = g & 1, hi1 = g & 2;
      const float s0a = hi0 ? acc[0] : acc[2], s1a = hi0 ? acc[1] : acc[3];
      float k0 = hi0 ? acc[2] : acc[0], k1 = hi0 ? acc[3] : acc[1];
      k0 += __shfl_xor_sync(0xffffffffu, s0a, 1);
      k1 += __shfl_xor_sync(0xffffffffu, s1a, 1);
      const float sb = hi1 ? k0 : k1;
      float m = hi1 ? k1 : k0;
      m += __shfl_xor_sync(0xffffffffu, sb, 2);
      m += __shfl_xor_sync(0xffffffffu, m, 4);
      if (g < 4) so[buf][i][col + (hi0 ? 2 : 0) + (hi1 ? 1 : 0)] = m;
    }
  }
  if (!local && cnt_all > 0) {
    __syncthreads();
    flush(buf ^ 1, ((cnt_all - 1) / TS) * TS);
  }
  if (!local && p.o) {  // the rows past the sequence's end
    const int r0 = max(seg_lo, n), rows = seg_hi - r0;
    const float z[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = tid; i < rows * (DVS / 4); i += NT) {
      const int r = i / (DVS / 4), e = (i % (DVS / 4)) * 4;
      if (c0 + e < dh) store4((T*)p.o + (tok0 + r0 + r) * p.ldo + h * dh + c0 + e, z);
    }
  }
  float* dst = nullptr;
  float mul = 1.f;
  if (local) {
    dst = p.seg + ((long long)bh * a.nseg + seg) * st;
  } else if (p.s_out && seg == (p.rev ? 0 : a.nseg - 1)) {
    dst = p.s_out + (long long)bh * st;
    mul = n > 0 ? p.s_out_mul * (p.rev ? dec : 1.f) : 1.f;
  }
  if (dst && col_ok) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = row_of(r);
      if (row >= dh) continue;
      float v[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = (r & 1 ? S[r / 2][c].y : S[r / 2][c].x) * mul;
      store4(dst + (long long)row * dh + c0 + col, v);
    }
  }
}

// ------------------------------------------------------------ segment states
// Walks the segments of one head in the pass's order, one thread per four
// state elements: on entry seg[s] is segment s's own contribution (from a zero
// state), on return the state coming into segment s.  In place; latency-bound
// (a load, a multiply-add and a store per segment, 16 loads in flight).
__global__ void __launch_bounds__(256) linattn_combine_kernel(const __grid_constant__ LinArgs a) {
  pdl_enter();
  const LinPass& p = a.pass[blockIdx.y];
  const int dh = a.dh, st = dh * dh, parts = (st / 4 + 255) / 256;
  const int bh = blockIdx.x / parts, b = bh / a.H, h = bh - b * a.H;
  const int e0 = ((blockIdx.x - bh * parts) * 256 + threadIdx.x) * 4;
  if (e0 >= st) return;
  const int n = valid_tokens(a, b);
  const float dec = a.decay[h];
  const float full = powf(dec, (float)a.seg_len);
  // the state's row and column: row-major, or groups of 4 columns (a.grouped)
  const int hi = a.grouped ? e0 / 4 / dh : e0 / dh, rest = a.grouped ? e0 / 4 - hi * dh : e0 - hi * dh;
  const int i = a.grouped ? rest : hi, j = a.grouped ? hi * 4 : rest;
  float x[4] = {0.f, 0.f, 0.f, 0.f};
  if (p.s_in) {
    const float* src = p.s_in + (long long)bh * st;
    const float mul = n > 0 ? p.s_in_mul : 1.f;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      x[c] = mul * (p.s_in_t ? src[(long long)(j + c) * dh + i] : src[i * dh + j + c]);
  }
  float* w = p.seg + (long long)bh * a.nseg * st + e0;
  const bool out = a.grouped && p.s_out;
  constexpr int kBatch = 16;  // loads in flight: each is a memory latency
  for (int s0 = 0; s0 < a.nseg; s0 += kBatch) {
    float loc[kBatch][4];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int s = p.rev ? a.nseg - 1 - (s0 + u) : s0 + u;
      if (s0 + u < a.nseg - (out ? 0 : 1)) load4(w + (long long)s * st, loc[u]);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (s0 + u >= a.nseg) break;
      const int s = p.rev ? a.nseg - 1 - (s0 + u) : s0 + u;
      store4(w + (long long)s * st, x);
      if (s0 + u == a.nseg - 1 && !out) break;
      const int lo = s * a.seg_len;
      const int m = min(max(n - lo, 0), a.seg_len);  // valid tokens of the segment
      if (m == 0) continue;
      const bool fresh = p.rev && n <= lo + a.seg_len;  // holds the last valid token
      const float f = (m == a.seg_len && !fresh) ? full : powf(dec, (float)(m - (fresh ? 1 : 0)));
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] = fmaf(f, x[c], loc[u][c]);
    }
  }
  if (out) {
    const float mul = n > 0 ? p.s_out_mul * (p.rev ? dec : 1.f) : 1.f;
#pragma unroll
    for (int c = 0; c < 4; ++c) x[c] *= mul;
    store4(p.s_out + (long long)bh * st + i * dh + j, x);
  }
}

// ----------------------------------------------------------------- one token
// S' = a S + k v^T, o = out_mul * S'^T q for one token: a CTA takes 32 columns
// of one head's state as 8 column quads x 32 row groups; a thread's rows (up to
// four) are loaded together, so the state streams through once at full
// sectors.  Bandwidth-bound: 8 dh^2 bytes per head.  256 sequences of 8 heads of
// width 128, a tenth of them idle: 44 us, 6.1 TB/s; one sequence of 8 heads of 64:
// 1.7 us, a launch.
template <class T>
__global__ void __launch_bounds__(256) linattn_step_kernel(const __grid_constant__ LinArgs a) {
  __shared__ float red[8][33];
  pdl_enter();
  const LinPass& p = a.pass[0];
  const int dh = a.dh, parts = (dh + 31) / 32;
  const int bh = blockIdx.x / parts, b = bh / a.H, h = bh - b * a.H;
  const int c0 = (blockIdx.x - bh * parts) * 32;
  const int tid = threadIdx.x, quad = tid & 7, rg = tid >> 3, warp = tid >> 5;
  const int col = c0 + quad * 4;
  const bool on = valid_tokens(a, b) > 0;
  const bool col_ok = col < dh;
  if (tid == 0) check_decay(a.decay[h], a.status);
  const float dec = on ? a.decay[h] : 1.f;
  const T* q = (const T*)p.q + (long long)b * p.ldq + h * dh;
  const T* k = (const T*)p.k + (long long)b * p.ldk + h * dh;
  const T* v = (const T*)p.v + (long long)b * p.ldv + h * dh;
  const long long s0 = (long long)bh * dh * dh + col;
  float S[4][4], kk[4], qq[4], vv[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = rg + 32 * i;
    const bool ok = row < dh && col_ok;
#pragma unroll
    for (int c = 0; c < 4; ++c) S[i][c] = 0.f;
    if (ok && p.s_in) load4(p.s_in + s0 + (long long)row * dh, S[i]);
    kk[i] = on && ok ? to_f(k[row]) : 0.f;
    qq[i] = on && ok ? to_f(q[row]) : 0.f;
  }
  if (on && col_ok) load4(v + col, vv);
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = rg + 32 * i;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      if (on) S[i][c] = fmaf(kk[i], vv[c], dec * S[i][c]);
      acc[c] = fmaf(qq[i], S[i][c], acc[c]);
    }
    if (row < dh && col_ok && p.s_out) store4(p.s_out + s0 + (long long)row * dh, S[i]);
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    acc[c] += __shfl_xor_sync(0xffffffffu, acc[c], 8);
    acc[c] += __shfl_xor_sync(0xffffffffu, acc[c], 16);
  }
  if ((tid & 31) < 8) {
#pragma unroll
    for (int c = 0; c < 4; ++c) red[warp][quad * 4 + c] = acc[c];
  }
  __syncthreads();
  if (tid < 32 && c0 + tid < dh) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += red[w][tid];
    ((T*)p.o)[(long long)b * p.ldo + h * dh + c0 + tid] =
        from_f<T>(on ? s * p.out_mul : 0.f);
  }
}

// ---------------------------------------------------------------- host side
namespace {
template <class T, int DK, int NW>
cudaError_t simt_launch(const Launch& lc, const LinArgs& a) {
  const int nslice = (a.dh + NW * 16 - 1) / (NW * 16);
  const dim3 grid(nslice * a.nseg * a.B * a.H, a.npass);
  cudaError_t e;
  if (a.nseg > 1) {
    e = launch_k(linattn_simt_kernel<T, DK, NW>, grid, dim3(NW * 32), 0, lc.stream, a, 1);
    if (e != cudaSuccess) return e;
    if ((e = linattn_combine(lc, a)) != cudaSuccess) return e;
  }
  e = launch_k(linattn_simt_kernel<T, DK, NW>, grid, dim3(NW * 32), 0, lc.stream, a, 0);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <class T>
cudaError_t simt_typed(const Launch& lc, const LinArgs& a) {
  if (a.dh <= 16) return simt_launch<T, 16, 1>(lc, a);
  if (a.dh <= 32) return simt_launch<T, 32, 2>(lc, a);
  if (a.dh <= 64) return simt_launch<T, 64, 4>(lc, a);
  return simt_launch<T, 128, 4>(lc, a);
}
}  // namespace

LinPlan linattn_plan(int dtype, int B, int T, int H, int dh, int npass, int sms, bool allow_tc,
                     bool ragged) {
  const long long heads = (long long)B * H * npass;
  LinPlan pl{allow_tc && dtype == 1 && T >= 32, 1, T};
  if (pl.tc) {
    // segments of whole chunks, enough for one CTA in every slot (two per SM up
    // to width 64): the walk is sequential, and a slot left empty is lost.  8 x 1024
    // tokens of 8 heads of 64 take 23 us so, 30 in one segment or in twice as many, 32
    // in two; where a call has one head a slot or so, one segment needs no states
    // (backward of 4 x 4095, 8 heads of 128: 109 us, 147 in two)
    const long long slots = (long long)sms * (dh <= 64 ? 2 : 1);
    const int chunks = (T + 127) / 128;
    long long n = std::max(1ll, std::min<long long>(slots / heads, chunks));
    // sequences of different lengths: three times as many, of four chunks at least, so
    // that slots whose segment is empty or short take another (4 sequences of up to
    // 16384 tokens, 8 heads of 128: 159 us for 182; were all of them full, 214 for 188)
    if (ragged && n > 1) n = std::max(n, std::min<long long>(3 * n, chunks / 4));
    const int per = (int)((chunks + n - 1) / n);
    pl.nseg = (chunks + per - 1) / per;
    pl.seg_len = per * 128;
    return pl;
  }
  // CTAs for eight on each SM, by segments of at least 24 tokens: the walk is
  // sequential, and one segment's latency is the pass's.  Eight fit up to width 32; by
  // their registers (fp32) 5 of width 64 do and 3 of width 128, so that there the CTAs
  // come in 1.6 and 2.7 waves.  Two CTAs an SM and 64
  // tokens took 277 us for 183 at 4 x 4096 of width 64, 39 for 31 at 1 x 200 of 4
  // heads of width 128; segments of 32 and of 24 tokens differ by 2 to 4 us in small calls
  const long long ctas = heads * (dh > 64 ? 2 : 1);
  const long long want = (8ll * sms + ctas - 1) / ctas;
  const long long most = std::max(1, T / 24);
  const long long n = std::max(1ll, std::min(want, most));
  if (n > 1) {
    pl.seg_len = (int)((T + n - 1) / n);
    pl.nseg = (T + pl.seg_len - 1) / pl.seg_len;
  }
  return pl;
}

cudaError_t linattn_simt(const Launch& lc, int dtype, const LinArgs& a) {
  return dtype == 0 ? simt_typed<float>(lc, a) : simt_typed<bf16>(lc, a);
}

cudaError_t linattn_combine(const Launch& lc, const LinArgs& a) {
  const dim3 grid((a.dh * a.dh / 4 + 255) / 256 * a.B * a.H, a.npass);
  cudaError_t e = launch_k(linattn_combine_kernel, grid, dim3(256), 0, lc.stream, a);
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t linattn_step(const Launch& lc, int dtype, const LinArgs& a) {
  const dim3 grid((a.dh + 31) / 32 * a.B * a.H);
  cudaError_t e = dtype == 0
                      ? launch_k(linattn_step_kernel<float>, grid, dim3(256), 0, lc.stream, a)
                      : launch_k(linattn_step_kernel<bf16>, grid, dim3(256), 0, lc.stream, a);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace bcmt
