// One AdamW step (Loshchilov and Hutter, "Decoupled weight decay regularization", 2019)
// over many tensors in one launch:
//   m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps),
// g times *grad_scale where there is one, p taken from and also written to a float32
// master where there is one.  The states are float32, or 8-bit codes with one float32
// scale for every 256 consecutive elements of a tensor:
//   m = c |c| s,  c in -127 .. 127,  s = max |m| / 127^2;   c = #{k >= 1: (k - 1/2)^2 <= |m| / s}
//   sqrt(v) = c^2 r,  c in 0 .. 255,  r = sqrt(max v) / 255^2;  c = #{k >= 1: (k - 1/2)^4 <= v / r^2},
// at least 1 where v > 0.  (The square, and the square of the root, spend the codes on
// small values: the smallest step of m is 1/16129 of its block's largest, that of v
// 1/4.2e9, so that a small v is not taken for 0 and its step not blown up.)
// What decides a code is rounded operation by operation, with no fused multiply-add:
// the codes are a function of the inputs that any IEEE machine gives.
#include <math.h>

#include <algorithm>

#include "adamw.h"
#include "common.cuh"
#include "internal.h"
#include "norm_rows.cuh"

namespace bcmt {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;   // elements of a CTA; with 8-bit states, where a launch has many,
                               // twice that, which spreads what a CTA begins with over more
constexpr int kBlock = 256;    // elements that share a scale

struct Rates {
  float rate, keep, ib2;   // lr / (1 - b1^t), 1 - lr wd, 1 / sqrt(1 - b2^t)
};
__device__ __forceinline__ Rates rates(const AdamwHyper& h) {
  Rates r{h.rate, h.keep, h.ib2};
  if (h.step_ptr || h.lr_ptr) {
    const float lr = h.lr_ptr ? *h.lr_ptr : h.lr;
    const double t = (double)(h.step_ptr ? *h.step_ptr : h.step);
    // 1 - b^t = -expm1(t ln b), good for b near 1 and every t
    r.rate = lr / -expm1f((float)(t * h.log_b1));
    r.ib2 = 1.f / sqrtf(-expm1f((float)(t * h.log_b2)));
    r.keep = 1.f - lr * h.decay;
  }
  return r;
}

__device__ __forceinline__ float root(float x) {
  float y;
  asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The moments, each operation rounded, and the weight (its update to a few units in the
// last place: it is lr times smaller than what it is added to).
__device__ __forceinline__ void moments(const AdamwHyper& h, float g, float& m, float& v) {
  m = __fadd_rn(__fmul_rn(m, h.b1), __fmul_rn(g, h.omb1));
  v = __fadd_rn(__fmul_rn(v, h.b2), __fmul_rn(__fmul_rn(g, h.omb2), g));
}
__device__ __forceinline__ float weight(const AdamwHyper& h, const Rates& r, float p, float m,
                                        float v) {
  return fmaf(p, r.keep, -__fdividef(r.rate * m, fmaf(root(v), r.ib2, h.eps)));
}

// The tensor of this CTA and the CTA's place in it.
template <int CAP>
__device__ __forceinline__ int find(const AdamwTable<CAP>& a, long long& at) {
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.e[mid].first <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  at = (long long)(blockIdx.x - a.e[lo].first) * a.chunk;
  return lo;
}

}  // namespace

// States in 32 bits.  Every element is read and written once and costs about 36
// instructions: bandwidth decides (52 M bf16 weights with masters: 214 us, 6.8 TB/s; 144 M
// fp32 weights: 575 us, 7.0 TB/s).
template <class T, bool MASTER, int CAP>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ AdamwTable<CAP> a) {
  pdl_enter();
  long long at;
  const AdamwEntry& t = a.e[find(a, at)];
  const AdamwHyper& h = a.h;
  const Rates r = rates(h);
  const float gs = h.grad_scale ? *h.grad_scale : 1.f;
  T* __restrict__ p = static_cast<T*>(t.p);
  const T* __restrict__ g = static_cast<const T*>(t.g);
  float* __restrict__ m = static_cast<float*>(t.m);
  float* __restrict__ v = static_cast<float*>(t.v);
  float* __restrict__ w = t.master;
  if (t.vec && at + kChunk <= t.n) {
#pragma unroll 2
    for (int u = 0; u < kChunk / (4 * kThreads); ++u) {
      const long long i = at + (u * kThreads + (int)threadIdx.x) * 4;
      float pv[4], gv[4], mv[4], vv[4];
      if (MASTER) load4(w + i, pv);
      else load4(p + i, pv);
      load4(g + i, gv);
      load4(m + i, mv);
      load4(v + i, vv);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        moments(h, gv[e] * gs, mv[e], vv[e]);
        pv[e] = weight(h, r, pv[e], mv[e], vv[e]);
      }
      store4(m + i, mv);
      store4(v + i, vv);
      if (MASTER) store4(w + i, pv);
      store4(p + i, pv);
    }
    return;
  }
  const long long end = at + kChunk < t.n ? at + kChunk : t.n;
  for (long long i = at + threadIdx.x; i < end; i += kThreads) {
    float mi = m[i], vi = v[i];
    moments(h, to_f(g[i]) * gs, mi, vi);
    const float pi = weight(h, r, MASTER ? w[i] : to_f(p[i]), mi, vi);
    m[i] = mi;
    v[i] = vi;
    if (MASTER) w[i] = pi;
    p[i] = from_f<T>(pi);
  }
}

namespace {

// A byte as a float: placed into the last byte of 2^23, whose unit in the last place is 1.
__device__ __forceinline__ float byte_float(uint32_t word, int i) {
  return __uint_as_float(__byte_perm(word, 0x4B000000u, 0x7440u | i));
}
// Four codes of m (two's complement) and of v as the values that they stand for, in pairs
// (one instruction for two operations, each rounded as it is alone).
__device__ __forceinline__ void decode_m(uint32_t word, float s, Pair* m) {
  word ^= 0x80808080u;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float x, y;
    split(add2(pair(byte_float(word, 2 * i), byte_float(word, 2 * i + 1)), both(-8388736.f)), x, y);
    m[i] = mul2(pair(x * fabsf(x), y * fabsf(y)), both(s));
  }
}
__device__ __forceinline__ void decode_v(uint32_t word, float r, Pair* v) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const Pair c = add2(pair(byte_float(word, 2 * i), byte_float(word, 2 * i + 1)), both(-8388608.f));
    const Pair q = mul2(mul2(c, c), both(r));
    v[i] = mul2(q, q);
  }
}
// A sum of products that stay rounded: one at a time (a packed product and a packed sum came out
// as one rounding).
__device__ __forceinline__ Pair sum2(Pair a, Pair b) {
  float a0, a1, b0, b1;
  split(a, a0, a1);
  split(b, b0, b1);
  return pair(__fadd_rn(a0, b0), __fadd_rn(a1, b1));
}
__device__ __forceinline__ float root_ftz(float x) {
  float y;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal_ftz(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float x, float y) {   // NaN where one is
  float z;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
  return z;
}
// A count of thresholds as the float 1.5 * 2^23 + count, whose last byte is the code: what is
// added to the root, rounded to an integer there, is the count or one more (the roots below are
// within 2^-20 of their values, and 2^-18 of them is added): the threshold decides.
constexpr float kToInt = 12582912.f, kMore = 1.f + 1.f / (1 << 18);
__device__ __forceinline__ void round2(Pair roots, Pair& t, Pair& k) {
  t = fma2(roots, both(kMore), both(kToInt));
  k = add2(t, both(-kToInt));
}
// Signed codes of m: x = |m| / s.  The threshold's square keeps the sign of k - 1/2, so that 0
// stays.
__device__ __forceinline__ void code_m(Pair m, float si, float& c0, float& c1) {
  float a, b, k0, k1;
  split(m, a, b);
  const float xa = fabsf(a) * si, xb = fabsf(b) * si;
  Pair t, k;
  round2(pair(copysignf(root_ftz(xa), a), copysignf(root_ftz(xb), b)), t, k);
  split(t, c0, c1);
  split(k, k0, k1);
  const float ha = fabsf(k0) - 0.5f, hb = fabsf(k1) - 0.5f;
  if (ha * fabsf(ha) > xa) c0 -= copysignf(1.f, a);
  if (hb * fabsf(hb) > xb) c1 -= copysignf(1.f, b);
}
// Codes of v: y = (v / r) / r; roots: of v.  least: kToInt + 1, the code of a v above 0 (kToInt in
// a block of zeros).
__device__ __forceinline__ void code_v(Pair v, Pair roots, float qi, float least, float& c0, float& c1) {
  const Pair q2 = both(qi), y = mul2(mul2(v, q2), q2);
  float a, b, ya, yb, r0, r1, h0, h1;
  split(v, a, b);
  split(y, ya, yb);
  split(mul2(roots, q2), r0, r1);
  Pair t, k;
  round2(pair(root_ftz(r0), root_ftz(r1)), t, k);
  split(t, c0, c1);
  Pair h = add2(k, both(-0.5f));
  h = mul2(h, h);
  split(mul2(h, h), h0, h1);
  if (h0 > ya) c0 -= 1.f;
  if (h1 > yb) c1 -= 1.f;
  c0 = fmaxf(c0, a > 0.f ? least : kToInt);
  c1 = fmaxf(c1, b > 0.f ? least : kToInt);
}
__device__ __forceinline__ uint32_t pack4(const float* t) {
  return __byte_perm(__byte_perm(__float_as_uint(t[0]), __float_as_uint(t[1]), 0x0040),
                     __byte_perm(__float_as_uint(t[2]), __float_as_uint(t[3]), 0x0040), 0x5410);
}

}  // namespace

// States in 8 bits: a warp takes a block of 256 elements, eight per lane, whose largest
// values are a maximum over the warp.  67 instructions an element against 10 bytes (bf16):
// issue slots decide (71% of them; 52 M weights: 128 us, 79 at the copy's rate).  Operation by
// operation it took 104 instructions and 195 us, without the next block on its way 167.  FTZ: a
// v below 2^-126 has no root (small_roots_do_not_count chooses).
template <class T, bool MASTER, bool FTZ, int CAP>
__global__ void __launch_bounds__(kThreads) adamw8_kernel(const __grid_constant__ AdamwTable<CAP> a) {
  pdl_enter();
  long long at;
  const AdamwEntry& t = a.e[find(a, at)];
  const AdamwHyper& h = a.h;
  const Rates r = rates(h);
  const float gs = h.grad_scale ? *h.grad_scale : 1.f;
  const int lane = threadIdx.x & 31;
  T* __restrict__ p = static_cast<T*>(t.p);
  const T* __restrict__ g = static_cast<const T*>(t.g);
  uint8_t* __restrict__ mc = static_cast<uint8_t*>(t.m);
  uint8_t* __restrict__ vc = static_cast<uint8_t*>(t.v);
  float* __restrict__ w = t.master;
  // a block as it is stored, fetched while the one before it is computed
  struct Stored {
    float s, r;
    Raw8<T> p, g;
    Raw8<float> w;
    uint2 m, v;
  };
  const long long end = min(t.n, at + a.chunk);
  auto fetch_block = [&](long long b0, Stored& x) {
    if (b0 >= end) return;
    const long long i = b0 + lane * 8;
    x.s = t.m_scale[b0 / kBlock];
    x.r = t.v_scale[b0 / kBlock];
    if (t.vec && b0 + kBlock <= t.n) {
      if (MASTER) fetch(w + i, x.w);
      else fetch(p + i, x.p);
      fetch(g + i, x.g);
      x.m = *reinterpret_cast<const uint2*>(mc + i);
      x.v = *reinterpret_cast<const uint2*>(vc + i);
    } else {   // zeros past the end, whose moments stay zeros
      const int left = (int)min(8ll, max(0ll, t.n - i));
      if (MASTER) gather8(w + i, 1, left, x.w);
      else gather8(p + i, 1, left, x.p);
      gather8(g + i, 1, left, x.g);
      x.m = x.v = make_uint2(0, 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t mb = e < left ? mc[i + e] : 0u, vb = e < left ? vc[i + e] : 0u;
        (e < 4 ? x.m.x : x.m.y) |= mb << 8 * (e & 3);
        (e < 4 ? x.v.x : x.v.y) |= vb << 8 * (e & 3);
      }
    }
  };
  const long long first = at + (threadIdx.x >> 5) * kBlock;
  constexpr int kStep = kThreads / 32 * kBlock;
  Stored next;
  fetch_block(first, next);
#pragma unroll 1
  for (long long b0 = first; b0 < end; b0 += kStep) {   // whole warps
    const Stored x = next;
    fetch_block(b0 + kStep, next);
    const long long blk = b0 / kBlock, i = b0 + lane * 8;
    const bool whole = t.vec && b0 + kBlock <= t.n;
    const int left = (int)min(8ll, max(0ll, t.n - i));
    float pv[8], gv[8];
    if (MASTER) widen(x.w, pv);
    else widen(x.p, pv);
    widen(x.g, gv);
    uint2 mw = x.m, vw = x.v;
    const float s0 = x.s, r0 = x.r;
    Pair m[4], v[4], roots[4];
    decode_m(mw.x, s0, m);
    decode_m(mw.y, s0, m + 2);
    decode_v(vw.x, r0, v);
    decode_v(vw.y, r0, v + 2);
    float mm = 0.f, vm = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const Pair x = mul2(pair(gv[2 * e], gv[2 * e + 1]), both(gs));
      m[e] = sum2(mul2(m[e], both(h.b1)), mul2(x, both(h.omb1)));
      v[e] = sum2(mul2(v[e], both(h.b2)), mul2(mul2(x, both(h.omb2)), x));
      float m0, m1, v0, v1;
      split(m[e], m0, m1);
      split(v[e], v0, v1);
      // p keep - rate m / (root(v) ib2 + eps)
      float d0, d1, q0, q1;
      roots[e] = FTZ ? pair(root_ftz(v0), root_ftz(v1)) : pair(root(v0), root(v1));
      split(fma2(roots[e], both(r.ib2), both(h.eps)), d0, d1);
      const Pair q = FTZ ? mul2(m[e], pair(reciprocal_ftz(d0), reciprocal_ftz(d1)))
                         : pair(__fdividef(m0, d0), __fdividef(m1, d1));
      split(fma2(q, both(-r.rate), mul2(pair(pv[2 * e], pv[2 * e + 1]), both(r.keep))), q0, q1);
      pv[2 * e] = q0;
      pv[2 * e + 1] = q1;
      mm = max_nan(mm, max_nan(fabsf(m0), fabsf(m1)));
      vm = max_nan(vm, max_nan(v0, v1));
    }
    // the largest as bits: the order of the values, with NaN above infinity
    const uint32_t mb = __reduce_max_sync(0xffffffffu, __float_as_uint(mm));
    const uint32_t vb = __reduce_max_sync(0xffffffffu, __float_as_uint(vm));
    float s = __fmul_rn(__uint_as_float(mb), (float)(1.0 / 16129.0));
    float q = __fmul_rn(__fsqrt_rn(__uint_as_float(vb)), (float)(1.0 / 65025.0));
    // below these the reciprocal (its square) is no float: held as zeros
    if (s < 0x1p-100f) s = 0.f;
    if (q < 0x1p-60f) q = 0.f;
    const float si = s == 0.f ? 0.f : __frcp_rn(s), qi = q == 0.f ? 0.f : __frcp_rn(q);
    const float least = qi > 0.f ? kToInt + 1.f : kToInt;
    float cm[8], cv[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      code_m(m[e], si, cm[2 * e], cm[2 * e + 1]);
      code_v(v[e], roots[e], qi, least, cv[2 * e], cv[2 * e + 1]);
    }
    mw = make_uint2(pack4(cm), pack4(cm + 4));
    vw = make_uint2(pack4(cv), pack4(cv + 4));
    if (lane == 0) {
      t.m_scale[blk] = s;
      t.v_scale[blk] = q;
    }
    if (whole) {
      *reinterpret_cast<uint2*>(mc + i) = mw;
      *reinterpret_cast<uint2*>(vc + i) = vw;
      if (MASTER) store8(w + i, pv);
      store8(p + i, pv);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < left) {
          mc[i + e] = (uint8_t)((e < 4 ? mw.x : mw.y) >> 8 * (e & 3));
          vc[i + e] = (uint8_t)((e < 4 ? vw.x : vw.y) >> 8 * (e & 3));
          if (MASTER) w[i + e] = pv[e];
          p[i + e] = from_f<T>(pv[e]);
        }
    }
  }
}

// The values that 8-bit states stand for, four per thread (52 M: 79 us, 6.7 TB/s).
__global__ void __launch_bounds__(kThreads)
    adamw8_values_kernel(const uint8_t* __restrict__ mc, const float* __restrict__ ms,
                         const uint8_t* __restrict__ vc, const float* __restrict__ vs,
                         float* __restrict__ m, float* __restrict__ v, long long n) {
  pdl_enter();
  const long long step = (long long)gridDim.x * kThreads * 4;
  for (long long i = ((long long)blockIdx.x * kThreads + threadIdx.x) * 4; i < n; i += step) {
    const float s = ms[i / kBlock], r = vs[i / kBlock];
    float a[4], b[4];
    auto decode = [&](uint32_t mw, uint32_t vw) {
      Pair x[2], y[2];
      decode_m(mw, s, x);
      decode_v(vw, r, y);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        split(x[e], a[2 * e], a[2 * e + 1]);
        split(y[e], b[2 * e], b[2 * e + 1]);
      }
    };
    if (i + 4 <= n) {
      decode(*reinterpret_cast<const uint32_t*>(mc + i), *reinterpret_cast<const uint32_t*>(vc + i));
      store4(m + i, a);
      store4(v + i, b);
    } else {
      uint32_t mw = 0, vw = 0;
      for (int e = 0; i + e < n; ++e) {
        mw |= (uint32_t)mc[i + e] << 8 * e;
        vw |= (uint32_t)vc[i + e] << 8 * e;
      }
      decode(mw, vw);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i + e < n) {
          m[i + e] = a[e];
          v[i + e] = b[e];
        }
    }
  }
}

namespace {

// Whether the root of a v below 2^-126 may count as 0: where it is less than 2^-24 of eps at
// every step (1 / sqrt(1 - b2^t) is largest at the first).
bool small_roots_do_not_count(const AdamwHyper& h) {
  return h.eps * 0x1p-24 >= 0x1p-63 / sqrt(1.0 - exp(h.log_b2));
}

template <class T, bool MASTER, int CAP>
cudaError_t launch_table(const Launch& lc, int bits, const AdamwHyper& h, const AdamwEntry* e,
                         int count, unsigned blocks, int chunk) {
  AdamwTable<CAP> a;
  a.chunk = chunk;
  std::copy(e, e + count, a.e);
  a.h = h;
  a.count = count;
  if (bits == 8 && small_roots_do_not_count(h))
    return launch_k(adamw8_kernel<T, MASTER, true, CAP>, dim3(blocks), dim3(kThreads), 0, lc.stream, a);
  return bits == 8 ? launch_k(adamw8_kernel<T, MASTER, false, CAP>, dim3(blocks), dim3(kThreads), 0, lc.stream, a)
                   : launch_k(adamw_kernel<T, MASTER, CAP>, dim3(blocks), dim3(kThreads), 0, lc.stream, a);
}
// The table travels with the launch: the smallest that holds it, 384 tensors a launch.
template <class T, bool MASTER>
cudaError_t launch_typed(const Launch& lc, int bits, const AdamwHyper& h, const AdamwEntry* e,
                         int count, unsigned blocks, int chunk) {
  if (count <= 32) return launch_table<T, MASTER, 32>(lc, bits, h, e, count, blocks, chunk);
  if (count <= 128) return launch_table<T, MASTER, 128>(lc, bits, h, e, count, blocks, chunk);
  return launch_table<T, MASTER, 384>(lc, bits, h, e, count, blocks, chunk);
}

}  // namespace

cudaError_t adamw_step(const Launch& lc, int dtype, int bits, bool master, const AdamwHyper& h,
                       const AdamwTensor* t, int count) {
  AdamwEntry e[384];
  int k = 0;
  unsigned long long blocks = 0;
  cudaError_t err = cudaSuccess;
  long long all = 0;
  for (int i = 0; i < count; ++i) all += t[i].n;
  const int chunk = bits == 8 && all > (1ll << 24) ? 2 * kChunk : kChunk;
  auto flush = [&] {
    if (k > 0)
      err = dtype == 0 ? launch_typed<float, false>(lc, bits, h, e, k, (unsigned)blocks, chunk)
            : master   ? launch_typed<bf16, true>(lc, bits, h, e, k, (unsigned)blocks, chunk)
                       : launch_typed<bf16, false>(lc, bits, h, e, k, (unsigned)blocks, chunk);
    k = 0;
    blocks = 0;
  };
  for (int i = 0; i < count && err == cudaSuccess; ++i) {
    if (t[i].n == 0) continue;
    const unsigned long long need = (unsigned long long)((t[i].n + chunk - 1) / chunk);
    if (k == 384 || blocks + need > 0x7fffffffull) flush();
    // 16-byte accesses of p and master, 8- or 16-byte ones of the rest
    const uintptr_t at = (uintptr_t)t[i].p | (uintptr_t)t[i].g | (uintptr_t)t[i].m |
                         (uintptr_t)t[i].v | (uintptr_t)t[i].master;
    e[k] = AdamwEntry{t[i].p, t[i].g, t[i].m, t[i].v, t[i].master, t[i].m_scale, t[i].v_scale,
                      t[i].n, (unsigned)blocks, at % 16 == 0};
    ++k;
    blocks += need;
  }
  if (err == cudaSuccess) flush();
  return err;
}

cudaError_t adamw_values(const Launch& lc, const uint8_t* mc, const float* ms, const uint8_t* vc,
                         const float* vs, float* m, float* v, long long n) {
  if (n == 0) return cudaSuccess;
  const unsigned blocks = (unsigned)std::min<long long>((n + 4 * kThreads - 1) / (4 * kThreads), 1ll << 22);
  return launch_k(adamw8_values_kernel, dim3(blocks), dim3(kThreads), 0, lc.stream, mc, ms, vc, vs,
                  m, v, n);
}

}  // namespace bcmt
