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

namespace bcmt {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;   // elements of a CTA
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
  at = (long long)(blockIdx.x - a.e[lo].first) * kChunk;
  return lo;
}

}  // namespace

// States in 32 bits.  Every element is read and written once and costs about 30
// instructions: bandwidth decides.
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
// Four codes of m (two's complement) and of v as the values that they stand for.
__device__ __forceinline__ void decode_m(uint32_t word, float s, float* m) {
  word ^= 0x80808080u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float c = byte_float(word, i) - 8388736.f;
    m[i] = __fmul_rn(c * fabsf(c), s);
  }
}
__device__ __forceinline__ void decode_v(uint32_t word, float r, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float c = byte_float(word, i) - 8388608.f, q = __fmul_rn(c * c, r);
    v[i] = __fmul_rn(q, q);
  }
}
constexpr float kToInt = 12582912.f;   // 1.5 * 2^23: adding it rounds to an integer
// The number of thresholds up to x.  The root is within 2^-21 of its value, and a little
// more is added, so that its rounding is the count or one more: the threshold decides.
__device__ __forceinline__ float count_m(float x) {
  float k = __fadd_rn(__fadd_rn(__fmul_rn(root(x), 1.f + 1.f / (1 << 19)), kToInt), -kToInt);
  const float h = k - 0.5f;
  if (__fmul_rn(h, h) > x) k -= 1.f;
  return fmaxf(k, 0.f);
}
__device__ __forceinline__ float count_v(float y) {
  float k = __fadd_rn(__fadd_rn(__fmul_rn(root(root(y)), 1.f + 1.f / (1 << 19)), kToInt), -kToInt);
  const float h = k - 0.5f, q = __fmul_rn(h, h);
  if (__fmul_rn(q, q) > y) k -= 1.f;
  return fmaxf(k, 0.f);
}
__device__ __forceinline__ uint32_t pack4(const float* k) {
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(__fadd_rn(k[i], kToInt));
  return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
}

}  // namespace

// States in 8 bits: a warp takes a block of 256 elements, eight per lane, whose largest
// values are a maximum over the warp.  About 70 instructions an element against 10 bytes
// (bf16): the arithmetic takes about as long as the bytes.
template <class T, bool MASTER, int CAP>
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
#pragma unroll 1
  for (int u = 0; u < kChunk / (kBlock * kThreads / 32); ++u) {
    const long long b0 = at + (u * (kThreads / 32) + (int)(threadIdx.x >> 5)) * kBlock;
    if (b0 >= t.n) return;   // the whole warp
    const long long blk = b0 / kBlock, i = b0 + lane * 8;
    const float s0 = t.m_scale[blk], r0 = t.v_scale[blk];
    const bool whole = t.vec && b0 + kBlock <= t.n;
    const int left = (int)min(8ll, max(0ll, t.n - i));
    float pv[8], gv[8], m[8], v[8];
    uint2 mw = make_uint2(0, 0), vw = make_uint2(0, 0);
    if (whole) {
      if (MASTER) load8(w + i, pv);
      else load8(p + i, pv);
      load8(g + i, gv);
      mw = *reinterpret_cast<const uint2*>(mc + i);
      vw = *reinterpret_cast<const uint2*>(vc + i);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool on = e < left;
        pv[e] = on ? (MASTER ? w[i + e] : to_f(p[i + e])) : 0.f;
        gv[e] = on ? to_f(g[i + e]) : 0.f;
        const uint32_t mb = on ? mc[i + e] : 0u, vb = on ? vc[i + e] : 0u;
        (e < 4 ? mw.x : mw.y) |= mb << 8 * (e & 3);
        (e < 4 ? vw.x : vw.y) |= vb << 8 * (e & 3);
      }
    }
    decode_m(mw.x, s0, m);
    decode_m(mw.y, s0, m + 4);
    decode_v(vw.x, r0, v);
    decode_v(vw.y, r0, v + 4);
    // the largest as bits: the order of the values, with NaN above infinity
    uint32_t mm = 0, vm = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      moments(h, gv[e] * gs, m[e], v[e]);
      pv[e] = weight(h, r, pv[e], m[e], v[e]);
      if (whole || e < left) {
        mm = max(mm, __float_as_uint(m[e]) & 0x7fffffffu);
        vm = max(vm, __float_as_uint(v[e]));
      }
    }
    mm = __reduce_max_sync(0xffffffffu, mm);
    vm = __reduce_max_sync(0xffffffffu, vm);
    float s = __fmul_rn(__uint_as_float(mm), (float)(1.0 / 16129.0));
    float q = __fmul_rn(__fsqrt_rn(__uint_as_float(vm)), (float)(1.0 / 65025.0));
    // below these the reciprocal (its square) is no float: held as zeros
    if (s < 0x1p-100f) s = 0.f;
    if (q < 0x1p-60f) q = 0.f;
    const float si = s == 0.f ? 0.f : __frcp_rn(s), qi = q == 0.f ? 0.f : __frcp_rn(q);
    float cm[8], cv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      cm[e] = copysignf(count_m(__fmul_rn(fabsf(m[e]), si)), m[e]);
      cv[e] = count_v(__fmul_rn(__fmul_rn(v[e], qi), qi));
      cv[e] = v[e] > 0.f && qi > 0.f ? fmaxf(cv[e], 1.f) : cv[e];
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

// The values that 8-bit states stand for, four per thread.
__global__ void __launch_bounds__(kThreads)
    adamw8_values_kernel(const uint8_t* __restrict__ mc, const float* __restrict__ ms,
                         const uint8_t* __restrict__ vc, const float* __restrict__ vs,
                         float* __restrict__ m, float* __restrict__ v, long long n) {
  pdl_enter();
  const long long step = (long long)gridDim.x * kThreads * 4;
  for (long long i = ((long long)blockIdx.x * kThreads + threadIdx.x) * 4; i < n; i += step) {
    const float s = ms[i / kBlock], r = vs[i / kBlock];
    float a[4], b[4];
    if (i + 4 <= n) {
      decode_m(*reinterpret_cast<const uint32_t*>(mc + i), s, a);
      decode_v(*reinterpret_cast<const uint32_t*>(vc + i), r, b);
      store4(m + i, a);
      store4(v + i, b);
    } else {
      uint32_t mw = 0, vw = 0;
      for (int e = 0; i + e < n; ++e) {
        mw |= (uint32_t)mc[i + e] << 8 * e;
        vw |= (uint32_t)vc[i + e] << 8 * e;
      }
      decode_m(mw, s, a);
      decode_v(vw, r, b);
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

template <class T, bool MASTER, int CAP>
cudaError_t launch_table(const Launch& lc, int bits, const AdamwHyper& h, const AdamwEntry* e,
                         int count, unsigned blocks) {
  AdamwTable<CAP> a;
  std::copy(e, e + count, a.e);
  a.h = h;
  a.count = count;
  return bits == 8 ? launch_k(adamw8_kernel<T, MASTER, CAP>, dim3(blocks), dim3(kThreads), 0, lc.stream, a)
                   : launch_k(adamw_kernel<T, MASTER, CAP>, dim3(blocks), dim3(kThreads), 0, lc.stream, a);
}
// The table travels with the launch: the smallest that holds it, 384 tensors a launch.
template <class T, bool MASTER>
cudaError_t launch_typed(const Launch& lc, int bits, const AdamwHyper& h, const AdamwEntry* e,
                         int count, unsigned blocks) {
  if (count <= 32) return launch_table<T, MASTER, 32>(lc, bits, h, e, count, blocks);
  if (count <= 128) return launch_table<T, MASTER, 128>(lc, bits, h, e, count, blocks);
  return launch_table<T, MASTER, 384>(lc, bits, h, e, count, blocks);
}

}  // namespace

cudaError_t adamw_step(const Launch& lc, int dtype, int bits, bool master, const AdamwHyper& h,
                       const AdamwTensor* t, int count) {
  AdamwEntry e[384];
  int k = 0;
  unsigned long long blocks = 0;
  cudaError_t err = cudaSuccess;
  auto flush = [&] {
    if (k > 0)
      err = dtype == 0 ? launch_typed<float, false>(lc, bits, h, e, k, (unsigned)blocks)
            : master   ? launch_typed<bf16, true>(lc, bits, h, e, k, (unsigned)blocks)
                       : launch_typed<bf16, false>(lc, bits, h, e, k, (unsigned)blocks);
    k = 0;
    blocks = 0;
  };
  for (int i = 0; i < count && err == cudaSuccess; ++i) {
    if (t[i].n == 0) continue;
    const unsigned long long need = (unsigned long long)((t[i].n + kChunk - 1) / kChunk);
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
