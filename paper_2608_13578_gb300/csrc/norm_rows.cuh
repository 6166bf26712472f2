// Rows of D channels over the threads of a warp or CTA: loads, stores and sums over a
// row, shared by the kernels of the norms around a block.
#pragma once

#include "common.cuh"
#include "pairs.cuh"

namespace bcmt {

namespace {

// Eight elements as they are stored.
template <class T> struct Raw8;
template <> struct Raw8<float> {
  float4 a, b;
};
template <> struct Raw8<bf16> {
  uint4 a;
};
__device__ __forceinline__ void widen(const Raw8<float>& r, float* v) {
  v[0] = r.a.x; v[1] = r.a.y; v[2] = r.a.z; v[3] = r.a.w;
  v[4] = r.b.x; v[5] = r.b.y; v[6] = r.b.z; v[7] = r.b.w;
}
__device__ __forceinline__ void widen(const Raw8<bf16>& r, float* v) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void zero(Raw8<float>& r) {
  r.a = r.b = make_float4(0.f, 0.f, 0.f, 0.f);
}
__device__ __forceinline__ void zero(Raw8<bf16>& r) { r.a = make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ void fetch(const float* p, Raw8<float>& r) {
  r.a = *reinterpret_cast<const float4*>(p);
  r.b = *reinterpret_cast<const float4*>(p + 4);
}
__device__ __forceinline__ void fetch(const bf16* p, Raw8<bf16>& r) {
  r.a = *reinterpret_cast<const uint4*>(p);
}
__device__ __forceinline__ void gather8(const float* p, int step, int n, Raw8<float>& r) {
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? p[(long)e * step] : 0.f;
  r.a = make_float4(v[0], v[1], v[2], v[3]);
  r.b = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void gather8(const bf16* p, int step, int n, Raw8<bf16>& r) {
  const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
  uint32_t v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? q[(long)e * step] : 0u;
  r.a = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

__device__ __forceinline__ Pair shfl_xor(Pair p, int o) {
  float x, y;
  split(p, x, y);
  return pair(__shfl_xor_sync(0xffffffffu, x, o), __shfl_xor_sync(0xffffffffu, y, o));
}

// Loads from shared memory that are not kept from an earlier one of the same place: where a
// value is read anew, its registers are meant to be free in between.
__device__ __forceinline__ uint32_t shared_address(const void* p) {
  return (uint32_t)__cvta_generic_to_shared(p);
}
__device__ __forceinline__ void load_shared(uint32_t p, Pair& x, Pair& y) {
  asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(x), "=l"(y) : "r"(p) : "memory");
}
__device__ __forceinline__ void load_shared(uint32_t p, uint4& v) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "r"(p) : "memory");
}
template <class T> __device__ __forceinline__ float load_shared(uint32_t p);
template <> __device__ __forceinline__ float load_shared<float>(uint32_t p) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(p) : "memory");
  return v;
}
template <> __device__ __forceinline__ float load_shared<bf16>(uint32_t p) {
  unsigned short v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(p) : "memory");
  return __uint_as_float((uint32_t)v << 16);
}
__device__ __forceinline__ void store_shared(uint32_t p, Pair x, Pair y) {
  asm volatile("st.shared.v2.b64 [%0], {%1, %2};" ::"r"(p), "l"(x), "l"(y) : "memory");
}
template <class T>
__device__ __forceinline__ void widen2(const Raw8<T>& r, Pair* p) {
  float v[8];
  widen(r, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = pair(v[2 * i], v[2 * i + 1]);
}

// The eight columns of a row that thread t of `tpr` takes in its j-th turn: VEC, eight
// consecutive ones in one 16-byte (fp32: two) access, for D a multiple of 8; else every
// tpr-th column, so that a warp's accesses are consecutive.  `count`: how many of them
// are below D.
template <bool VEC>
struct Cols {
  int first, step, count;
  __device__ __forceinline__ Cols(int first_, int step_, int count_)
      : first(first_), step(step_), count(count_) {}
  __device__ __forceinline__ Cols(int t, int tpr, int j, int D) {
    if (VEC) {
      first = (t + j * tpr) * 8;
      step = 1;
      count = first < D ? 8 : 0;
    } else {
      first = t + j * 8 * tpr;
      step = tpr;
      count = first < D ? min(8, (D - first + tpr - 1) / tpr) : 0;
    }
  }
};

template <bool VEC, class T>
__device__ __forceinline__ void read8(const T* row, const Cols<VEC>& c, bool live, Raw8<T>& r) {
  if (VEC) {
    if (live && c.count) fetch(row + c.first, r);
    else zero(r);
  } else {
    gather8(row + c.first, c.step, live ? c.count : 0, r);
  }
}
// A vector of weights (either type), zeros past D.
template <bool VEC>
__device__ __forceinline__ void read_weight(const void* w, bool is_bf16, const Cols<VEC>& c,
                                            float* v) {
  if (is_bf16) {
    Raw8<bf16> r;
    read8<VEC>(static_cast<const bf16*>(w), c, true, r);
    widen(r, v);
  } else {
    Raw8<float> r;
    read8<VEC>(static_cast<const float*>(w), c, true, r);
    widen(r, v);
  }
}
template <bool VEC, class T>
__device__ __forceinline__ void write8(T* row, const Cols<VEC>& c, const float* v) {
  if (VEC) {
    if (c.count) store8(row + c.first, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < c.count) row[c.first + (long)e * c.step] = from_f<T>(v[e]);
  }
}

template <bool VEC, class T>
__device__ __forceinline__ void write8(T* row, const Cols<VEC>& c, const Pair* p) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) split(p[i], v[2 * i], v[2 * i + 1]);
  write8<VEC>(row, c, v);
}

// Sums of NV (1, 2 or 4) values over the threads of a row, given to all of them.  Each
// step of a warp's sum halves the values while there is more than one (a lane keeps one
// half of them and hands the other to its partner), then the lanes: 4 values take 6
// exchanges, not 20.  Up to 32 threads: lanes of a warp.  More: the row's warps add
// through shared memory, `slot` alternating between two buffers, so that one barrier a
// sum is enough.
__device__ __forceinline__ void bar_sync(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
constexpr int kMaxWarps = 24;
struct RowShared {
  float4 sums[2][kMaxWarps];
};
template <int TPR, int NV>
__device__ __forceinline__ void row_sums(float (&v)[NV], RowShared& sh, int& slot, int warp0,
                                         int nw, int bar) {
  static_assert(NV == 1 || NV == 2 || NV == 4, "");
  const int lane = threadIdx.x & 31;
  constexpr int W = TPR < 32 ? TPR : 32;
  float a[2], s;
  if (NV == 4) {
    const bool up = lane & 2;   // keeps values 2, 3
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float give = up ? v[i] : v[NV == 4 ? 2 + i : 0], keep = up ? v[NV == 4 ? 2 + i : 0] : v[i];
      a[i] = keep + __shfl_xor_sync(0xffffffffu, give, 2);
    }
  } else {
    a[0] = v[0];
    a[1] = NV == 2 ? v[NV == 2 ? 1 : 0] : 0.f;
  }
  if (NV >= 2) {
    const bool up = lane & 1;   // keeps the second of its values
    const float give = up ? a[0] : a[1], keep = up ? a[1] : a[0];
    s = keep + __shfl_xor_sync(0xffffffffu, give, 1);
  } else {
    s = a[0];
  }
#pragma unroll
  for (int o = W / 2; o >= NV; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (TPR <= 32) {
    // lane i (of every NV) holds the sum of value i
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = NV == 1 ? s : __shfl_sync(0xffffffffu, s, (lane & ~(NV - 1)) | i);
  } else {
    float4* buf = sh.sums[slot];
    slot ^= 1;
    if (lane < NV) reinterpret_cast<float*>(buf + (threadIdx.x >> 5))[lane] = s;
    bar_sync(bar, nw * 32);
    // lane: a value (lane mod NV) of a warp; the warps' together, in the same order in every lane
    float f = 0.f;
#pragma unroll 1
    for (int w = lane / NV; w < nw; w += 32 / NV)
      f += reinterpret_cast<const float*>(buf + warp0 + w)[lane & (NV - 1)];
#pragma unroll
    for (int o = 16; o >= NV; o >>= 1) f += __shfl_xor_sync(0xffffffffu, f, o);
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = NV == 1 ? f : __shfl_sync(0xffffffffu, f, i);
  }
}

// Asynchronous copies to shared memory: a thread waits for those that it has issued.
// 16 bytes, of which the first n are read and the others are zeros.
__device__ __forceinline__ void copy_async16(uint32_t s, const void* g, int n) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(s), "l"(g), "r"(n) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory");
}

}  // namespace

}  // namespace bcmt
