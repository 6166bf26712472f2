// Backward of the norms around a block (the formulas are in norms.cu), for one type of
// rows.
#pragma once

#include <atomic>

#include "norm_rows.cuh"
#include "norms.h"

namespace bcmt {

// Backward.  Workers (the TPR threads of one row at a time) walk segments of consecutive
// rows, each of one gate; a thread's columns are the same in every row, so the columns'
// sums stay in its registers (SMEM_ACC: rows too wide for that keep them in shared
// memory), and reach global memory once per CTA, the gate's once per segment.  The next
// row's elements are loaded while the sums of this one are taken.
template <class T, int TPR, int J, bool VEC, bool POST, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) norm_bwd_kernel(const NormBwd a) {
  extern __shared__ float dyn[];
  __shared__ RowShared sh;
  constexpr int E = 8 * J;
  constexpr bool SMEM_ACC = J > 1;
  constexpr int NACC = POST ? 4 : 2;
  pdl_enter();
  const int tpr = TPR > 32 ? a.tpr : TPR;
  const int rg = threadIdx.x / tpr, t = threadIdx.x - rg * tpr;
  const int nw = tpr / 32, warp0 = rg * nw, bar = 1 + rg;
  const int D = a.D;
  const float inv = 1.f / D;
  const long long workers = (long long)gridDim.x * a.rows_per_cta;
  long long seg = (long long)blockIdx.x * a.rows_per_cta + rg;
  int slot = 0;

  float acc[SMEM_ACC ? 1 : NACC][SMEM_ACC ? 1 : E];
  float gacc[SMEM_ACC ? 1 : E];
  auto add = [&](int i, int e, float v) {
    if constexpr (SMEM_ACC) dyn[(i * E + e) * THREADS + t] += v;
    else if (i == NACC) gacc[e] += v;
    else acc[i][e] += v;
  };
  if constexpr (SMEM_ACC) {
    for (int i = 0; i < (NACC + 1) * E; ++i) dyn[i * THREADS + t] = 0.f;
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      gacc[e] = 0.f;
#pragma unroll
      for (int i = 0; i < NACC; ++i) acc[i][e] = 0.f;
    }
  }
  float w[E], pw[POST ? E : 1], pb[POST ? E : 1], g[E];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const Cols<VEC> c(t, tpr, j, D);
    read_weight<VEC>(a.weight, a.w_bf16, c, w + 8 * j);
    if (POST) {
      read_weight<VEC>(a.post_weight, a.w_bf16, c, pw + 8 * j);
      if (a.post_bias) read_weight<VEC>(a.post_bias, a.w_bf16, c, pb + 8 * j);
      else
#pragma unroll
        for (int e = 0; e < 8; ++e) pb[8 * j + e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) g[8 * j + e] = 1.f;
  }

  // segment `s` covers rows [first, end)
  auto bounds = [&](long long s, long long& first, long long& end) {
    const long long grp = s / a.segs_per_group, k = s - grp * a.segs_per_group;
    first = grp * a.seg_group_rows + k * a.seg_rows;
    end = min(first + a.seg_rows, (grp + 1) * a.seg_group_rows);
    if (s >= a.nseg || first > end) end = first;
  };
  Raw8<T> rdh[J], rdn[J], ry[J], rh[J];
  auto read_rows = [&](long long row, bool live) {
    const long long at = live ? row * D : 0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const Cols<VEC> c(t, tpr, j, D);
      if (a.dh) read8<VEC>(static_cast<const T*>(a.dh) + at, c, live, rdh[j]);
      else zero(rdh[j]);
      read8<VEC>(static_cast<const T*>(a.dn) + at, c, live, rdn[j]);
      read8<VEC>(static_cast<const T*>(a.h) + at, c, live, rh[j]);
      if (POST || a.gate) read8<VEC>(static_cast<const T*>(a.branch) + at, c, live, ry[j]);
      else zero(ry[j]);
    }
  };

  long long first, end;
  bounds(seg, first, end);
  read_rows(first, first < end);
  // every worker makes the same number of turns (a.turns segments of a.seg_rows rows):
  // lanes of a warp that belong to different workers stay together
  for (int turn = 0; turn < a.turns; ++turn) {
    if (a.gate && a.group_rows > 1) {
      const long long grp = seg / a.segs_per_group;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const Cols<VEC> c(t, tpr, j, D);
        Raw8<T> r;
        read8<VEC>(static_cast<const T*>(a.gate) + (first < end ? grp * D : 0), c, first < end, r);
        widen(r, g + 8 * j);
      }
    }
    for (long long k = 0; k < a.seg_rows; ++k) {
      const long long row = first + k;
      const bool live = row < end;
      float dh[E], dn[E], y[E], h[E];
#pragma unroll
      for (int j = 0; j < J; ++j) {
        widen(rdh[j], dh + 8 * j);
        widen(rdn[j], dn + 8 * j);
        widen(ry[j], y + 8 * j);
        widen(rh[j], h + 8 * j);
      }
      if (k + 1 < a.seg_rows) {
        read_rows(row + 1, row + 1 < end);
      } else if (turn + 1 < a.turns) {
        long long f, e;
        bounds(seg + workers, f, e);
        read_rows(f, f < e);
      }
      if (a.gate && a.group_rows == 1) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Cols<VEC> c(t, tpr, j, D);
          Raw8<T> r;
          read8<VEC>(static_cast<const T*>(a.gate) + (live ? row * D : 0), c, live, r);
          widen(r, g + 8 * j);
        }
      }
      float mh = 0.f, my = 0.f;
      if (a.layer) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) {
          s[0] += h[e];
          if (POST) s[1] += y[e];
        }
        row_sums<TPR, 2>(s, sh, slot, warp0, nw, bar);
        mh = s[0] * inv;
        my = s[1] * inv;
      }
      // the squares, and the sums of e = dn w and e (h - mean)
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const Cols<VEC> c(t, tpr, j, D);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = 8 * j + i;
          h[e] = i < c.count ? h[e] - mh : 0.f;
          if (POST) y[e] = i < c.count ? y[e] - my : 0.f;
          const float d = dn[e] * w[e];
          s[0] = fmaf(h[e], h[e], s[0]);
          if (POST) s[1] = fmaf(y[e], y[e], s[1]);
          s[2] += d;
          s[3] = fmaf(d, h[e], s[3]);
        }
      }
      row_sums<TPR, 4>(s, sh, slot, warp0, nw, bar);
      const float rh_ = live ? 1.f / sqrtf(s[0] * inv + a.eps) : 0.f;
      const float ry_ = POST && live ? 1.f / sqrtf(s[1] * inv + a.eps) : 0.f;
      const float c1 = a.layer ? rh_ * s[2] * inv : 0.f;
      const float c2 = rh_ * rh_ * s[3] * inv;
      float b[2] = {0.f, 0.f};
      float* ds = dh;   // the sum's gradient, then dz, then dy
#pragma unroll
      for (int j = 0; j < J; ++j) {
        float out[8], gg[8];
        const Cols<VEC> c(t, tpr, j, D);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = 8 * j + i;
          const float hh = h[e] * rh_;
          ds[e] += fmaf(rh_ * w[e], dn[e], -fmaf(hh, c2, c1));
          add(0, e, dn[e] * hh);
          if (a.layer) add(1, e, dn[e]);
          out[i] = a.alpha * ds[e];
          const float yh = POST ? y[e] * ry_ : y[e];
          if (a.gate) {
            gg[i] = ds[e] * (POST ? fmaf(yh, pw[e], pb[e]) : yh);
            if (a.group_rows > 1) add(NACC, e, gg[i]);
            ds[e] *= g[e];
          }
          if (POST) {
            add(POST ? 2 : 0, e, ds[e] * yh);
            if (a.layer) add(POST ? 3 : 0, e, ds[e]);
            ds[e] *= pw[e];
            b[0] += ds[e];
            b[1] = fmaf(ds[e], y[e], b[1]);
          }
        }
        if (live) {
          if (a.dx) write8<VEC>(static_cast<T*>(a.dx) + row * D, c, out);
          if (a.gate && a.group_rows == 1 && a.dgate)
            write8<VEC>(static_cast<T*>(a.dgate) + row * D, c, gg);
        }
      }
      if (POST) {
        row_sums<TPR, 2>(b, sh, slot, warp0, nw, bar);
        const float d1 = a.layer ? ry_ * b[0] * inv : 0.f;
        const float d2 = ry_ * ry_ * ry_ * b[1] * inv;
#pragma unroll
        for (int e = 0; e < E; ++e) ds[e] = fmaf(ry_, ds[e], -fmaf(y[e], d2, d1));
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const Cols<VEC> c(t, tpr, j, D);
        if (live) write8<VEC>(static_cast<T*>(a.dbranch) + row * D, c, ds + 8 * j);
      }
    }
    // the gate's gradient of this segment
    if (a.gate && a.group_rows > 1 && a.dgate) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const Cols<VEC> c(t, tpr, j, D);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (SMEM_ACC) {
            float& f = dyn[(NACC * E + 8 * j + e) * THREADS + t];
            v[e] = f;
            f = 0.f;
          } else {
            v[e] = gacc[8 * j + e];
            gacc[8 * j + e] = 0.f;
          }
        }
        if (seg < a.nseg) {
          if (a.segs_per_group == 1) write8<VEC>(static_cast<T*>(a.dgate) + seg * D, c, v);
          else write8<VEC>(a.gate_part + seg * D, c, v);
        }
      }
    }
    seg += workers;
    bounds(seg, first, end);
  }
  // the CTA's sums: its workers' through shared memory, one vector at a time
#pragma unroll
  for (int i = 0; i < NACC; ++i) {
    if ((i & 1) && !a.layer) continue;
    float* part = a.part + ((long long)blockIdx.x * 4 + i) * D;
    if constexpr (SMEM_ACC) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = dyn[(i * E + 8 * j + e) * THREADS + t];
        write8<VEC>(part, Cols<VEC>(t, tpr, j, D), v);
      }
    } else if (a.rows_per_cta == 1) {
      write8<VEC>(part, Cols<VEC>(t, tpr, 0, D), acc[i]);
    } else {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) dyn[e * THREADS + threadIdx.x] = acc[i][e];
      __syncthreads();
      if (rg == 0) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = 0.f;
          for (int k = 0; k < a.rows_per_cta; ++k) v[e] += dyn[e * THREADS + k * tpr + t];
        }
        write8<VEC>(part, Cols<VEC>(t, tpr, 0, D), v);
      }
    }
  }
}

namespace {

template <class T, int TPR, int J, bool POST, int THREADS, int CTAS>
cudaError_t bwd_shape(const Launch& lc, const NormBwd& a, int ctas, int threads, int smem) {
  static std::atomic<unsigned long long> done_v{0}, done_s{0};
  const dim3 grid(ctas), block(threads);
  if (a.D % 8 == 0) {
    auto k = norm_bwd_kernel<T, TPR, J, true, POST, THREADS, CTAS>;
    if (smem > 40960) {
      cudaError_t e = smem_opt_in(k, smem, &done_v);
      if (e != cudaSuccess) return e;
    }
    return launch_k(k, grid, block, smem, lc.stream, a);
  }
  auto k = norm_bwd_kernel<T, TPR, J, false, POST, THREADS, CTAS>;
  if (smem > 40960) {
    cudaError_t e = smem_opt_in(k, smem, &done_s);
    if (e != cudaSuccess) return e;
  }
  return launch_k(k, grid, block, smem, lc.stream, a);
}
template <class T, bool POST>
cudaError_t bwd_typed(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  if (pl.tpr == 16) return bwd_shape<T, 16, 1, POST, 256, 2>(lc, a, pl.ctas, pl.threads, pl.smem);
  if (pl.tpr == 32) return bwd_shape<T, 32, 1, POST, 256, 2>(lc, a, pl.ctas, pl.threads, pl.smem);
  if (pl.wide) return bwd_shape<T, 64, 2, POST, 512, 1>(lc, a, pl.ctas, pl.threads, pl.smem);
  if (pl.threads > 256) return bwd_shape<T, 64, 1, POST, 512, 1>(lc, a, pl.ctas, pl.threads, pl.smem);
  return bwd_shape<T, 64, 1, POST, 256, 2>(lc, a, pl.ctas, pl.threads, pl.smem);
}

}  // namespace

}  // namespace bcmt
