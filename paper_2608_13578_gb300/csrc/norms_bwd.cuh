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
// rows' elements are on their way to shared memory meanwhile (RING: bf16 rows whose
// elements are not in 16-byte pieces wait in registers instead, and with SMEM_ACC the next
// row is fetched into L2).
//
// With A = sum s yh and B = sum s over the rows of one gate, its gradient is pw A + pb B,
// and it adds g A to dpw and g B to dpb: the sums take A and B, and what depends on the
// gate is done once for its segment.
template <class T>
constexpr int ring_stages() {   // rows of a worker in shared memory, this one among them
  return sizeof(T) == 2 ? 3 : 2;
}

template <class T, int TPR, int J, bool VEC, bool POST, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) norm_bwd_kernel(const NormBwd a) {
  extern __shared__ float4 dyn4[];
  __shared__ RowShared sh;
  constexpr int Q = 4 * J;   // pairs of columns of a thread
  constexpr bool SMEM_ACC = J > 1;
  constexpr int NACC = POST ? 4 : 3;   // dw, db, A, B
  constexpr int kStages = ring_stages<T>();
  constexpr bool RING = J == 1 && (VEC || sizeof(T) == 4), AHEAD = J == 1 && !RING;
  // ring: stage, array (dn, h, branch, dh), column group; a thread's 16 bytes (two of them
  // for fp32) beside the next thread's
  constexpr int PIECES = sizeof(T) / 2;
  constexpr int STAGE16 = 4 * J * PIECES * THREADS, RING16 = RING ? kStages * STAGE16 : 0;
  // totals of dpw and dpb, then the sums (SMEM_ACC) or the buffer in which the workers add
  // theirs: pair q of a thread beside the next thread's
  Pair* const tot = reinterpret_cast<Pair*>(dyn4 + RING16) + threadIdx.x;
  Pair* const dyn = tot + (POST ? 2 * Q * THREADS : 0);
  pdl_enter();
  const int tpr = TPR > 32 ? a.tpr : TPR;
  const int rg = threadIdx.x / tpr, t = threadIdx.x - rg * tpr;
  const int nw = tpr / 32, warp0 = rg * nw, bar = 1 + rg;
  const int D = a.D;
  const float inv = 1.f / D;
  const bool read_y = POST || a.gate, per_row = a.gate && a.group_rows == 1;
  const int workers = gridDim.x * a.rows_per_cta, seg_rows = (int)a.seg_rows;
  long long seg = (long long)blockIdx.x * a.rows_per_cta + rg;
  int slot = 0;
  // VEC: a thread has eight columns of a group or none
  bool on[J];
#pragma unroll
  for (int j = 0; j < J; ++j) on[j] = Cols<VEC>(t, tpr, j, D).count > 0;

  [[maybe_unused]] Pair acc[SMEM_ACC ? 1 : NACC][SMEM_ACC ? 1 : Q];
  // sum i of pair q: acc + x y, acc + x
  auto add_product = [&](int i, int q, Pair x, Pair y) {
    if constexpr (SMEM_ACC) dyn[(i * Q + q) * THREADS] = fma2(x, y, dyn[(i * Q + q) * THREADS]);
    else acc[i][q] = fma2(x, y, acc[i][q]);
  };
  auto add = [&](int i, int q, Pair x) {
    if constexpr (SMEM_ACC) dyn[(i * Q + q) * THREADS] = add2(x, dyn[(i * Q + q) * THREADS]);
    else acc[i][q] = add2(x, acc[i][q]);
  };
  if constexpr (SMEM_ACC) {
    for (int i = 0; i < NACC * Q; ++i) dyn[i * THREADS] = 0;
  } else {
#pragma unroll
    for (int i = 0; i < NACC; ++i)
#pragma unroll
      for (int q = 0; q < Q; ++q) acc[i][q] = 0;
  }
  if (POST) {
    for (int i = 0; i < 2 * Q; ++i) tot[i * THREADS] = 0;
  }
  // of a column group: the pre norm's weights and gp = g pw (g without a post norm), in
  // registers, or (SMEM_ACC) read anew
  Pair w[4], gp[4];
  auto vector = [&](const void* p, int j, Pair* out) {
    float v[8];
    read_weight<VEC>(p, a.w_bf16, Cols<VEC>(t, tpr, j, D), v);
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = pair(v[2 * i], v[2 * i + 1]);
  };
  auto gate_row = [&](int j, long long i, bool live, Pair* g) {   // row i of the gate
    Raw8<T> r;
    read8<VEC>(static_cast<const T*>(a.gate) + (live ? i * D : 0), Cols<VEC>(t, tpr, j, D), live, r);
    widen2(r, g);
  };
  auto gates = [&](int j, long long i, bool live) {
#pragma unroll
    for (int e = 0; e < 4; ++e) gp[e] = both(1.f);
    if (POST) vector(a.post_weight, j, gp);
    if (a.gate) {
      Pair g[4];
      gate_row(j, i, live, g);
#pragma unroll
      for (int e = 0; e < 4; ++e) gp[e] = mul2(gp[e], g[e]);
    }
  };
  if (!SMEM_ACC) vector(a.weight, 0, w);

  // segment `s` covers rows [first, end)
  auto bounds = [&](long long s, int& first, int& end) {
    const long long grp = s / a.segs_per_group, k = s - grp * a.segs_per_group;
    first = (int)(grp * a.seg_group_rows + k * a.seg_rows);
    end = (int)min((long long)first + a.seg_rows, (grp + 1) * a.seg_group_rows);
    if (s >= a.nseg) first = end = 0;
  };
  const T* const src[4] = {static_cast<const T*>(a.dn), static_cast<const T*>(a.h),
                           read_y ? static_cast<const T*>(a.branch) : nullptr,
                           static_cast<const T*>(a.dh)};
  // what is not read, and columns past the row, stay zero from here on
  Raw8<T> next[AHEAD ? 4 : 1];
  auto place = [&](float4* stage, int x, int j, int piece) {
    return stage + ((x * J + j) * PIECES + piece) * THREADS;
  };
  float4* const ring0 = dyn4 + threadIdx.x;
  if constexpr (RING) {
    for (int i = 0; i < kStages * 4 * J * PIECES; ++i) ring0[i * THREADS] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  auto request = [&](float4* stage, int row, bool live) {
    const Cols<VEC> c(t, tpr, 0, D);
    const long long at = live ? (long long)row * D : 0;
    if constexpr (RING) {
      if (live) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (src[x] == nullptr || !on[0]) continue;
          const T* p = src[x] + at + c.first;
          if (VEC) {
#pragma unroll
            for (int q = 0; q < PIECES; ++q) copy_async16(place(stage, x, 0, q), p + q * (16 / sizeof(T)));
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e < c.count)
                copy_async4(reinterpret_cast<float*>(place(stage, x, 0, e / 4)) + (e & 3),
                            p + (long)e * c.step);
          }
        }
      } else {   // past the segment: a row of zeros adds nothing
        for (int i = 0; i < 4 * PIECES; ++i) stage[i * THREADS] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      copy_commit();
    } else if constexpr (AHEAD) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (src[x]) read8<VEC>(src[x] + at, c, live, next[AHEAD ? x : 0]);
        else zero(next[AHEAD ? x : 0]);
      }
    } else if (live) {   // into L2 meanwhile: one request a line of 128 bytes
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int per = 128 / (int)sizeof(T);
        if (src[x])
          for (int i = t * per; i < D; i += tpr * per)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(src[x] + at + i));
      }
    }
  };
  auto take = [&](float4* stage, int x, int j, int row, bool live, Pair* p) {
    Raw8<T> r;
    if constexpr (AHEAD) r = next[x];
    else if constexpr (!RING) {
      if (src[x]) read8<VEC>(src[x] + (live ? (long long)row * D : 0), Cols<VEC>(t, tpr, j, D), live, r);
      else zero(r);
    } else if constexpr (sizeof(T) == 2) r.a = *reinterpret_cast<const uint4*>(place(stage, x, j, 0));
    else {
      r.a = *place(stage, x, j, 0);
      r.b = *place(stage, x, j, PIECES - 1);
    }
    widen2(r, p);
  };

  // every worker makes the same number of turns (a.turns segments of a.seg_rows rows):
  // lanes of a warp that belong to different workers stay together.  ahead_*: the next
  // row to be requested
  int first, end, ahead_row, ahead_end, ahead_left = seg_rows, ahead_turn = 1;
  float4 *in = ring0, *out_stage = ring0;
  bounds(seg, first, end);
  ahead_row = first;
  ahead_end = end;
  const long long seg0 = seg;
  auto advance = [&] {
    request(in, ahead_row, ahead_row < ahead_end);
    in = in == ring0 + (kStages - 1) * STAGE16 ? ring0 : in + STAGE16;
    ++ahead_row;
    if (--ahead_left == 0) {
      ahead_left = seg_rows;
      if (ahead_turn < a.turns) bounds(seg0 + (long long)ahead_turn * workers, ahead_row, ahead_end);
      else ahead_end = 0;
      ++ahead_turn;
    }
  };
  if constexpr (RING) {
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) advance();
  } else {
    advance();
  }
  for (int turn = 0; turn < a.turns; ++turn) {
    if (!SMEM_ACC && !per_row) gates(0, seg / a.segs_per_group, first < end);
    for (int k = 0; k < seg_rows; ++k) {
      const int row = first + k;
      const bool live = row < end;
      Pair dn[Q], y[Q], h[Q];
      if constexpr (RING) copy_wait<kStages - 2>();
      float4* const stage = out_stage;
      out_stage = out_stage == ring0 + (kStages - 1) * STAGE16 ? ring0 : out_stage + STAGE16;
      Pair ds[Q];   // dh, then the sum's gradient, then dz, then dy
#pragma unroll
      for (int j = 0; j < J; ++j) {
        take(stage, 0, j, row, live, dn + 4 * j);
        take(stage, 1, j, row, live, h + 4 * j);
        take(stage, 2, j, row, live, y + 4 * j);
        if constexpr (AHEAD) take(stage, 3, j, row, live, ds + 4 * j);
      }
      if (!SMEM_ACC && per_row) gates(0, row, live);
      advance();
      float mh = 0.f, my = 0.f;
      if (a.layer) {
        Pair sh_ = 0, sy = 0;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          sh_ = add2(sh_, h[q]);
          if (POST) sy = add2(sy, y[q]);
        }
        if (POST) {
          float s[2] = {fold(sh_), fold(sy)};
          row_sums<TPR, 2>(s, sh, slot, warp0, nw, bar);
          mh = s[0] * inv;
          my = s[1] * inv;
        } else {
          float s[1] = {fold(sh_)};
          row_sums<TPR, 1>(s, sh, slot, warp0, nw, bar);
          mh = s[0] * inv;
        }
      }
      // the squares, and the sums of e = dn w and e (h - mean)
      Pair p[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const Cols<VEC> c(t, tpr, j, D);
        const Pair mhj = both(on[j] ? -mh : 0.f), myj = both(on[j] ? -my : 0.f);
        if (SMEM_ACC) vector(a.weight, j, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int q = 4 * j + i;
          h[q] = add2(h[q], mhj);
          if (POST) y[q] = add2(y[q], myj);
          if (!VEC) {
            float u, v;
            split(h[q], u, v);
            h[q] = pair(2 * i < c.count ? u : 0.f, 2 * i + 1 < c.count ? v : 0.f);
            split(y[q], u, v);
            y[q] = pair(2 * i < c.count ? u : 0.f, 2 * i + 1 < c.count ? v : 0.f);
          }
          const Pair d = mul2(dn[q], w[i]);
          p[0] = fma2(h[q], h[q], p[0]);
          if (POST) p[1] = fma2(y[q], y[q], p[1]);
          p[2] = add2(p[2], d);
          p[3] = fma2(d, h[q], p[3]);
        }
      }
      float s[4] = {fold(p[0]), fold(p[1]), fold(p[2]), fold(p[3])};
      row_sums<TPR, 4>(s, sh, slot, warp0, nw, bar);
      const float rh = live ? rsqrtf(s[0] * inv + a.eps) : 0.f;
      const float ry = POST && live ? rsqrtf(s[1] * inv + a.eps) : 0.f;
      const Pair rh2 = both(rh), ry2 = both(ry), alpha = both(a.alpha);
      const Pair c1 = both(a.layer ? -rh * s[2] * inv : 0.f), c2 = both(-rh * rh * s[3] * inv);
      Pair b0 = 0, b1 = 0;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        Pair out[4];
        const Cols<VEC> c(t, tpr, j, D);
        if constexpr (!AHEAD) take(stage, 3, j, row, live, ds + 4 * j);
        if (SMEM_ACC) {
          vector(a.weight, j, w);
          gates(j, per_row ? row : seg / a.segs_per_group, live);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int q = 4 * j + i;
          const Pair hh = mul2(h[q], rh2);
          ds[q] = add2(ds[q], fma2(rh2, mul2(w[i], dn[q]), fma2(hh, c2, c1)));
          add_product(0, q, dn[q], hh);
          add(1, q, dn[q]);
          out[i] = mul2(alpha, ds[q]);
          add_product(2, q, ds[q], POST ? mul2(y[q], ry2) : y[q]);
          if (POST) add(POST ? 3 : 0, q, ds[q]);
          ds[q] = mul2(ds[q], gp[i]);
          if (POST) {
            b0 = add2(b0, ds[q]);
            b1 = fma2(ds[q], y[q], b1);
          }
        }
        if (live && a.dx) write8<VEC>(static_cast<T*>(a.dx) + (long long)row * D, c, out);
      }
      if (POST) {
        float b[2] = {fold(b0), fold(b1)};
        row_sums<TPR, 2>(b, sh, slot, warp0, nw, bar);
        const Pair d1 = both(a.layer ? -ry * b[0] * inv : 0.f), d2 = both(-ry * ry * ry * b[1] * inv);
#pragma unroll
        for (int q = 0; q < Q; ++q) ds[q] = fma2(ry2, ds[q], fma2(y[q], d2, d1));
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const Cols<VEC> c(t, tpr, j, D);
        if (live) write8<VEC>(static_cast<T*>(a.dbranch) + (long long)row * D, c, ds + 4 * j);
      }
      // A and B of this row's gate, or of the segment's that ends here
      if (per_row || k + 1 == seg_rows) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Cols<VEC> c(t, tpr, j, D);
          Pair s0[4], s1[4], v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            constexpr int kB = POST ? 3 : 0;
            if constexpr (SMEM_ACC) {
              s0[i] = dyn[(2 * Q + 4 * j + i) * THREADS];
              s1[i] = POST ? dyn[(kB * Q + 4 * j + i) * THREADS] : 0;
              dyn[(2 * Q + 4 * j + i) * THREADS] = 0;
              if (POST) dyn[(kB * Q + 4 * j + i) * THREADS] = 0;
            } else {
              s0[i] = acc[2][i];
              s1[i] = POST ? acc[kB][i] : 0;
              acc[2][i] = 0;
              if (POST) acc[kB][i] = 0;
            }
            v[i] = both(1.f);
          }
          if (a.gate)
            gate_row(j, per_row ? row : seg / a.segs_per_group, per_row ? live : seg < a.nseg, v);
          if (POST) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              tot[(4 * j + i) * THREADS] = fma2(v[i], s0[i], tot[(4 * j + i) * THREADS]);
              tot[(Q + 4 * j + i) * THREADS] = fma2(v[i], s1[i], tot[(Q + 4 * j + i) * THREADS]);
            }
          }
          if (!a.dgate) continue;
          if (POST) {
            vector(a.post_weight, j, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) s0[i] = mul2(s0[i], v[i]);
            if (a.post_bias) {
              vector(a.post_bias, j, v);
#pragma unroll
              for (int i = 0; i < 4; ++i) s0[i] = fma2(v[i], s1[i], s0[i]);
            }
          }
          if (per_row) {
            if (live) write8<VEC>(static_cast<T*>(a.dgate) + (long long)row * D, c, s0);
          } else if (seg < a.nseg) {
            if (a.segs_per_group == 1) write8<VEC>(static_cast<T*>(a.dgate) + seg * D, c, s0);
            else write8<VEC>(a.gate_part + seg * D, c, s0);
          }
        }
      }
    }
    seg += workers;
    bounds(seg, first, end);
  }
  if constexpr (RING) copy_wait<0>();
  // the CTA's sums (dw, db, dpw, dpb): its workers' added through shared memory
  const int last = POST ? 4 : 2;
#pragma unroll
  for (int i = 0; i < last; ++i) {
    if (!(a.wanted >> i & 1)) continue;
    float* part = a.part + ((long long)blockIdx.x * 4 + i) * D;
    // where vector i of this CTA's threads lies
    const Pair* at = i >= 2 ? tot + (i - 2) * Q * THREADS : SMEM_ACC ? dyn + i * Q * THREADS : dyn;
    __syncthreads();
    if constexpr (!SMEM_ACC) {
      if (i < 2) {
#pragma unroll
        for (int q = 0; q < 4; ++q) dyn[q * THREADS] = acc[i < 2 ? i : 0][q];
        __syncthreads();
      }
    }
    if (rg == 0) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        Pair v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          v[q] = at[(4 * j + q) * THREADS];
          for (int k = 1; k < a.rows_per_cta; ++k) v[q] = add2(v[q], at[(4 * j + q) * THREADS + k * tpr]);
        }
        write8<VEC>(part, Cols<VEC>(t, tpr, j, D), v);
      }
    }
  }
}

namespace {

// Shared memory of a launch: the ring, the totals, and the sums (SMEM_ACC) or the buffer
// in which a CTA's workers add theirs.
template <class T, int J, bool VEC, bool POST, int THREADS>
constexpr int bwd_smem() {
  return (J == 1 && (VEC || sizeof(T) == 4) ? ring_stages<T>() * 4 * (int)sizeof(T) / 2 * THREADS * 16 : 0) +
         (POST ? 2 * 8 * J * THREADS * 4 : 0) + (J > 1 ? (POST ? 4 : 3) * 8 * J : 8) * THREADS * 4;
}
template <class T, int TPR, int J, bool VEC, bool POST, int THREADS, int CTAS>
cudaError_t bwd_launch(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  static std::atomic<unsigned long long> done{0};
  constexpr int smem = bwd_smem<T, J, VEC, POST, THREADS>();
  static_assert(smem <= 227 * 1024 - (int)sizeof(RowShared), "");
  auto k = norm_bwd_kernel<T, TPR, J, VEC, POST, THREADS, CTAS>;
  if (smem > 40960) {
    cudaError_t e = smem_opt_in(k, smem, &done);
    if (e != cudaSuccess) return e;
  }
  return launch_k(k, dim3(pl.ctas), dim3(pl.threads), smem, lc.stream, a);
}
template <class T, int TPR, int J, bool POST, int THREADS, int CTAS>
cudaError_t bwd_shape(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  return a.D % 8 == 0 ? bwd_launch<T, TPR, J, true, POST, THREADS, CTAS>(lc, a, pl)
                      : bwd_launch<T, TPR, J, false, POST, THREADS, CTAS>(lc, a, pl);
}
template <class T, bool POST>
cudaError_t bwd_typed(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  if (pl.tpr == 16) return bwd_shape<T, 16, 1, POST, 256, 2>(lc, a, pl);
  if (pl.tpr == 32) return bwd_shape<T, 32, 1, POST, 256, 2>(lc, a, pl);
  if (pl.wide) return bwd_shape<T, 64, 2, POST, 512, 1>(lc, a, pl);
  if (pl.threads > 256) return bwd_shape<T, 64, 1, POST, 512, 1>(lc, a, pl);
  return bwd_shape<T, 64, 1, POST, 256, 2>(lc, a, pl);
}

}  // namespace

}  // namespace bcmt
