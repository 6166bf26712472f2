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
  constexpr int E = 8 * J;
  constexpr bool SMEM_ACC = J > 1;
  constexpr bool RING = J == 1 && (VEC || sizeof(T) == 4), AHEAD = J == 1 && !RING;
  constexpr int NACC = POST ? 4 : 3;   // dw, db, A, B
  constexpr int kStages = ring_stages<T>();
  // ring: stage, array (dn, h, branch, dh), column group; a thread's 16 bytes (two of them
  // for fp32) beside the next thread's
  constexpr int PIECES = sizeof(T) / 2;
  constexpr int RING16 = RING ? kStages * 4 * J * PIECES * THREADS : 0;
  // totals of dpw and dpb, then the sums (SMEM_ACC) or the buffer in which the workers add
  // theirs: value e of a thread beside the next thread's
  float* const tot = reinterpret_cast<float*>(dyn4 + RING16);
  float* const dyn = tot + (POST ? 2 * E * THREADS : 0);
  pdl_enter();
  const int tpr = TPR > 32 ? a.tpr : TPR;
  const int rg = threadIdx.x / tpr, t = threadIdx.x - rg * tpr;
  const int nw = tpr / 32, warp0 = rg * nw, bar = 1 + rg;
  const int D = a.D;
  const float inv = 1.f / D;
  const bool read_y = POST || a.gate, per_row = a.gate && a.group_rows == 1;
  const long long workers = (long long)gridDim.x * a.rows_per_cta;
  long long seg = (long long)blockIdx.x * a.rows_per_cta + rg;
  int slot = 0;
  // VEC: a thread has eight columns of a group or none
  bool on[J];
#pragma unroll
  for (int j = 0; j < J; ++j) on[j] = Cols<VEC>(t, tpr, j, D).count > 0;

  [[maybe_unused]] float acc[SMEM_ACC ? 1 : NACC][SMEM_ACC ? 1 : E];
  auto add = [&](int i, int e, float v) {
    if constexpr (SMEM_ACC) dyn[(i * E + e) * THREADS + threadIdx.x] += v;
    else acc[i][e] += v;
  };
  if constexpr (SMEM_ACC) {
    for (int i = 0; i < NACC * E; ++i) dyn[i * THREADS + threadIdx.x] = 0.f;
  } else {
#pragma unroll
    for (int i = 0; i < NACC; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[i][e] = 0.f;
  }
  if (POST) {
    for (int i = 0; i < 2 * E; ++i) tot[i * THREADS + threadIdx.x] = 0.f;
  }
  // of a column group: the pre norm's weights and gp = g pw (g without a post norm), in
  // registers, or (SMEM_ACC) read anew
  float w[8], gp[8];
  auto weights = [&](int j) { read_weight<VEC>(a.weight, a.w_bf16, Cols<VEC>(t, tpr, j, D), w); };
  auto gate_row = [&](int j, long long i, bool live, float* g) {   // row i of the gate
    Raw8<T> r;
    read8<VEC>(static_cast<const T*>(a.gate) + (live ? i * D : 0), Cols<VEC>(t, tpr, j, D), live, r);
    widen(r, g);
  };
  auto gates = [&](int j, long long i, bool live) {
#pragma unroll
    for (int e = 0; e < 8; ++e) gp[e] = 1.f;
    if (POST) read_weight<VEC>(a.post_weight, a.w_bf16, Cols<VEC>(t, tpr, j, D), gp);
    if (a.gate) {
      float g[8];
      gate_row(j, i, live, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) gp[e] *= g[e];
    }
  };
  if (!SMEM_ACC) weights(0);

  // segment `s` covers rows [first, end)
  auto bounds = [&](long long s, long long& first, long long& end) {
    const long long grp = s / a.segs_per_group, k = s - grp * a.segs_per_group;
    first = grp * a.seg_group_rows + k * a.seg_rows;
    end = min(first + a.seg_rows, (grp + 1) * a.seg_group_rows);
    if (s >= a.nseg || first > end) end = first;
  };
  const T* const src[4] = {static_cast<const T*>(a.dn), static_cast<const T*>(a.h),
                           read_y ? static_cast<const T*>(a.branch) : nullptr,
                           static_cast<const T*>(a.dh)};
  // what is not read, and columns past the row, stay zero from here on
  Raw8<T> next[AHEAD ? 4 : 1];
  auto place = [&](int stage, int x, int j, int piece) {
    return dyn4 + (((stage * 4 + x) * J + j) * PIECES + piece) * THREADS + threadIdx.x;
  };
  if constexpr (RING) {
    for (int i = 0; i < kStages * 4 * J * PIECES; ++i)
      dyn4[i * THREADS + threadIdx.x] = make_float4(0.f, 0.f, 0.f, 0.f);
  }
  auto request = [&](int stage, long long row, bool live) {
    if constexpr (RING) {
      if (live) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if (src[x] == nullptr) continue;
#pragma unroll
          for (int j = 0; j < J; ++j) {
            const Cols<VEC> c(t, tpr, j, D);
            const T* p = src[x] + row * D + c.first;
            if (VEC) {
              if (on[j]) {
#pragma unroll
                for (int q = 0; q < PIECES; ++q)
                  copy_async16(place(stage, x, j, q), p + q * (16 / sizeof(T)));
              }
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (e < c.count)
                  copy_async4(reinterpret_cast<float*>(place(stage, x, j, e / 4)) + (e & 3),
                              p + (long)e * c.step);
            }
          }
        }
      } else {   // past the segment: a row of zeros adds nothing
#pragma unroll
        for (int i = 0; i < 4 * J * PIECES; ++i)
          *place(stage, i / (J * PIECES), i / PIECES % J, i % PIECES) = make_float4(0.f, 0.f, 0.f, 0.f);
      }
      copy_commit();
    } else if constexpr (AHEAD) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const Cols<VEC> c(t, tpr, 0, D);
        if (src[x]) read8<VEC>(src[x] + (live ? row * D : 0), c, live, next[AHEAD ? x : 0]);
        else zero(next[AHEAD ? x : 0]);
      }
    } else if (live) {   // into L2 meanwhile: one request a line of 128 bytes
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int per = 128 / (int)sizeof(T);
        if (src[x])
          for (int i = t * per; i < D; i += tpr * per)
            asm volatile("prefetch.global.L2 [%0];" ::"l"(src[x] + row * D + i));
      }
    }
  };
  auto take = [&](int stage, int x, int j, long long row, bool live, float* v) {
    Raw8<T> r;
    if constexpr (AHEAD) r = next[x];
    else if constexpr (!RING) {
      if (src[x]) read8<VEC>(src[x] + (live ? row * D : 0), Cols<VEC>(t, tpr, j, D), live, r);
      else zero(r);
    } else if constexpr (sizeof(T) == 2) r.a = *reinterpret_cast<const uint4*>(place(stage, x, j, 0));
    else {
      r.a = *place(stage, x, j, 0);
      r.b = *place(stage, x, j, PIECES - 1);
    }
    widen(r, v);
  };

  // every worker makes the same number of turns (a.turns segments of a.seg_rows rows):
  // lanes of a warp that belong to different workers stay together.  ahead_*: the next
  // row to be requested
  long long first, end, ahead_first, ahead_end, ahead_k = 0;
  int ahead_turn = 0, in = 0, out_stage = 0;
  bounds(seg, first, end);
  ahead_first = first;
  ahead_end = end;
  const long long seg0 = seg;
  auto advance = [&] {
    const long long row = ahead_first + ahead_k;
    request(in, row, ahead_turn < a.turns && row < ahead_end);
    in = in + 1 == kStages ? 0 : in + 1;
    if (++ahead_k == a.seg_rows) {
      ahead_k = 0;
      ++ahead_turn;
      bounds(seg0 + ahead_turn * workers, ahead_first, ahead_end);
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
    for (long long k = 0; k < a.seg_rows; ++k) {
      const long long row = first + k;
      const bool live = row < end;
      float dn[E], y[E], h[E];
      if constexpr (RING) copy_wait<kStages - 2>();
      const int stage = out_stage;
      out_stage = out_stage + 1 == kStages ? 0 : out_stage + 1;
      float ds[E];   // dh, then the sum's gradient, then dz, then dy
#pragma unroll
      for (int j = 0; j < J; ++j) {
        take(stage, 0, j, row, live, dn + 8 * j);
        take(stage, 1, j, row, live, h + 8 * j);
        take(stage, 2, j, row, live, y + 8 * j);
        if constexpr (AHEAD) take(stage, 3, j, row, live, ds + 8 * j);
      }
      if (!SMEM_ACC && per_row) gates(0, row, live);
      advance();
      float mh = 0.f, my = 0.f;
      if (a.layer) {
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < E; ++e) {
          s[0] += h[e];
          if (POST) s[1] += y[e];
        }
        if (POST) {
          row_sums<TPR, 2>(s, sh, slot, warp0, nw, bar);
          my = s[1] * inv;
        } else {
          float s1[1] = {s[0]};
          row_sums<TPR, 1>(s1, sh, slot, warp0, nw, bar);
          s[0] = s1[0];
        }
        mh = s[0] * inv;
      }
      // the squares, and the sums of e = dn w and e (h - mean)
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const Cols<VEC> c(t, tpr, j, D);
        const float mhj = on[j] ? mh : 0.f, myj = on[j] ? my : 0.f;
        if (SMEM_ACC) weights(j);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = 8 * j + i;
          h[e] -= mhj;
          if (POST) y[e] -= myj;
          if (!VEC && i >= c.count) h[e] = y[e] = 0.f;
          const float d = dn[e] * w[i];
          s[0] = fmaf(h[e], h[e], s[0]);
          if (POST) s[1] = fmaf(y[e], y[e], s[1]);
          s[2] += d;
          s[3] = fmaf(d, h[e], s[3]);
        }
      }
      row_sums<TPR, 4>(s, sh, slot, warp0, nw, bar);
      const float rh = live ? 1.f / sqrtf(s[0] * inv + a.eps) : 0.f;
      const float ry = POST && live ? 1.f / sqrtf(s[1] * inv + a.eps) : 0.f;
      const float c1 = a.layer ? rh * s[2] * inv : 0.f;
      const float c2 = rh * rh * s[3] * inv;
      float b[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < J; ++j) {
        float out[8];
        const Cols<VEC> c(t, tpr, j, D);
        if constexpr (!AHEAD) take(stage, 3, j, row, live, ds + 8 * j);
        if (SMEM_ACC) {
          weights(j);
          gates(j, per_row ? row : seg / a.segs_per_group, live);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = 8 * j + i;
          const float hh = h[e] * rh;
          ds[e] += fmaf(rh, w[i] * dn[e], -fmaf(hh, c2, c1));
          add(0, e, dn[e] * hh);
          add(1, e, dn[e]);
          out[i] = a.alpha * ds[e];
          add(2, e, ds[e] * (POST ? y[e] * ry : y[e]));
          if (POST) add(POST ? 3 : 0, e, ds[e]);
          ds[e] *= gp[i];
          if (POST) {
            b[0] += ds[e];
            b[1] = fmaf(ds[e], y[e], b[1]);
          }
        }
        if (live && a.dx) write8<VEC>(static_cast<T*>(a.dx) + row * D, c, out);
      }
      if (POST) {
        row_sums<TPR, 2>(b, sh, slot, warp0, nw, bar);
        const float d1 = a.layer ? ry * b[0] * inv : 0.f;
        const float d2 = ry * ry * ry * b[1] * inv;
#pragma unroll
        for (int e = 0; e < E; ++e) ds[e] = fmaf(ry, ds[e], -fmaf(y[e], d2, d1));
      }
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const Cols<VEC> c(t, tpr, j, D);
        if (live) write8<VEC>(static_cast<T*>(a.dbranch) + row * D, c, ds + 8 * j);
      }
      // A and B of this row's gate, or of the segment's that ends here
      if (per_row || k + 1 == a.seg_rows) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Cols<VEC> c(t, tpr, j, D);
          float s0[8], s1[8], v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if constexpr (SMEM_ACC) {
              float& f = dyn[(2 * E + 8 * j + e) * THREADS + threadIdx.x];
              s0[e] = f;
              f = s1[e] = 0.f;
              if (POST) {
                float& q = dyn[((POST ? 3 : 0) * E + 8 * j + e) * THREADS + threadIdx.x];
                s1[e] = q;
                q = 0.f;
              }
            } else {
              s0[e] = acc[2][e];
              s1[e] = POST ? acc[POST ? 3 : 0][e] : 0.f;
              acc[2][e] = 0.f;
              if (POST) acc[POST ? 3 : 0][e] = 0.f;
            }
          }
          if (a.gate) {
            gate_row(j, per_row ? row : seg / a.segs_per_group, live || !per_row ? seg < a.nseg : false, v);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 1.f;
          }
          if (POST) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              tot[(8 * j + e) * THREADS + threadIdx.x] += v[e] * s0[e];
              tot[(E + 8 * j + e) * THREADS + threadIdx.x] += v[e] * s1[e];
            }
          }
          if (!a.dgate) continue;
          if (POST) {
            read_weight<VEC>(a.post_weight, a.w_bf16, c, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) s0[e] *= v[e];
            if (a.post_bias) {
              read_weight<VEC>(a.post_bias, a.w_bf16, c, v);
#pragma unroll
              for (int e = 0; e < 8; ++e) s0[e] = fmaf(v[e], s1[e], s0[e]);
            }
          }
          if (per_row) {
            if (live) write8<VEC>(static_cast<T*>(a.dgate) + row * D, c, s0);
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
    if ((i & 1) && !a.layer) continue;
    float* part = a.part + ((long long)blockIdx.x * 4 + i) * D;
    // where vector i of this CTA's threads lies
    const float* at = i >= 2 ? tot + (i - 2) * E * THREADS : SMEM_ACC ? dyn + i * E * THREADS : dyn;
    __syncthreads();
    if constexpr (!SMEM_ACC) {
      if (i < 2) {
#pragma unroll
        for (int e = 0; e < 8; ++e) dyn[e * THREADS + threadIdx.x] = acc[i < 2 ? i : 0][e];
        __syncthreads();
      }
    }
    if (rg == 0) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = 0.f;
          for (int k = 0; k < a.rows_per_cta; ++k) v[e] += at[(8 * j + e) * THREADS + k * tpr + t];
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
