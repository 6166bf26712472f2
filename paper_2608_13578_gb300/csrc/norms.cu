// The end of a block of the language model and the norm before the next one:
//   z = post(y) or y,   h = alpha x + g z,   n = pre(h)
// over rows of D channels, and the gradients.  post and pre are layer norms
// (v - mean) r w + b with r = 1 / sqrt(mean (v - mean)^2 + eps), or root-mean-square
// norms (mean = 0); the gate g is a row of D channels for every group of consecutive
// rows (one for all, one per sequence, one per row), or absent.
//
// Backward, with hh = (h - mean) r the normalised rows and all means over a row:
//   e  = dn w,   s = dh + r (e - mean(e) - hh mean(e hh))          (the sum's gradient)
//   dx = alpha s,   dg = sum over the gate's rows of s z,   dz = g s
//   dy = r_y (dz pw - mean(dz pw) - yh mean(dz pw yh)),
//   dw = sum dn hh,  db = sum dn,  dpw = sum dz yh,  dpb = sum dz  (over the rows)
// (mean(e) and mean(dz pw) only in layer norms).  Both passes read each row once from
// global memory and take the mean first, then the squares around it.  Everything between
// the loads and the stores is fp32, rounded once to the stored type.
#include <algorithm>
#include <atomic>

#include "internal.h"
#include "norm_rows.cuh"
#include "norms.h"

namespace bcmt {

// Forward: a row belongs to TPR threads, each with J times eight of its columns; the row
// stays in registers between its loads and its stores.  Up to 1024 columns a row is one
// warp's, so that its sums need no barrier.  Bytes and the launch decide: 8192 x 512 bf16
// 7.2 us (5.1 at the copy's rate), 16384 x 768 fp32 36 us (30); in wide rows a CTA's loads wait for
// its sums, 8192 x 4096 59 us (40).  Few
// rows that are no multiples of 16 bytes, or short ones, go element by element (65000 x 201 bf16:
// 46 us, 16).
template <class T, int TPR, int J, bool VEC>
__global__ void __launch_bounds__(TPR > 128 ? TPR : 128) norm_fwd_kernel(const NormFwd a) {
  __shared__ RowShared sh;
  constexpr int E = 8 * J;
  pdl_enter();
  const int t = threadIdx.x % TPR;
  const long long row = (long long)blockIdx.x * (blockDim.x / TPR) + threadIdx.x / TPR;
  const bool live = row < a.rows;
  const int D = a.D, warp0 = (threadIdx.x / TPR) * (TPR / 32), bar = 1 + threadIdx.x / TPR;
  const long long at = (live ? row : 0) * D;
  int slot = 0;
  float z[E];
  Raw8<T> xr[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const Cols<VEC> c(t, TPR, j, D);
    Raw8<T> y;
    read8<VEC>(static_cast<const T*>(a.branch) + at, c, live, y);
    read8<VEC>(static_cast<const T*>(a.x) + at, c, live, xr[j]);
    widen(y, z + 8 * j);
  }
  const float inv = 1.f / D;
  // mean and 1 / deviation of the row in z
  auto stats = [&](float& mean, float& r) {
    mean = 0.f;
    if (a.layer) {
      float s[1] = {0.f};
#pragma unroll
      for (int e = 0; e < E; ++e) s[0] += z[e];
      row_sums<TPR, 1>(s, sh, slot, warp0, TPR / 32, bar);
      mean = s[0] * inv;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const Cols<VEC> c(t, TPR, j, D);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = z[8 * j + e] - mean;
        q[0] += e < c.count ? d * d : 0.f;
      }
    }
    row_sums<TPR, 1>(q, sh, slot, warp0, TPR / 32, bar);
    r = 1.f / sqrtf(q[0] * inv + a.eps);
  };
  float mean, r;
  if (a.post_weight) {
    stats(mean, r);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const Cols<VEC> c(t, TPR, j, D);
      float w[8], b[8] = {};
      read_weight<VEC>(a.post_weight, a.w_bf16, c, w);
      if (a.post_bias) read_weight<VEC>(a.post_bias, a.w_bf16, c, b);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[8 * j + e] = (z[8 * j + e] - mean) * r * w[e] + b[e];
    }
  }
  const T* gate = a.gate ? static_cast<const T*>(a.gate) + (live ? row : 0) / a.group_rows * D
                         : nullptr;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const Cols<VEC> c(t, TPR, j, D);
    float x[8];
    widen(xr[j], x);
    if (gate) {
      Raw8<T> gr;
      float g[8];
      read8<VEC>(gate, c, live, gr);
      widen(gr, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[8 * j + e] *= g[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) z[8 * j + e] = fmaf(a.alpha, x[e], z[8 * j + e]);
    if (live) write8<VEC>(static_cast<T*>(a.h) + at, c, z + 8 * j);
  }
  stats(mean, r);
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const Cols<VEC> c(t, TPR, j, D);
    float w[8], b[8] = {}, n[8];
    read_weight<VEC>(a.weight, a.w_bf16, c, w);
    if (a.bias) read_weight<VEC>(a.bias, a.w_bf16, c, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) n[e] = (z[8 * j + e] - mean) * r * w[e] + b[e];
    if (live) write8<VEC>(static_cast<T*>(a.n) + at, c, n);
  }
}

// Forward over many rows whose width is no multiple of 16 bytes: workers (one warp a row, or
// several) walk rows that come through a ring in shared memory as the 16-byte pieces that they
// lie in, as in the backward; the norms' weights, and the gate where all rows share it, stay in
// shared memory in fp32, so that an element costs one load of each array and a quarter of a
// load of each vector.  Issue slots decide in bf16, whose elements are half as wide: 16384 x 1001
// bf16 50 us (20 at the copy's rate; element by element from global memory 88), fp32 48 us (39;
// 60); 8192 x 4099 bf16 72 us (40; 162).
constexpr int kNormWalkJ = 2;   // groups of eight columns a lane: 72 registers, 24 warps
template <class T, int TPR>
__global__ void __launch_bounds__(kMaxWarps * 32, 1) norm_fwd_walk_kernel(const __grid_constant__ NormFwd a,
                                                              const __grid_constant__ NormWalk pl) {
  extern __shared__ float4 dyn4[];
  __shared__ RowShared sh;
  constexpr int J = kNormWalkJ, E = 8 * J, ES = sizeof(T);
  pdl_enter();
  const int tid = threadIdx.x, nt = blockDim.x, wt = TPR > 32 ? pl.tpr : 32, W = nt / wt;
  const int worker = tid / wt, t = tid - worker * wt, lane = tid & 31, wr = t >> 5;
  const int nw = wt / 32, warp0 = worker * nw, bar = 1 + worker, D = a.D, S = pl.stages;
  const float inv = 1.f / D;
  const int col0 = wr * 256 * J + lane;
  int slot = 0;
  auto columns = [&](int j) {
    const int first = col0 + 256 * j;
    return Cols<false>(first, 32, max(0, min(8, (D - first + 31) / 32)));
  };
  const int slot16 = (D * ES + 30) / 16;
  const uint32_t base = shared_address(dyn4), stage_bytes = 2 * slot16 * 16;
  const uint32_t ring = base + worker * S * stage_bytes, ring_end = ring + S * stage_bytes;
  // vectors: post weight, post bias, gate, weight, bias; a lane's 16 bytes beside the next one's
  constexpr int V = 2 * J * 512;
  const uint32_t vectors = base + W * S * stage_bytes + wr * 5 * V + lane * 16;
  const bool one = a.gate && a.group_rows >= a.rows;
  if (worker == 0) {
    const void* const src[5] = {a.post_weight, a.post_bias, one ? a.gate : nullptr, a.weight, a.bias};
#pragma unroll
    for (int i = 0; i < 5; ++i) {
#pragma unroll 1
      for (int j = 0; j < J; ++j) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = i == 0 || i == 2 ? 1.f : 0.f;
        if (src[i]) read_weight<false>(src[i], i == 2 ? ES == 2 : a.w_bf16, columns(j), v);
        store_shared(vectors + i * V + 2 * j * 512, pair(v[0], v[1]), pair(v[2], v[3]));
        store_shared(vectors + i * V + 2 * j * 512 + 512, pair(v[4], v[5]), pair(v[6], v[7]));
      }
    }
  }
  auto vector = [&](int i, int j, float* v) {
    Pair p[4];
    load_shared(vectors + i * V + 2 * j * 512, p[0], p[1]);
    load_shared(vectors + i * V + 2 * j * 512 + 512, p[2], p[3]);
#pragma unroll
    for (int e = 0; e < 4; ++e) split(p[e], v[2 * e], v[2 * e + 1]);
  };
  auto request = [&](uint32_t stage, long long row) {
    if (row < a.rows) {
      const long long all = a.rows * D * ES, from = row * D * ES, first = from & ~15ll;
      const int n = (int)((from - first) + D * ES + 15) / 16;
      const int left = (int)min((long long)n * 16, all - first);   // the last piece of all may be shorter
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const char* p = static_cast<const char*>(x ? a.x : a.branch) + first;
        for (int i = t; i < n; i += wt)
          copy_async16(stage + (x * slot16 + i) * 16, p + 16 * i, min(16, left - 16 * i));
      }
    }
    copy_commit();
  };
  auto take = [&](uint32_t stage, int x, int j, long long row, int count, float* v) {
    const uint32_t at = stage + x * slot16 * 16 + (uint32_t)((row * D * ES) & 15) + (col0 + 256 * j) * ES;
    if (count == 8) {   // all groups but a row's last
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = load_shared<T>(at + e * 32 * ES);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < count ? load_shared<T>(at + e * 32 * ES) : 0.f;
    }
  };
  auto put = [&](T* row, const Cols<false>& c, const float* v) {
    T* p = row + c.first;
    if (c.count == 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e * 32] = from_f<T>(v[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (e < c.count) p[e * 32] = from_f<T>(v[e]);
    }
  };
  const long long step = (long long)gridDim.x * W;
  long long row = (long long)blockIdx.x * W + worker, ahead = row;
  uint32_t in = ring, cur = ring;
  auto advance = [&] {
    request(in, ahead);
    ahead += step;
    in = in + stage_bytes == ring_end ? ring : in + stage_bytes;
  };
  for (int i = 0; i < S - 1; ++i) advance();
  __syncthreads();   // the vectors
  float z[E];
  auto stats = [&](float& mean, float& r) {
    mean = 0.f;
    if (a.layer) {
      float s[1] = {0.f};
#pragma unroll
      for (int e = 0; e < E; ++e) s[0] += z[e];
      row_sums<TPR, 1>(s, sh, slot, warp0, nw, bar);
      mean = s[0] * inv;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int count = columns(j).count;
      if (count == 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = z[8 * j + e] - mean;
          q[0] = fmaf(d, d, q[0]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = z[8 * j + e] - mean;
          q[0] += e < count ? d * d : 0.f;
        }
      }
    }
    row_sums<TPR, 1>(q, sh, slot, warp0, nw, bar);
    r = 1.f / sqrtf(q[0] * inv + a.eps);
  };
#pragma unroll 1
  for (; row < a.rows; row += step) {
    if (S > 2) copy_wait<1>();
    else copy_wait<0>();
    if (TPR > 32) bar_sync(bar, wt);   // others' copies are here, and have left the stage before
    else __syncwarp();
    advance();
    const uint32_t stage = cur;
    cur = cur + stage_bytes == ring_end ? ring : cur + stage_bytes;
    const long long at = row * D;
#pragma unroll
    for (int j = 0; j < J; ++j) take(stage, 0, j, row, columns(j).count, z + 8 * j);
    float mean, r;
    if (a.post_weight) stats(mean, r);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const Cols<false> c = columns(j);
      float v[8], u[8];
      if (a.post_weight) {
        vector(0, j, v);
        vector(1, j, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) z[8 * j + e] = (z[8 * j + e] - mean) * r * v[e] + u[e];
      }
      if (a.gate) {
        if (one) {
          vector(2, j, v);
        } else {
          Raw8<T> g;
          read8<false>(static_cast<const T*>(a.gate) + row / a.group_rows * D, c, true, g);
          widen(g, v);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) z[8 * j + e] *= v[e];
      }
      take(stage, 1, j, row, c.count, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) z[8 * j + e] = fmaf(a.alpha, v[e], z[8 * j + e]);
      put(static_cast<T*>(a.h) + at, c, z + 8 * j);
    }
    stats(mean, r);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      float v[8], u[8];
      vector(3, j, v);
      vector(4, j, u);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (z[8 * j + e] - mean) * r * v[e] + u[e];
      put(static_cast<T*>(a.n) + at, columns(j), v);
    }
  }
  copy_wait<0>();
}

// Sums of the CTAs' and segments' parts: blockIdx.y is one of the four vectors of weights
// (with one gate for all rows the last two are A and B), or 4 + a gate; a CTA adds 32
// columns with 16 lines of threads, each over every 16th part, then the lines in order.
// Latency decides (two dependent turns of loads, about 5 us after the backward); with 32 lines
// fewer CTAs fit beside one another and 16384 x 768 with 16 gates takes 49 us for 42.
__global__ void __launch_bounds__(512) norm_join_kernel(const NormJoin a) {
  __shared__ float s[16][33];
  pdl_enter();
  const int lane = threadIdx.x & 31, col = blockIdx.x * 32 + lane, line = threadIdx.x >> 5;
  const long long y = blockIdx.y + (long long)a.first;
  const bool one = a.mode == kGateOne;
  void* const out = y < 4 ? a.out[y] : a.dgate;
  if (!out) return;
  auto sum = [&](const float* in, long long n, long long stride) {   // in line 0
    float v = 0.f;
    if (col < a.D) {
      // ten loads at a time: the parts of up to 160 CTAs are one turn
      for (long long i = line; i < n; i += 160) {
        float u[10];
#pragma unroll
        for (int k = 0; k < 10; ++k) u[k] = i + 16 * k < n ? in[(i + 16 * k) * stride + col] : 0.f;
#pragma unroll
        for (int k = 0; k < 10; ++k) v += u[k];
      }
    }
    __syncthreads();
    s[line][lane] = v;
    __syncthreads();
    if (line == 0) {
#pragma unroll
      for (int i = 1; i < 16; ++i) v += s[i][lane];
    }
    return v;
  };
  auto part = [&](int i) { return sum(a.part + (long long)i * a.D, a.nparts, 4ll * a.D); };
  auto weight = [&](const void* w, bool is_bf16) {
    return is_bf16 ? to_f(static_cast<const bf16*>(w)[col]) : static_cast<const float*>(w)[col];
  };
  const bool on = line == 0 && col < a.D;
  float v;
  if (y < 4) {
    v = part((int)y);
    if (on && one && y >= 2) v *= weight(a.gate, a.t_bf16);
  } else if (one) {
    v = part(2);
    if (a.post_weight && on) v *= weight(a.post_weight, a.w_bf16);
    if (a.post_bias) {
      const float b = part(3);
      if (on) v = fmaf(weight(a.post_bias, a.w_bf16), b, v);
    }
  } else {
    v = sum(a.gate_part + (y - 4) * a.segs_per_group * a.D, a.segs_per_group, a.D);
  }
  if (!on) return;
  const long long at = y < 4 ? col : (y - 4) * a.D + col;
  if (y < 4 ? a.w_bf16 : a.t_bf16) static_cast<bf16*>(out)[at] = from_f<bf16>(v);
  else static_cast<float*>(out)[at] = v;
}

namespace {

template <class T, int TPR, int J>
cudaError_t fwd_shape(const Launch& lc, const NormFwd& a) {
  constexpr int threads = TPR > 128 ? TPR : 128, rows = threads / TPR;
  const dim3 grid((unsigned)((a.rows + rows - 1) / rows));
  return a.D % 8 == 0 ? launch_k(norm_fwd_kernel<T, TPR, J, true>, grid, dim3(threads), 0, lc.stream, a)
                      : launch_k(norm_fwd_kernel<T, TPR, J, false>, grid, dim3(threads), 0, lc.stream, a);
}
template <class T>
cudaError_t fwd_typed(const Launch& lc, const NormFwd& a) {
  if (a.D <= 128) return fwd_shape<T, 16, 1>(lc, a);
  if (a.D <= 256) return fwd_shape<T, 32, 1>(lc, a);
  if (a.D <= 512) return fwd_shape<T, 32, 2>(lc, a);
  if (a.D <= 1024) return fwd_shape<T, 32, 4>(lc, a);
  if (a.D <= 2048) return fwd_shape<T, 64, 4>(lc, a);
  if (a.D <= 4096) return fwd_shape<T, 128, 4>(lc, a);
  return fwd_shape<T, 256, 4>(lc, a);
}

template <class T, int TPR>
cudaError_t walk_launch(const Launch& lc, const NormFwd& a, const NormWalk& w) {
  static std::atomic<unsigned long long> done{0};
  auto k = norm_fwd_walk_kernel<T, TPR>;
  cudaError_t e = smem_opt_in(k, kNormSmem, &done);
  if (e != cudaSuccess) return e;
  return launch_k(k, dim3(w.ctas), dim3(w.threads), w.smem, lc.stream, a, w);
}

// Whether, and how, a forward call walks: rows that are no multiples of 16 bytes, at least four
// for every worker.  (Up to 256 channels a warp a row alone is quicker: 65000 x 201 bf16 46 us,
// walked 57.)
bool walk_plan(const NormFwd& a, int es, int sms, NormWalk& w) {
  if (a.D % 8 == 0 || a.D <= 256) return false;
  w.tpr = (a.D + 256 * kNormWalkJ - 1) / (256 * kNormWalkJ) * 32;
  for (int W = kMaxWarps * 32 / w.tpr; W >= 1; --W) {
    const int row = 2 * ((a.D * es + 30) / 16) * 16, vectors = 5 * 2 * kNormWalkJ * 16 * w.tpr;
    for (w.stages = 3; w.stages >= 2; --w.stages) {
      w.smem = W * w.stages * row + vectors;
      if (w.smem > kNormSmem) continue;
      w.threads = W * w.tpr;
      w.ctas = sms;
      return a.rows >= 4ll * W * sms;
    }
  }
  return false;
}
template <class T>
cudaError_t walk_typed(const Launch& lc, const NormFwd& a, const NormWalk& w) {
  return w.tpr == 32 ? walk_launch<T, 32>(lc, a, w) : walk_launch<T, 64>(lc, a, w);
}

}  // namespace

NormPlan norm_plan(long long rows, int D, int es, long long groups, bool post, int sms) {
  NormPlan p{};
  if (rows < 1) return p;
  p.mode = groups == 0 ? kGateNone : groups == rows ? kGateRows : groups == 1 ? kGateOne : kGateGroups;
  // threads of a row: 8, 16 or one warp of 8 J columns a lane, or the warps that cost least
  // by a count of instructions (190 a group of eight columns, 180 for the sums; spills and the
  // type are not in it).  Measured, 403 MB of layer-normed rows with a post norm and 16 gates, us
  // with J = 2 / 3 / 4 (from 3 on, rows of several warps spill):
  //   D      768      1024     1280         1536         2048         2560         2816         4096
  //   bf16   245/143  191/249  267/208/427  229/179/367  200/227/293  287/215/297  271/200/275  224/253/293
  //   fp32   207/215  211/248  214/231/342  208/223/318  211/233/293  222/271/356  227/263/344  231/273/328
  // The rule takes the faster side in bf16 but for 2560, where it takes two; in fp32 two are
  // faster at each, and it takes three at 768, 1280, 1536 and 2816.
  p.tpr = D <= 64 ? 8 : D <= 128 ? 16 : 32;
  p.J = 1;
  const int most = 16 / (post ? 2 : 1);
  for (int J = 2, best = 1 << 30; D > 256 && J <= 4; ++J) {
    const int n = (D + 256 * J - 1) / (256 * J), cost = n * (J * 190 + 180);
    // more than two groups take too many registers without the roles, four with them
    if (n <= most && cost < best && (J < 3 || (post && (J == 3 || best == 1 << 30)))) {
      best = cost;
      p.J = J;
      p.tpr = n * 32;
    }
  }
  const int R = p.tpr < 32 ? 32 / p.tpr : 1, wt = std::max(32, p.tpr), roles = post ? 2 : 1;
  // segments are of whole steps of R rows
  const long long g = p.mode == kGateGroups ? groups : 1, gr = rows / g, gs = (gr + R - 1) / R;
  const int arrays = p.mode == kGateRows ? 5 : 4;
  const bool vec = D % 8 == 0;
  // workers of a CTA: as many as there are steps for, registers and shared memory allow; the
  // rings are to hold the next step at least.  totals: whether workers walk several gates'
  // segments and keep totals of dpw and dpb over them
  auto cut = [&](bool totals) {
    p.gp_smem = p.mode != kGateRows && (post || p.mode != kGateNone);
    p.tot_smem = totals;
    p.pw_smem = post && p.mode == kGateRows;
    p.one_seg = !totals;
    long long W = norm_max_warps(p.J, p.tpr <= 32) * 32 / (wt * roles);
    W = std::max(1ll, std::min(W, (g * gs + sms - 1) / sms));
    auto size = [&](int stages, int slots) {   // whether it fits
      const long long nt = W * wt;
      p.stages = stages;
      p.ds_slots = slots;
      const long long stage16 = vec ? (long long)arrays * p.J * (es / 2) * nt
                                    : arrays * W * (((long long)R * D * es + 30) / 16);
      const long long rest16 = (p.pw_smem ? 6 : 2) * p.J * wt + (post ? slots * 2 * p.J * nt : 0) +
                               (p.gp_smem ? 2 * p.J * nt : 0) + (p.tot_smem ? 4 * p.J * nt : 0);
      // the CTA's sums go through the rings at the end
      p.ring16 = (int)std::max(stages * stage16, 2ll * p.J * nt * roles);
      p.smem = (int)(p.ring16 + rest16) * 16;
      return p.smem <= kNormSmem;
    };
    while (!size(2, 2) && W > 1) --W;
    if (p.smem <= kNormSmem) {
      if (!size(3, 2)) size(2, 2);
    } else if (!size(1, 2) && !size(2, 1) && !size(1, 1)) {
      p.tot_smem = p.pw_smem = false;
      size(1, 1);
    }
    p.threads = (int)(W * wt) * roles;
    p.ctas = (int)std::min<long long>((g * gs + W - 1) / W, sms);
    // each gate's steps in equal parts, so that the workers' longest walk is short; a gate for
    // all rows (or none): a segment a worker
    const long long workers = p.ctas * W;
    long long best = -1;
    for (long long turns = (g + workers - 1) / workers, i = 0; i < (totals ? 8 : 1); ++i, ++turns) {
      const long long s = std::min(gs, std::max(1ll, turns * workers / g)), len = (gs + s - 1) / s;
      if (best < 0 || turns * len < best) {
        best = turns * len;
        p.segs_per_group = (gs + len - 1) / len;
        p.seg_rows = len * R;
      }
    }
    // one segment a worker at most, the longest walk within an eighth of the mean
    return g * p.segs_per_group <= workers && best * workers * 8 <= g * gs * 9 + workers * 8;
  };
  if (!cut(false) && post && p.mode == kGateGroups) cut(true);
  p.seg_group_rows = gr;
  p.nseg = g * p.segs_per_group;
  p.part_bytes = (size_t)p.ctas * 4 * D * 4;
  p.gate_bytes = p.mode == kGateGroups && p.segs_per_group > 1 ? (size_t)p.nseg * D * 4 : 0;
  return p;
}

cudaError_t norm_forward(const Launch& lc, int dtype, const NormFwd& a, int sms) {
  if (a.rows == 0) return cudaSuccess;
  NormWalk w;
  if (walk_plan(a, dtype == 0 ? 4 : 2, sms, w))
    return dtype == 0 ? walk_typed<float>(lc, a, w) : walk_typed<bf16>(lc, a, w);
  return dtype == 0 ? fwd_typed<float>(lc, a) : fwd_typed<bf16>(lc, a);
}

cudaError_t norm_backward(const Launch& lc, int dtype, const NormPlan& pl, NormBwd a,
                          const NormJoin& j) {
  if (pl.ctas == 0) return cudaSuccess;
  a.tpr = pl.tpr;
  a.stages = pl.stages;
  a.mode = pl.mode;
  a.ring16 = pl.ring16;
  a.ds_slots = pl.ds_slots;
  a.gp_smem = pl.gp_smem;
  a.tot_smem = pl.tot_smem;
  a.pw_smem = pl.pw_smem;
  a.one_seg = pl.one_seg;
  if (pl.mode == kGateOne && a.dgate) a.wanted |= a.post_bias ? 12 : 4;
  a.seg_rows = pl.seg_rows;
  a.segs_per_group = pl.segs_per_group;
  a.seg_group_rows = pl.seg_group_rows;
  a.nseg = pl.nseg;
  // by type; without a post norm, with one, with one and a gate per row
  static constexpr decltype(&norms_bwd_f32) kCalls[2][3] = {
      {norms_bwd_f32, norms_bwd_f32_post, norms_bwd_f32_post_rows},
      {norms_bwd_bf16, norms_bwd_bf16_post, norms_bwd_bf16_post_rows}};
  cudaError_t e = kCalls[dtype != 0][a.post_weight ? 1 + (pl.mode == kGateRows) : 0](lc, a, pl);
  if (e != cudaSuccess) return e;
  // gates beyond the grid's second axis take further launches
  const long long gates = pl.mode == kGateOne ? 1 : pl.gate_bytes ? pl.nseg / pl.segs_per_group : 0;
  const long long all = (gates ? 4 + gates : a.post_weight ? 4 : 2);
  for (long long y = 0; y < all && e == cudaSuccess; y += 65535) {
    NormJoin q = j;
    q.first = y;
    q.nparts = pl.ctas;
    q.segs_per_group = pl.segs_per_group;
    q.mode = pl.mode;
    q.gate = a.gate;
    q.post_weight = a.post_weight;
    q.post_bias = a.post_bias;
    e = launch_k(norm_join_kernel, dim3((a.D + 31) / 32, (unsigned)std::min<long long>(65535, all - y)),
                 dim3(512), 0, lc.stream, q);
  }
  return e;
}

}  // namespace bcmt
