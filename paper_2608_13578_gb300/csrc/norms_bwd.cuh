// Backward of the norms around a block (the formulas are in norms.cu), for one type of
// rows.
#pragma once

#include <atomic>

#include "norm_rows.cuh"
#include "norms.h"

namespace bcmt {

// Backward.  A worker takes a row at a time (or 2 or 4 short ones) and walks segments of
// consecutive rows, each of one gate.  Its warps have two roles: the first takes dn, h and dh
// to the sum's gradient ds, with dx and the sums of dw and db; the second takes ds (through
// shared memory) and the branch to dbranch, with the sums for the post norm and the gate.
// Each so needs half the registers and has half the chain of sums over a row, and the second
// is a row behind the first.  Without a post norm the first role does it all.
//
// A thread's columns are the same in every row, so the columns' sums stay in its registers
// and reach global memory once per CTA, the gate's once per segment.  A lane has 8 J columns,
// up to 32: what a sum over a row costs is shared by more of them (a single warp with all of
// 1024 columns, 32 a lane, is slower than two: 4095 x 1001 fp32 57 us for 31).  Rows come through rings
// in shared memory by asynchronous copies.  VEC (16-byte rows): a thread copies its own
// columns to its own places and needs no barrier.  Else the role's threads copy the 16-byte
// pieces that a row lies in, and read elements.
//
// With A = sum ds yh and B = sum ds over the rows of one gate, its gradient is pw A + pb B,
// and it adds g A to dpw and g B to dpb: the sums take A and B, and what depends on the
// gate is done once for its segment (a gate for all rows: when the CTAs' sums are joined).
// A gate per row (ROWS) comes through the ring too, and the sums take g ds.
//
// What bounds it: the latency of a row's sums with 12 to 20 warps an SM (168 to 96 registers a
// thread), and issue slots (990 instructions for both roles of a row of 768).  Measured, both
// kernels of a call: 16384 x 768 bf16 40 us (22.7 at the copy's rate), 16384 x 4096 165 us (121), 4095 x 1001
// fp32 with a gate per row 31 us (20), 65536 x 64 18 us (7.6), 8192 x 8192 without a post norm
// 140 us (121), 8192 x 512 14 us (6.3), 16384 x 768 32 us (19).  One role with 8 columns a lane took 57, 211, 106 and 88 us for the first four.
enum { kRolePre, kRolePost, kRoleAll };

template <class T, int TPR, int J, bool VEC, bool ROWS, int ROLE>
__device__ __forceinline__ void norm_bwd_role(const NormBwd& a, float4* dyn4, RowShared& sh) {
  constexpr bool POST = ROLE != kRoleAll, LAST = ROLE != kRolePre;   // LAST: has the branch
  constexpr int Q = 4 * J;                         // pairs of columns of a thread
  constexpr int NACC = ROLE == kRoleAll ? 3 : 2;   // dw, db, A | A, B
  constexpr int ES = sizeof(T), PIECES = ES / 2;
  constexpr int R = TPR < 32 ? 32 / TPR : 1;       // rows of a worker at a time
  // arrays of the ring: dn, h, dh | branch (, gate) | dn, h, dh, branch (, gate)
  constexpr int NPRE = ROLE == kRolePost ? 0 : 3, NA = NPRE + (LAST ? 1 + ROWS : 0);
  constexpr int kBranch = NPRE, kGate = NPRE + 1;
  constexpr int kA = ROLE == kRoleAll ? 2 : 0;     // where A is
  constexpr bool KEEP = TPR == 32 || J <= (ROLE == kRolePre ? 3 : 2);   // a row stays in registers

  const int nt = POST ? blockDim.x / 2 : blockDim.x;   // threads of a role
  const int tid = threadIdx.x - (ROLE == kRolePost ? nt : 0);
  const int tpr = TPR > 32 ? a.tpr : TPR, wt = TPR > 32 ? tpr : 32;   // threads of a row, of a worker's role
  const int worker = tid / wt, in_worker = tid - worker * wt, W = nt / wt;
  const int sub = in_worker / tpr, t = in_worker - sub * tpr;
  const int nw = tpr / 32, warp0 = (threadIdx.x >> 5) - (in_worker >> 5);
  const int bar = 1 + worker + (ROLE == kRolePost ? W : 0);            // of the role's threads of a row
  const int handover = 1 + worker + (TPR > 32 ? 2 * W : 0);            // of the worker's two roles
  const int D = a.D, S = a.stages;
  const float inv = 1.f / D;
  const bool read_y = POST || ROWS || a.gate;
  const int workers = gridDim.x * W;
  int slot = 0;

  // columns: a warp has 256 J consecutive ones, in groups of 256
  const int wr = TPR > 32 ? in_worker >> 5 : 0, lane = tid & 31, wid = tid >> 5;
  const int col0 = wr * 256 * J + (VEC ? 8 : 1) * (TPR < 32 ? t : lane);
  constexpr int STEP = TPR < 32 ? TPR : 32;   // between a thread's columns of a group (not VEC)
  auto columns = [&](int j) {
    const int first = col0 + 256 * j;
    return Cols<VEC>(first, VEC ? 1 : STEP,
                     VEC ? (first < D ? 8 : 0) : max(0, min(8, (D - first + STEP - 1) / STEP)));
  };

  // shared memory (byte addresses): the rings; ds; the pre norm's weights (ROWS: and the post
  // norm's) for all workers; a thread's gp = g pw (g without a post norm) and totals of dpw
  // and dpb.  But for rings of pieces, each warp has a place of its own, with 16 bytes of a lane
  // beside the next lane's: all offsets in it are constants
  constexpr int STAGE = NA * J * PIECES * 512, G = 512, V = 2 * J * G;   // V: a vector of fp32
  const int nwarps = nt / 32;
  const int slot16 = VEC ? 0 : (R * D * ES + 30) / 16;    // of one array of one worker
  const uint32_t stage_bytes = VEC ? STAGE : NA * slot16 * 16;
  const uint32_t base = shared_address(dyn4);
  const uint32_t first_ring = S * 3 * (VEC ? J * PIECES * 512 * nwarps : slot16 * 16 * W);
  const uint32_t ring = base + (ROLE == kRolePost ? first_ring : 0) +
                        (VEC ? wid * S * STAGE + lane * 16 : worker * S * stage_bytes);
  const uint32_t dss = base + a.ring16 * 16 + wid * a.ds_slots * V + lane * 16;
  const uint32_t ws0 = base + a.ring16 * 16 + (POST ? nwarps * a.ds_slots * V : 0);
  const uint32_t ws = ws0 + wr * ((ROWS && a.pw_smem) ? 3 : 1) * V + lane * 16;
  const uint32_t gps0 = ws0 + (wt / 32) * ((ROWS && a.pw_smem) ? 3 : 1) * V;
  const uint32_t gps = gps0 + wid * V + lane * 16;
  const uint32_t tot0 = gps0 + (a.gp_smem ? nwarps * V : 0), tot = tot0 + wid * 2 * V + lane * 16;
  auto get2 = [](uint32_t p, Pair* v) {
    load_shared(p, v[0], v[1]);
    load_shared(p + G, v[2], v[3]);
  };
  auto put2 = [](uint32_t p, const Pair* v) {
    store_shared(p, v[0], v[1]);
    store_shared(p + G, v[2], v[3]);
  };
  auto vector = [&](const void* p, int j, Pair* out) {
    float v[8];
    read_weight<VEC>(p, a.w_bf16, columns(j), v);
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = pair(v[2 * i], v[2 * i + 1]);
  };
  auto gate_row = [&](int j, long long i, Pair* g) {   // row i of the gate
    Raw8<T> r;
    read8<VEC>(static_cast<const T*>(a.gate) + i * D, columns(j), true, r);
    widen2(r, g);
  };
  if (worker == 0) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      Pair v[4];
      if (ROLE != kRolePost) {
        vector(a.weight, j, v);
        put2(ws + 2 * j * G, v);
      } else if (ROWS && a.pw_smem) {
        vector(a.post_weight, j, v);
        put2(ws + V + 2 * j * G, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = 0;
        if (a.post_bias) vector(a.post_bias, j, v);
        put2(ws + 2 * V + 2 * j * G, v);
      }
    }
  }
  // gp where the gate changes by segments at most
  auto gates = [&](long long i) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      Pair v[4], g[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = both(1.f);
      if (POST) vector(a.post_weight, j, v);
      if (a.gate) {
        gate_row(j, i, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = mul2(v[e], g[e]);
      }
      put2(gps + 2 * j * G, v);
    }
  };
  if (ROLE == kRolePost && !ROWS && a.mode == kGateGroups && !a.one_seg) {
    const Pair z[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < J; ++j)
      for (int i = 0; i < 2; ++i) {
        if (a.tot_smem) put2(tot + i * V + 2 * j * G, z);
        else write8<VEC>(a.part + ((long long)blockIdx.x * 4 + 2 + i) * D, columns(j), z);
      }
  }

  Pair acc[NACC][Q];
#pragma unroll
  for (int i = 0; i < NACC; ++i)
#pragma unroll
    for (int q = 0; q < Q; ++q) acc[i][q] = 0;

  // segment `s` covers rows [first, end)
  auto bounds = [&](long long s, int& first, int& end) {
    if (s >= a.nseg) {
      first = end = 0;
      return;
    }
    const long long grp = s / a.segs_per_group, k = s - grp * a.segs_per_group;
    first = (int)(grp * a.seg_group_rows + k * a.seg_rows);
    end = (int)min((long long)first + a.seg_rows, (grp + 1) * a.seg_group_rows);
  };
  auto source = [&](int x) {
    return static_cast<const T*>(x >= NPRE ? x == kGate ? a.gate : read_y ? a.branch : nullptr
                                 : x == 0 ? a.dn : x == 1 ? a.h : a.dh);
  };
  // rows from `row` on into a stage (VEC: this thread's, zeros where it has none)
  auto request = [&](uint32_t stage, int row, int end) {
    if (VEC) {
      const bool live = R == 1 || row + sub < end;
      const long long at = (long long)(live ? row + sub : row) * D;
#pragma unroll
      for (int x = 0; x < NA; ++x) {
        if (source(x) == nullptr) continue;
        const T* p = source(x) + at;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Cols<VEC> c = columns(j);
          const bool on = live && c.count;
#pragma unroll
          for (int q = 0; q < PIECES; ++q)
            copy_async16(stage + ((x * J + j) * PIECES + q) * G, p + (on ? c.first + q * (16 / ES) : 0),
                         on ? 16 : 0);
        }
      }
    } else {
      const long long all = a.rows * D * ES, from = (long long)row * D * ES;
      const int rows = R == 1 ? 1 : min(R, end - row);
      const long long first = from & ~15ll;
      const int n = (int)((from - first) + rows * D * ES + 15) / 16;
      const int left = (int)min((long long)n * 16, all - first);   // the last piece of all may be shorter
#pragma unroll
      for (int x = 0; x < NA; ++x) {
        if (source(x) == nullptr) continue;
        const char* p = reinterpret_cast<const char*>(source(x)) + first;
        for (int i = in_worker; i < n; i += wt)
          copy_async16(stage + (x * slot16 + i) * 16, p + 16 * i, min(16, left - 16 * i));
      }
    }
  };
  // eight columns of array x in the stage that holds rows from `row` on (at byte `mis` of it)
  auto take = [&](uint32_t stage, int x, int j, uint32_t mis, int count, Pair* p) {
    if (VEC) {
      const uint32_t at = stage + (x * J + j) * PIECES * G;
      if (ES == 2) {
        Raw8<bf16> r;
        load_shared(at, r.a);
        widen2(r, p);
      } else {
        get2(at, p);
      }
    } else {
      const uint32_t at = stage + x * slot16 * 16 + mis + 256 * j * ES;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = e < count ? load_shared<T>(at + e * STEP * ES) : 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = pair(v[2 * i], v[2 * i + 1]);
    }
  };
  auto keep = [&](Pair v, int i, int count) {   // pair i of eight columns, zero past count
    if (VEC) return v;
    float x, y;
    split(v, x, y);
    return pair(2 * i < count ? x : 0.f, 2 * i + 1 < count ? y : 0.f);
  };
  auto sync_row = [&] {
    if (TPR > 32) bar_sync(bar, wt);
    else __syncwarp();
  };

  // the rows that are requested next, and where
  const long long seg0 = (long long)blockIdx.x * W + worker;
  long long ahead_seg = seg0;
  int ahead_row, ahead_end;
  uint32_t in = ring, cur = ring;
  const uint32_t ring_end = ring + S * stage_bytes;
  bounds(ahead_seg, ahead_row, ahead_end);
  auto advance = [&] {
    if (ahead_row < ahead_end) {
      request(in, ahead_row, ahead_end);
      ahead_row += R;
      if (ahead_row >= ahead_end) {
        ahead_seg += workers;
        bounds(ahead_seg, ahead_row, ahead_end);
      }
    }
    copy_commit();
    in = in + stage_bytes == ring_end ? ring : in + stage_bytes;
  };
  for (int i = 0; i < (S == 1 ? 1 : S - 1); ++i) advance();
  __syncthreads();   // the weights
  int ds_at = 0;     // the place of ds
  [[maybe_unused]] bool handed = false;

  for (long long seg = seg0; seg < a.nseg; seg += workers) {
    int first, end;
    bounds(seg, first, end);
    const long long grp = seg / a.segs_per_group;
    if (LAST && !ROWS && a.gp_smem) gates(a.mode == kGateGroups ? grp : 0);
#pragma unroll 1
    for (int row0 = first; row0 < end; row0 += R) {
      if (S > 2) copy_wait<1>();
      else copy_wait<0>();
      if (!VEC) sync_row();   // others' copies are here, and have left the stage before
      if (S > 1) advance();
      else if (ahead_row < ahead_end) {   // into L2 meanwhile: a request a line of 128 bytes
        constexpr int per = 128 / ES;
#pragma unroll
        for (int x = 0; x < NA; ++x)
          if (source(x))
            for (int i = t * per; i < D; i += tpr * per)
              asm volatile("prefetch.global.L2 [%0];" ::"l"(source(x) + (long long)ahead_row * D + i));
      }
      const uint32_t stage = cur;
      cur = cur + stage_bytes == ring_end ? ring : cur + stage_bytes;
      const int row = row0 + sub;
      const bool live = R == 1 || row < end;
      const long long at = (long long)row * D;
      // where a thread's first column is in pieces that begin before the row
      const uint32_t mis = VEC ? 0 : (uint32_t)(((long long)row0 * D * ES) & 15) + (sub * D + col0) * ES;
      auto cols = [&](int j) {   // a lane's columns, none in rows past the segment
        Cols<VEC> c = columns(j);
        if (!VEC && !live) c.count = 0;
        return c;
      };
      // mean and 1 / deviation of array x; the row in v (KEEP) less the mean
      Pair kept[KEEP ? Q : 1];
      auto load = [&](int x, int j, int count, Pair* v) {
        if (KEEP) {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = kept[KEEP ? 4 * j + i : 0];
        } else {
          take(stage, x, j, mis, count, v);
        }
      };
      auto mean = [&](int x) {
        Pair s = 0;
        if (!KEEP && !a.layer) return 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          Pair v[4];
          take(stage, x, j, mis, cols(j).count, v);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (KEEP) kept[KEEP ? 4 * j + i : 0] = v[i];
            s = add2(s, v[i]);
          }
        }
        if (!a.layer) return 0.f;
        float m[1] = {fold(s)};
        row_sums<TPR, 1>(m, sh, slot, warp0, nw, bar);
        return m[0] * inv;
      };
      Pair ds[ROLE == kRoleAll ? 1 : 4];
      if constexpr (ROLE != kRolePost) {
        const float mh = mean(1);
        // the squares, and the sums of e = dn w and e (h - mean)
        Pair p[3] = {0, 0, 0};
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Cols<VEC> c = cols(j);
          const Pair m = both(!VEC || c.count ? -mh : 0.f);
          Pair v[4], d[4], w[4];
          load(1, j, c.count, v);
          take(stage, 0, j, mis, c.count, d);
          get2(ws + 2 * j * G, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const Pair h = keep(add2(v[i], m), i, c.count), e = mul2(d[i], w[i]);
            if (KEEP) kept[KEEP ? 4 * j + i : 0] = h;
            p[0] = fma2(h, h, p[0]);
            p[1] = add2(p[1], e);
            p[2] = fma2(e, h, p[2]);
          }
        }
        float s[4] = {fold(p[0]), fold(p[1]), fold(p[2]), 0.f};
        row_sums<TPR, 4>(s, sh, slot, warp0, nw, bar);
        const float rh = live ? rsqrtf(s[0] * inv + a.eps) : 0.f;
        const Pair rh2 = both(rh), alpha = both(a.alpha);
        const Pair c1 = both(a.layer ? -rh * s[1] * inv : 0.f), c2 = both(-rh * rh * s[2] * inv);
        if (POST && a.ds_slots == 1) {   // the last row's ds has been read
          if (handed) bar_sync(handover, 2 * wt);
          handed = true;
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Cols<VEC> c = cols(j);
          const Pair m = both(KEEP ? 0.f : !VEC || c.count ? -mh : 0.f);
          Pair dn[4], h[4], g[4], w[4];
          take(stage, 0, j, mis, c.count, dn);
          load(1, j, c.count, h);
          get2(ws + 2 * j * G, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int q = 4 * j + i;
            if (!KEEP) h[i] = keep(add2(h[i], m), i, c.count);
            h[i] = mul2(h[i], rh2);
            g[i] = fma2(rh2, mul2(w[i], dn[i]), fma2(h[i], c2, c1));
            acc[0][q] = fma2(dn[i], h[i], acc[0][q]);
            acc[1][q] = add2(acc[1][q], dn[i]);
          }
          if (a.dh) {
            take(stage, 2, j, mis, c.count, dn);
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = add2(g[i], dn[i]);
          }
          if (POST) put2(dss + ds_at + 2 * j * G, g);
          if (a.dx && live) {
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = mul2(alpha, g[i]);
            write8<VEC>(static_cast<T*>(a.dx) + at, c, h);
          }
          if constexpr (ROLE == kRoleAll) {
            Pair y[4];
            if (read_y) take(stage, kBranch, j, mis, c.count, y);
            if (ROWS) {
              if (a.dgate && live) {
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = mul2(g[i], y[i]);
                write8<VEC>(static_cast<T*>(a.dgate) + at, c, h);
              }
              take(stage, kGate, j, mis, c.count, w);
            } else if (read_y) {
#pragma unroll
              for (int i = 0; i < 4; ++i) acc[kA][4 * j + i] = fma2(g[i], y[i], acc[kA][4 * j + i]);
              get2(gps + 2 * j * G, w);
            }
            if (read_y) {
#pragma unroll
              for (int i = 0; i < 4; ++i) g[i] = mul2(g[i], w[i]);
            }
            if (live) write8<VEC>(static_cast<T*>(a.dbranch) + at, c, g);
          }
        }
      } else {
        const float my = mean(kBranch);
        Pair p = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Cols<VEC> c = cols(j);
          const Pair m = both(!VEC || c.count ? -my : 0.f);
          Pair v[4];
          load(kBranch, j, c.count, v);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const Pair y = keep(add2(v[i], m), i, c.count);
            if (KEEP) kept[KEEP ? 4 * j + i : 0] = y;
            p = fma2(y, y, p);
          }
        }
        float s[1] = {fold(p)};
        row_sums<TPR, 1>(s, sh, slot, warp0, nw, bar);
        const float ry = live ? rsqrtf(s[0] * inv + a.eps) : 0.f;
        const Pair ry2 = both(ry);
        bar_sync(handover, 2 * wt);   // ds is here
        Pair b0 = 0, b1 = 0, dz[Q];
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Cols<VEC> c = cols(j);
          const Pair m = both(!VEC || c.count ? -my : 0.f);
          Pair y[4], gp[4];
          get2(dss + ds_at + 2 * j * G, ds);
          load(kBranch, j, c.count, y);
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = mul2(KEEP ? y[i] : keep(add2(y[i], m), i, c.count), ry2);
          if (ROWS) {
            if (a.pw_smem) get2(ws + V + 2 * j * G, gp);
            else vector(a.post_weight, j, gp);
            if (a.dgate) {
              Pair dg[4], pb[4] = {0, 0, 0, 0};
              if (a.pw_smem) get2(ws + 2 * V + 2 * j * G, pb);
              else if (a.post_bias) vector(a.post_bias, j, pb);
#pragma unroll
              for (int i = 0; i < 4; ++i) dg[i] = mul2(ds[i], fma2(y[i], gp[i], pb[i]));
              if (live) write8<VEC>(static_cast<T*>(a.dgate) + at, c, dg);
            }
            Pair g[4];
            take(stage, kGate, j, mis, c.count, g);
#pragma unroll
            for (int i = 0; i < 4; ++i) ds[i] = mul2(ds[i], g[i]);
          } else {
            get2(gps + 2 * j * G, gp);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int q = 4 * j + i;
            acc[0][q] = fma2(ds[i], y[i], acc[0][q]);
            acc[1][q] = add2(acc[1][q], ds[i]);
            dz[q] = mul2(ds[i], gp[i]);
            b0 = add2(b0, dz[q]);
            b1 = fma2(dz[q], y[i], b1);
          }
        }
        if (a.ds_slots == 1) bar_sync(handover, 2 * wt);   // read
        float b[2] = {fold(b0), fold(b1)};
        row_sums<TPR, 2>(b, sh, slot, warp0, nw, bar);
        const Pair d1 = both(a.layer ? -ry * b[0] * inv : 0.f), d2 = both(-ry * ry * b[1] * inv);
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const Cols<VEC> c = cols(j);
          const Pair m = both(KEEP ? 0.f : -my);
          Pair y[4];
          load(kBranch, j, c.count, y);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            y[i] = fma2(ry2, dz[4 * j + i], fma2(KEEP ? y[i] : add2(y[i], m), d2, d1));
          if (live) write8<VEC>(static_cast<T*>(a.dbranch) + at, c, y);
        }
      }
      if (ROLE == kRolePre) bar_sync(handover, 2 * wt);   // ds is there
      if (POST && a.ds_slots == 2) ds_at = V - ds_at;
      if (S == 1) {
        if (!VEC) sync_row();
        advance();
      }
    }
    if (!LAST || ROWS || a.mode != kGateGroups) continue;
    // A and B of the gate's segment that ends here: the gate's gradient, and dpw and dpb
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const Cols<VEC> c = columns(j);
      Pair s0[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) s0[i] = acc[kA][4 * j + i];
      if (POST) {
        Pair g[4], pw[4], s1[4];
        gate_row(j, grp, g);
#pragma unroll
        for (int i = 0; i < 4; ++i) s1[i] = acc[1][4 * j + i];
        Pair u[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (a.one_seg) {   // the worker's only segment
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][4 * j + e] = mul2(acc[i][4 * j + e], g[e]);
            continue;
          }
          float* part = a.part + ((long long)blockIdx.x * 4 + 2 + i) * D;
          if (a.tot_smem) {
            get2(tot + i * V + 2 * j * G, u);
          } else {
            Raw8<float> r;
            read8<VEC>(part, c, true, r);
            widen2(r, u);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            u[e] = fma2(acc[i][4 * j + e], g[e], u[e]);
            acc[i][4 * j + e] = 0;
          }
          if (a.tot_smem) put2(tot + i * V + 2 * j * G, u);
          else write8<VEC>(part, c, u);
        }
        vector(a.post_weight, j, pw);
#pragma unroll
        for (int i = 0; i < 4; ++i) s0[i] = mul2(s0[i], pw[i]);
        if (a.post_bias) {
          vector(a.post_bias, j, pw);
#pragma unroll
          for (int i = 0; i < 4; ++i) s0[i] = fma2(pw[i], s1[i], s0[i]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[kA][4 * j + i] = 0;
      }
      if (!a.dgate) continue;
      // rows side by side in a warp: theirs together
      if (R > 1) {
#pragma unroll
        for (int o = TPR; o < 32; o <<= 1)
#pragma unroll
          for (int i = 0; i < 4; ++i) s0[i] = add2(s0[i], shfl_xor(s0[i], o));
      }
      if (sub == 0) {
        if (a.segs_per_group == 1) write8<VEC>(static_cast<T*>(a.dgate) + seg * D, c, s0);
        else write8<VEC>(a.gate_part + seg * D, c, s0);
      }
    }
  }
  if (ROLE == kRolePre && handed) bar_sync(handover, 2 * wt);
  copy_wait<0>();
  // the CTA's sums (dw, db | dpw, dpb, or for one gate A, B): its rows' added through shared
  // memory
  const uint32_t buf0 = base + (ROLE == kRolePost ? nwarps * V : 0);
  constexpr bool kTotals = ROLE == kRolePost && !ROWS;
#pragma unroll
  for (int i = 0; i < NACC; ++i) {
    const int v = i + (ROLE == kRolePost ? 2 : 0);
    const bool want = (a.wanted >> v & 1) && !(kTotals && a.mode == kGateGroups && !a.tot_smem && !a.one_seg);
    __syncthreads();
    if (want) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        Pair* p = acc[i] + 4 * j;
        if (kTotals && a.tot_smem) get2(tot + (i & 1) * V + 2 * j * G, p);
        if (R > 1) {   // rows side by side in a warp
#pragma unroll
          for (int o = TPR; o < 32; o <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = add2(p[e], shfl_xor(p[e], o));
        }
        put2(buf0 + wid * V + lane * 16 + 2 * j * G, p);
      }
    }
    __syncthreads();
    if (tid < tpr && want) {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        Pair s[4] = {0, 0, 0, 0}, u[4];
        for (int k = wr; k < nwarps; k += wt / 32) {
          get2(buf0 + k * V + 2 * j * G + lane * 16, u);
#pragma unroll
          for (int e = 0; e < 4; ++e) s[e] = add2(s[e], u[e]);
        }
        write8<VEC>(a.part + ((long long)blockIdx.x * 4 + v) * D, columns(j), s);
      }
    }
  }
}

template <class T, int TPR, int J, bool VEC, bool POST, bool ROWS, int MAXT>
__global__ void __launch_bounds__(MAXT, 1) norm_bwd_kernel(const __grid_constant__ NormBwd a) {
  extern __shared__ float4 dyn4[];
  __shared__ RowShared sh;
  pdl_enter();
  if constexpr (!POST) norm_bwd_role<T, TPR, J, VEC, ROWS, kRoleAll>(a, dyn4, sh);
  else if (threadIdx.x < blockDim.x / 2) norm_bwd_role<T, TPR, J, VEC, ROWS, kRolePre>(a, dyn4, sh);
  else norm_bwd_role<T, TPR, J, VEC, ROWS, kRolePost>(a, dyn4, sh);
}

namespace {

template <class T, int TPR, int J, bool VEC, bool POST, bool ROWS>
cudaError_t bwd_launch(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  static std::atomic<unsigned long long> done{0};
  auto k = norm_bwd_kernel<T, TPR, J, VEC, POST, ROWS, norm_max_warps(J, TPR <= 32) * 32>;
  cudaError_t e = smem_opt_in(k, kNormSmem, &done);
  if (e != cudaSuccess) return e;
  return launch_k(k, dim3(pl.ctas), dim3(pl.threads), pl.smem, lc.stream, a);
}
template <class T, int TPR, int J, bool POST, bool ROWS>
cudaError_t bwd_shape(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  return a.D % 8 == 0 ? bwd_launch<T, TPR, J, true, POST, ROWS>(lc, a, pl)
                      : bwd_launch<T, TPR, J, false, POST, ROWS>(lc, a, pl);
}
template <class T, bool POST, bool ROWS>
cudaError_t bwd_typed(const Launch& lc, const NormBwd& a, const NormPlan& pl) {
  if (pl.tpr == 8) return bwd_shape<T, 8, 1, POST, ROWS>(lc, a, pl);
  if (pl.tpr == 16) return bwd_shape<T, 16, 1, POST, ROWS>(lc, a, pl);
  if (pl.tpr == 32 && pl.J == 1) return bwd_shape<T, 32, 1, POST, ROWS>(lc, a, pl);
  if (pl.tpr == 32 && pl.J == 2) return bwd_shape<T, 32, 2, POST, ROWS>(lc, a, pl);
  if constexpr (POST) {
    if (pl.tpr == 32) return bwd_shape<T, 32, 3, POST, ROWS>(lc, a, pl);
  }
  if (pl.J == 2) return bwd_shape<T, 64, 2, POST, ROWS>(lc, a, pl);
  if constexpr (POST) {
    if (pl.J == 3) return bwd_shape<T, 64, 3, POST, ROWS>(lc, a, pl);
    return bwd_shape<T, 64, 4, POST, ROWS>(lc, a, pl);
  }
  return cudaErrorInvalidValue;
}

}  // namespace

}  // namespace bcmt
