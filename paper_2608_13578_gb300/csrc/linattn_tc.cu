// Linear attention with a decay per head on the tcgen05 tensor cores (bf16,
// head widths up to 128): the chunked form of the recurrence.
//
// A CTA walks the 128-token chunks of one segment of one head.  With S the
// state coming into a chunk, w(t) = a^(tokens from the chunk's start to t,
// counting t) and rows in time order,
//   O = ((Q K^T) o D) V + diag(w) (Q S),   D[t][s] = a^(t-s) for s <= t, else 0,
//   S <- a^n S + K'^T V,                   K'[s] = a^(n-1-s) K[s],  n valid rows.
// A reverse walk flips the order of the rows (D transposed, w and K' from the
// other end) and does not decay the incoming state by the last valid token.
//
// Tiles are [128 tokens x DP] bf16 (DP = 64 or 128 channels, the head width
// zero-padded by TMA), two stages of Q, K, V ahead of the products.  The
// decayed scores P go from TMEM through registers back to TMEM as the bf16 A
// operand of P V, in place of the scores.  The state is kept in fp32 registers
// (a thread holds half a row); its bf16 copy in shared memory is the B operand
// of Q S.  K' is written over K as bf16 and its rounding error over Q as a
// second bf16 term, so that the running state carries 16 bits of each decayed
// key: at DP = 64 the two terms are the two 64-row halves of one M = 128
// product, at DP = 128 two accumulated products.
#include <algorithm>

#include "attn_common.cuh"
#include "common.cuh"
#include "linattn.h"
#include "tc.cuh"
#include "tmap.h"

namespace bcmt {
using namespace attn;

struct LinTcArgs {
  CUtensorMap map[4];
  LinArgs a;
  int mq[3], mk[3], mv[3];  // the pass's maps
};

namespace {

constexpr int kRows = 128;  // tokens of a chunk

// D[tmem] (+)= A[tmem] * B for one 16-deep K step: A bf16 pairs packed in 32-bit
// columns, lane = row.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc,
                                            uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Whole warp: 16 columns of the warp's lane quarter (no wait).
__device__ __forceinline__ void tmem_ld16_issue(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
// Whole warp: 8 columns of the warp's lane quarter, written.
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// Barrier of the two warps that share a lane quarter.
__device__ __forceinline__ void pair_sync(int quarter) {
  asm volatile("bar.sync %0, 64;" ::"r"(quarter + 1) : "memory");
}

template <int DP>
struct TcGeo {
  static constexpr int kHalves = DP / 64;
  static constexpr uint32_t kTile = kRows * DP * 2;  // one operand tile
  static constexpr uint32_t kHalf = kRows * 128;     // its 64-channel halves
  static constexpr uint32_t kState = DP * DP * 2;    // the state's bf16 copy
  static constexpr uint32_t kStage = 3 * kTile;
  // TMEM columns: scores (P over their first 64), P V, Q S, state increment
  static constexpr uint32_t kCols = DP == 64 ? 256 : 512;
  static constexpr uint32_t cO1 = DP == 64 ? 64 : 128, cO2 = cO1 + DP, cD = cO2 + DP;
  static constexpr int kSmem = 1024 + 2 * kStage + kState + 4 * 256 + 64;
};

}  // namespace

template <int DP, bool LOCAL>
__global__ void __launch_bounds__(256, DP == 64 ? 2 : 1)
    linattn_tc_kernel(const __grid_constant__ LinTcArgs A, unsigned* status) {
  using G = TcGeo<DP>;
  constexpr int HC = DP / 2;  // columns of a row that a thread holds
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = align1024(smem_raw);
  uint8_t* sS = smem + 2 * G::kStage;
  float* pw = reinterpret_cast<float*>(sS + G::kState);  // a^0 .. a^128
  float* cw = pw + 132;                                  // column weights of a 32-block
  float* dz = cw + 32;                                   // dz[31 + d] = a^d, 0 for d < 0
  uint64_t* bar = reinterpret_cast<uint64_t*>(pw + 256);
  uint64_t* bar_full = bar;  // stage loaded (2)
  uint64_t* bar_a = bar + 2;  // scores and Q S done
  uint64_t* bar_d = bar + 3;  // state increment done
  uint64_t* bar_c = bar + 4;  // P V done
  uint32_t* tslot = reinterpret_cast<uint32_t*>(bar + 5);

  const LinArgs& a = A.a;
  const int ps = blockIdx.y;
  const LinPass& p = a.pass[ps];
  const int seg = blockIdx.x % a.nseg, bh = blockIdx.x / a.nseg;
  const int b = bh / a.H, h = bh - b * a.H;
  const bool rev = p.rev != 0;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3, g = warp >> 2;
  const int r = q * 32 + lane;

  if (tid == 0) {
    for (int i = 0; i < 5; ++i) tc::mbar_init(&bar[i], 1);
    tc::fence_mbar_init();
    tc::prefetch_tmap(&A.map[A.mk[ps]]);
    tc::prefetch_tmap(&A.map[A.mv[ps]]);
    if (!LOCAL) tc::prefetch_tmap(&A.map[A.mq[ps]]);
  }
  // nobody needs the last segment's own contribution
  if (LOCAL && seg == (rev ? 0 : a.nseg - 1)) {
    pdl_enter();
    return;
  }
  if (warp == 0) {
    tc::tmem_alloc(tslot, G::kCols);
    tc::tmem_relinquish();
  }
  pdl_enter();
  const int n = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  const int seg_lo = seg * a.seg_len, seg_hi = min(a.T, seg_lo + a.seg_len);
  const int t_lo = min(seg_lo, n), t_hi = min(seg_hi, n);
  const int nch = (t_hi - t_lo + kRows - 1) / kRows;
  const float dec = a.decay[h];
  const int dh = a.dh;
  const long long tok0 = (long long)b * a.T;
  const long long st = (long long)dh * dh;

  auto chunk_start = [&](int i) { return t_lo + (rev ? nch - 1 - i : i) * kRows; };
  auto load = [&](int i) {  // thread 0: chunk i of the walk into stage i % 2
    uint8_t* s = smem + (i & 1) * G::kStage;
    uint64_t* bf = &bar_full[i & 1];
    const int row = (int)(tok0 + chunk_start(i));
    tc::mbar_arrive_expect_tx(bf, (LOCAL ? 2 : 3) * G::kTile);
#pragma unroll
    for (int f = 0; f < G::kHalves; ++f) {
      if (!LOCAL) tc::tma_load_3d(s + f * G::kHalf, &A.map[A.mq[ps]], bf, f * 64, h, row);
      tc::tma_load_3d(s + G::kTile + f * G::kHalf, &A.map[A.mk[ps]], bf, f * 64, h, row);
      tc::tma_load_3d(s + 2 * G::kTile + f * G::kHalf, &A.map[A.mv[ps]], bf, f * 64, h, row);
    }
  };
  if (tid == 0) {
    if (nch > 0) load(0);
    if (nch > 1) load(1);
  }
  for (int i = tid; i < 129; i += 256) pw[i] = powf(dec, (float)i);
  if (tid < 32) cw[tid] = powf(dec, (float)(rev ? tid : 31 - tid));
  if (tid >= 64 && tid < 128) dz[tid - 64] = tid - 64 < 31 ? 0.f : powf(dec, (float)(tid - 95));

  // ---- the incoming state: fp32 in registers, bf16 in shared memory.  Thread:
  // state row srow, columns g*HC .. g*HC + HC - 1; at DP = 64 the warps of the
  // lower two lane quarters hold the sums of the keys' second terms.
  const bool lo_part = DP == 64 && q < 2;
  const int srow = DP == 64 ? r & 63 : r;
  float S[HC];
#pragma unroll
  for (int c = 0; c < HC; ++c) S[c] = 0.f;
  bool have = false;  // a state to apply
  if (!LOCAL) {
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
    have = src != nullptr;
    if (src && !lo_part && srow < dh) {
#pragma unroll
      for (int c = 0; c < HC; c += 4) {
        const int col = g * HC + c;
        if (col >= dh) continue;
        if (sj == 1) {
          load4(src + srow * si + col, S + c);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) S[c + e] = src[srow * si + (col + e) * sj];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) S[c + e] *= mul;
      }
    }
  }
  auto put_state = [&]() {
    if (lo_part) return;
    uint8_t* base = sS + (DP == 128 ? g * (DP * 128) : 0);
#pragma unroll
    for (int u = 0; u < HC / 8; ++u)
      *reinterpret_cast<uint4*>(base + tc::sw128_offset(srow, DP == 128 ? u : g * 4 + u)) =
          pack8(S + 8 * u);
  };
  if (have) put_state();
  tc::fence_proxy_async_smem();
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = *tslot;
  const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16);
  constexpr uint32_t idS = tc::idesc_bf16(128, 128, 0, 0);
  constexpr uint32_t idQS = tc::idesc_bf16(128, DP, 0, 1);
  constexpr uint32_t idD = tc::idesc_bf16(128, DP, 1, 1);
  bool ok = true;
  int i = 0;

  for (; i < nch; ++i) {
    uint8_t* sQ = smem + (i & 1) * G::kStage;
    uint8_t* sK = sQ + G::kTile;
    uint8_t* sV = sK + G::kTile;
    const int t0 = chunk_start(i);
    const int m = min(kRows, t_hi - t0);  // valid rows
    const int fresh = rev && t0 + m == n ? 1 : 0;
    ok = tc::mbar_wait(&bar_full[i & 1], (i >> 1) & 1, status) && ok;
    if (!LOCAL) {
      if (tid == 0) {
        tc::fence_after_sync();
        if (ok) {
#pragma unroll
          for (int kk = 0; kk < DP / 16; ++kk)
            tc::mma_bf16(tmem, p_kmaj(sQ, 0, kk), p_kmaj(sK, 0, kk), idS, kk > 0 ? 1u : 0u);
          if (have) {
#pragma unroll
            for (int kk = 0; kk < DP / 16; ++kk)
              tc::mma_bf16(tmem + G::cO2, p_kmaj(sQ, 0, kk),
                           tc::sdesc(tc::smem_u32(sS) + kk * 2048, DP * 128, 1024), idQS,
                           kk > 0 ? 1u : 0u);
          }
        }
        tc::mma_commit(bar_a);
      }
      __syncwarp();
      ok = tc::mbar_wait(bar_a, i & 1, status) && ok;
      tc::fence_after_sync();

      // ---- decayed scores: row r, columns 32 j + 16 g .. + 15 of every block j
      uint32_t pk[4][8];
#pragma unroll
      for (int j0 = 0; j0 < 4; j0 += 2) {
        uint32_t sr[2][16];
#pragma unroll
        for (int j = j0; j < j0 + 2; ++j)
          if (rev ? j >= q : j <= q) tmem_ld16_issue(trow + 32 * j + 16 * g, sr[j - j0]);
        tc::tmem_wait();
#pragma unroll
        for (int j = j0; j < j0 + 2; ++j) {
          const uint32_t* x = sr[j - j0];
          if (j == q) {
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
              float v[2];
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const int l = 16 * g + e + y;
                const bool in = rev ? l >= lane && 32 * j + l < m : l <= lane;
                const float w = dz[31 + (rev ? l - lane : lane - l)];
                v[y] = in ? __uint_as_float(x[e + y]) * w : 0.f;
              }
              pk[j][e >> 1] = pack2(v[0], v[1]);
            }
          } else if (rev ? j > q : j < q) {
            const float base = rev ? pw[32 * (j - q) - lane] : pw[32 * (q - j) + lane - 31];
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
              float w[4], v[4];
              load4(cw + 16 * g + e, w);
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                v[y] = __uint_as_float(x[e + y]) * (base * w[y]);
                if (rev && 32 * j + 16 * g + e + y >= m) v[y] = 0.f;
              }
              pk[j][e >> 1] = pack2(v[0], v[1]);
              pk[j][(e >> 1) + 1] = pack2(v[2], v[3]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) pk[j][e] = 0u;
          }
        }
      }
      tc::fence_before_sync();
      pair_sync(q);  // both warps of the quarter have their scores: P may replace them
      tc::fence_after_sync();
#pragma unroll
      for (int j = 0; j < 4; ++j) tmem_st8(trow + 16 * j + 8 * g, pk[j]);
      tmem_st_wait();
    }

    // ---- K' in two bf16 terms, over K and Q
#pragma unroll
    for (int x = 0; x < DP / 16; ++x) {
      const int idx = x * 256 + tid;
      const int f = idx >> 10, row = (idx >> 3) & 127, u = idx & 7;
      const uint32_t off = f * G::kHalf + tc::sw128_offset(row, u);
      const float w = row < m ? pw[rev ? row : m - 1 - row] : 0.f;
      float v[8], hi[8];
      load8(reinterpret_cast<const bf16*>(sK + off), v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = row < m ? v[e] * w : 0.f;
      const uint4 ph = pack8(v);
      unpack8(ph, hi);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] -= hi[e];
      *reinterpret_cast<uint4*>(sK + off) = ph;
      *reinterpret_cast<uint4*>(sQ + off) = pack8(v);
    }
    if (m < kRows) {  // rows past the end may hold anything: they meet zero weights
      for (int idx = tid; idx < (kRows - m) * (DP / 8); idx += 256) {
        const int row = m + idx / (DP / 8), u = idx % (DP / 8);
        *reinterpret_cast<uint4*>(sV + (u >> 3) * G::kHalf + tc::sw128_offset(row, u & 7)) =
            make_uint4(0, 0, 0, 0);
      }
    }
    tc::fence_proxy_async_smem();
    tc::fence_before_sync();
    __syncthreads();
    if (tid == 0) {
      tc::fence_after_sync();
      if (ok) {
#pragma unroll
        for (int kk = 0; kk < kRows / 16; ++kk)
          tc::mma_bf16(tmem + G::cD,
                       // DP = 64: the second terms' rows (over Q), then the first's
                       tc::sdesc(tc::smem_u32(DP == 64 ? sQ : sK) + kk * 2048, G::kHalf, 1024),
                       tc::sdesc(tc::smem_u32(sV) + kk * 2048, G::kHalf, 1024), idD,
                       kk > 0 ? 1u : 0u);
        if (DP == 128) {
#pragma unroll
          for (int kk = 0; kk < kRows / 16; ++kk)
            tc::mma_bf16(tmem + G::cD, tc::sdesc(tc::smem_u32(sQ) + kk * 2048, G::kHalf, 1024),
                         tc::sdesc(tc::smem_u32(sV) + kk * 2048, G::kHalf, 1024), idD, 1u);
        }
      }
      tc::mma_commit(bar_d);
      if (!LOCAL) {
        if (ok) {
#pragma unroll
          for (int kk = 0; kk < kRows / 16; ++kk)
            mma_bf16_ts(tmem + G::cO1, tmem + kk * 8,
                        tc::sdesc(tc::smem_u32(sV) + kk * 2048, G::kHalf, 1024), idQS,
                        kk > 0 ? 1u : 0u);
        }
        tc::mma_commit(bar_c);
      }
    }
    __syncwarp();

    // ---- the new state
    ok = tc::mbar_wait(bar_d, i & 1, status) && ok;
    tc::fence_after_sync();
    const float f = pw[m - fresh];
#pragma unroll
    for (int c0 = 0; c0 < HC; c0 += 32) {
      float d[32];
      tc::tmem_ld32(trow + G::cD + g * HC + c0, d);
#pragma unroll
      for (int c = 0; c < 32; ++c) S[c0 + c] = fmaf(f, S[c0 + c], d[c]);
    }
    if (!LOCAL) {
      if (i + 1 < nch) put_state();
      // ---- the chunk's output rows
      ok = tc::mbar_wait(bar_c, i & 1, status) && ok;
      tc::fence_after_sync();
      const float wq = r < m ? pw[rev ? m - r - fresh : r + 1] : 0.f;
      bf16* dst = (bf16*)p.o + (tok0 + t0 + r) * p.ldo + h * dh;
#pragma unroll
      for (int c0 = 0; c0 < HC; c0 += 16) {
        uint32_t x1[16], x2[16];
        tmem_ld16_issue(trow + G::cO1 + g * HC + c0, x1);
        if (have) tmem_ld16_issue(trow + G::cO2 + g * HC + c0, x2);
        tc::tmem_wait();
        float o[16];
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          o[c] = __uint_as_float(x1[c]);
          if (have) o[c] = fmaf(wq, __uint_as_float(x2[c]), o[c]);
          o[c] *= p.out_mul;
        }
        if (r < m && ok) {
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int col = g * HC + c0 + 8 * u;
            if (col < dh) *reinterpret_cast<uint4*>(dst + col) = pack8(o + 8 * u);
          }
        }
      }
    }
    have = true;
    tc::fence_proxy_async_smem();
    tc::fence_before_sync();
    // the stage's products are done and every thread is past its tiles
    if (!__syncthreads_and(ok)) break;
    tc::fence_after_sync();
    if (tid == 0 && i + 2 < nch) load(i + 2);
  }
  if (i < nch) {  // a wait ran out: let the loads in flight land before leaving
    if (tid == 0) {
      tc::mbar_wait(&bar_full[i & 1], (i >> 1) & 1, status);
      if (i + 1 < nch) tc::mbar_wait(&bar_full[(i + 1) & 1], ((i + 1) >> 1) & 1, status);
    }
    ok = false;
    __syncthreads();
  }

  if (!LOCAL) {  // the rows past the sequence's end
    const int r0 = max(seg_lo, n), rows = seg_hi - r0;
    const int dv = dh / 8;
    for (int x = tid; x < rows * dv; x += 256) {
      const int rr = x / dv, u = x - rr * dv;
      *reinterpret_cast<uint4*>((bf16*)p.o + (tok0 + r0 + rr) * p.ldo + h * dh + u * 8) =
          make_uint4(0, 0, 0, 0);
    }
  }
  float* dst = nullptr;
  float mul = 1.f;
  if (LOCAL) {
    dst = p.seg + ((long long)bh * a.nseg + seg) * st;
  } else if (p.s_out && seg == (rev ? 0 : a.nseg - 1)) {
    dst = p.s_out + (long long)bh * st;
    mul = n > 0 ? p.s_out_mul * (rev ? dec : 1.f) : 1.f;
  }
  if (dst) {  // uniform over the CTA; the stages are idle here
    if (DP == 64) {
      float* x = reinterpret_cast<float*>(smem);
      if (lo_part) {
#pragma unroll
        for (int c = 0; c < HC; ++c) x[srow * 65 + g * HC + c] = S[c];
      }
      __syncthreads();
      if (!lo_part) {
#pragma unroll
        for (int c = 0; c < HC; ++c) S[c] += x[srow * 65 + g * HC + c];
      }
    }
    if (!lo_part && srow < dh && ok) {
#pragma unroll
      for (int c = 0; c < HC; c += 4) {
        const int col = g * HC + c;
        if (col >= dh) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = S[c + e] * mul;
        store4(dst + (long long)srow * dh + col, v);
      }
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 0) tc::tmem_dealloc(tmem, G::kCols);
}

// ---------------------------------------------------------------- host side
namespace {

template <int DP>
cudaError_t tc_launch(const Launch& lc, const LinTcArgs& A) {
  using G = TcGeo<DP>;
  static std::atomic<unsigned long long> opted{0}, opted_local{0};
  cudaError_t e = smem_opt_in(linattn_tc_kernel<DP, false>, G::kSmem, &opted);
  if (e != cudaSuccess) return e;
  const dim3 grid(A.a.nseg * A.a.B * A.a.H, A.a.npass);
  if (A.a.nseg > 1) {
    if ((e = smem_opt_in(linattn_tc_kernel<DP, true>, G::kSmem, &opted_local)) != cudaSuccess)
      return e;
    e = launch_k(linattn_tc_kernel<DP, true>, grid, dim3(256), G::kSmem, lc.stream, A, lc.status);
    if (e != cudaSuccess) return e;
    if ((e = linattn_combine(lc, A.a)) != cudaSuccess) return e;
  }
  e = launch_k(linattn_tc_kernel<DP, false>, grid, dim3(256), G::kSmem, lc.stream, A, lc.status);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t linattn_tc(const Launch& lc, const LinArgs& a) {
  LinTcArgs A;
  A.a = a;
  int nmaps = 0;
  const void* base[4];
  long lds[4];
  bool good = true;
  // one map per distinct operand: channels x heads x tokens of all sequences
  auto map_of = [&](const void* x, long ld) {
    for (int i = 0; i < nmaps; ++i)
      if (base[i] == x && lds[i] == ld) return i;
    const uint64_t dims[3] = {(uint64_t)a.dh, (uint64_t)a.H, (uint64_t)a.B * a.T};
    const uint64_t strides[2] = {(uint64_t)a.dh * 2, (uint64_t)ld * 2};
    const uint32_t box[3] = {64, 1, kRows};
    base[nmaps] = x;
    lds[nmaps] = ld;
    good = make_tmap_bf16(&A.map[nmaps], x, 3, dims, strides, box) && good;
    return nmaps++;
  };
  for (int i = 0; i < a.npass; ++i) {
    A.mq[i] = map_of(a.pass[i].q, a.pass[i].ldq);
    A.mk[i] = map_of(a.pass[i].k, a.pass[i].ldk);
    A.mv[i] = map_of(a.pass[i].v, a.pass[i].ldv);
  }
  if (!good) return cudaErrorInvalidValue;
  return a.dh <= 64 ? tc_launch<64>(lc, A) : tc_launch<128>(lc, A);
}

}  // namespace bcmt
