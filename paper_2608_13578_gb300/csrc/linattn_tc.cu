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
// zero-padded by TMA) in two stages.  Three roles share a CTA:
//  * one thread issues the loads and the products: A = Q K^T, B = Q S, C = P V,
//    D = K'^T V, in that order for each chunk;
//  * four warps ("rows", thread = token row) turn the scores into P, which goes
//    back to TMEM over the scores as the bf16 A operand of C, and store the
//    chunk's output C + w B;
//  * four warps ("state", thread = state row) keep S in fp32 registers, write its
//    bf16 copy (the B operand of Q S), and write K' over K, with its rounding
//    error as a second bf16 term over Q, so that the running state carries 16
//    bits of each decayed key.  At DP = 64 the two terms are the halves of one
//    M = 128 product, at DP = 128 two accumulated products.
// Only D -> S -> B is sequential over the chunks; the rest of a chunk runs beside
// its neighbours' chain.
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
// Whole warp: 16 columns of the warp's lane quarter, written.
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// 32 bytes in one store (sm_100 and later); the address 32-byte aligned.
__device__ __forceinline__ void store32(void* p, const uint4& a, const uint4& b) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x),
               "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
               : "memory");
}
// a^n.  Out of line, and the loops below mostly rolled: the roles run different
// code at the same time, and unrolled copies of it (over 100 KB) made
// instruction fetch the kernel's bound (13 us a chunk instead of under 3).
__device__ __noinline__ float decay_pow(float a, int n) { return powf(a, (float)n); }

// A warpgroup's share of the CTA's registers.
template <int N>
__device__ __forceinline__ void reg_dec() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void reg_inc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
// The n lowest bits, n from 0 to 32.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : (1u << n) - 1u; }
// A warp's arrival: its lanes' earlier writes and TMEM accesses come first.
__device__ __forceinline__ void warp_arrive(uint64_t* bar, int lane) {
  tc::fence_before_sync();
  __syncwarp();
  if (lane == 0) tc::mbar_arrive(bar);
}

// A row weight as two bf16 terms, the first in the low half.
__device__ __forceinline__ uint32_t weight_terms(float w) {
  const bf16 hi = __float2bfloat16_rn(w);
  return pack2(w, w - __bfloat162float(hi));
}
// K' of one 16-byte unit (8 channels of a row) in two bf16 terms, by three
// packed bf16 operations a pair: with w = wh + wl, hi = rn(k wh), whose rounding
// error e = k wh - hi is a bf16 number (one fused operation gives it exactly),
// and lo = rn(k wl + e).  hi + lo is k w to about 2^-17.
__device__ __forceinline__ void key_terms(const uint4& k, uint32_t w, uint4& hi, uint4& lo) {
  const __nv_bfloat162 w2 = *reinterpret_cast<const __nv_bfloat162*>(&w);
  const __nv_bfloat162 wh = __low2bfloat162(w2), wl = __high2bfloat162(w2);
  const uint32_t kk[4] = {k.x, k.y, k.z, k.w};
  uint32_t h[4], l[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162*>(&kk[e]);
    const __nv_bfloat162 p = __hmul2_rn(x, wh);
    const __nv_bfloat162 y = __hfma2(x, wl, __hfma2(x, wh, __hneg2(p)));
    h[e] = *reinterpret_cast<const uint32_t*>(&p);
    l[e] = *reinterpret_cast<const uint32_t*>(&y);
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
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
  // at most 227 KB
  static constexpr int kSmem = 1024 + 2 * kStage + kState + 4 * 256 + 4 * 128 + 96;
};

}  // namespace

// `steps` K steps of a product whose operands advance by da and db 16-byte units
// (a from shared memory), accumulating from the first step on if `acc0`.
__device__ __forceinline__ void issue(uint32_t d, uint64_t a, uint32_t da, uint64_t b, uint32_t db,
                                      uint32_t idesc, int steps, uint32_t acc0) {
#pragma unroll 4
  for (int kk = 0; kk < steps; ++kk, a += da, b += db)
    tc::mma_bf16(d, a, b, idesc, kk > 0 ? 1u : acc0);
}
// The products of D: K'^T V into `acc`, K' in two terms over K and Q.
template <int DP>
__device__ __forceinline__ void issue_state(uint32_t acc, const uint8_t* sQ, const uint8_t* sK,
                                            const uint8_t* sV) {
  using G = TcGeo<DP>;
  constexpr uint32_t id = tc::idesc_bf16(128, DP, 1, 1);
  const uint64_t q = tc::sdesc(tc::smem_u32(sQ), G::kHalf, 1024);
  const uint64_t k = tc::sdesc(tc::smem_u32(sK), G::kHalf, 1024);
  const uint64_t v = tc::sdesc(tc::smem_u32(sV), G::kHalf, 1024);
  if (DP == 64) {  // rows 0..63 the second terms (over Q), rows 64..127 the first
    issue(acc, q, 128, v, 128, id, kRows / 16, 0u);
  } else {
    issue(acc, k, 128, v, 128, id, kRows / 16, 0u);
    issue(acc, q, 128, v, 128, id, kRows / 16, 1u);
  }
}

// Zeroes the rows m .. 127 of a tile (threads t of nt).
template <int DP>
__device__ __forceinline__ void clear_rows(uint8_t* tile, int m, int t, int nt) {
  for (int x = t; x < (kRows - m) * (DP / 8); x += nt) {
    const int row = m + x / (DP / 8), u = x % (DP / 8);
    *reinterpret_cast<uint4*>(tile + (u >> 3) * TcGeo<DP>::kHalf + tc::sw128_offset(row, u & 7)) =
        make_uint4(0, 0, 0, 0);
  }
}

// The tokens of a segment that one CTA walks.
struct Walk {
  int n, seg_lo, seg_hi, t_lo, t_hi, nch;
  bool rev;
  __device__ __forceinline__ Walk(const LinArgs& a, int b, int seg, bool r) : rev(r) {
    n = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
    seg_lo = seg * a.seg_len;
    seg_hi = min(a.T, seg_lo + a.seg_len);
    t_lo = min(seg_lo, n);
    t_hi = min(seg_hi, n);
    nch = (t_hi - t_lo + kRows - 1) / kRows;
  }
  __device__ __forceinline__ int start(int i) const { return t_lo + (rev ? nch - 1 - i : i) * kRows; }
  __device__ __forceinline__ int rows(int i) const { return min(kRows, t_hi - start(i)); }
  // 1 where the incoming state is not decayed by the chunk's first token in walk order
  __device__ __forceinline__ int fresh(int i) const { return rev && start(i) + rows(i) == n; }
};

// ------------------------------------------------------------------ the pass
// Registers: the CTA's three warpgroups start with an equal share (80 a thread
// where two CTAs share an SM, else 168); the state's rows need more, the single
// issuing thread less (32 + 80 + 128 = 3 * 80, 88 + 168 + 240 <= 3 * 168).
template <int DP>
__global__ void __launch_bounds__(384, DP == 64 ? 2 : 1)
    linattn_tc_kernel(const __grid_constant__ LinTcArgs A, unsigned* status) {
  using G = TcGeo<DP>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = align1024(smem_raw);
  uint8_t* sS = smem + 2 * G::kStage;
  float* pw = reinterpret_cast<float*>(sS + G::kState) + 127;  // pw[d] = a^|d|, d = -127 .. 128
  uint32_t* pt = reinterpret_cast<uint32_t*>(pw + 129);        // a^0 .. a^127 in two bf16 terms
  uint64_t* bar = reinterpret_cast<uint64_t*>(pt + 128);
  uint64_t* bar_full = bar;   // a stage's tiles have landed (2)
  uint64_t* bar_a = bar + 2;  // products A .. D done
  uint64_t* bar_b = bar + 3;
  uint64_t* bar_c = bar + 4;
  uint64_t* bar_d = bar + 5;
  uint64_t* bar_p = bar + 6;  // P written (rows)
  uint64_t* bar_o = bar + 7;  // C and B read (rows)
  uint64_t* bar_k = bar + 8;  // K' written (state)
  uint64_t* bar_s = bar + 9;  // the state's copy written (state)
  uint64_t* bar_z = bar + 10;  // the rows past the end cleared (state; at most one chunk)
  uint32_t* tslot = reinterpret_cast<uint32_t*>(bar + 11);

  const LinArgs& a = A.a;
  const int ps = blockIdx.y;
  const LinPass& p = a.pass[ps];
  const int seg = blockIdx.x % a.nseg, bh = blockIdx.x / a.nseg;
  const int b = bh / a.H, h = bh - b * a.H;
  const bool rev = p.rev != 0;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3;
  const int r = q * 32 + lane;

  if (tid == 0) {
    for (int i = 0; i < 6; ++i) tc::mbar_init(&bar[i], 1);
    for (int i = 6; i < 11; ++i) tc::mbar_init(&bar[i], 4);
    tc::fence_mbar_init();
  }
  if (warp == 8) {
    if (lane < 3) tc::prefetch_tmap(&A.map[lane == 0 ? A.mq[ps] : lane == 1 ? A.mk[ps] : A.mv[ps]]);
    tc::tmem_alloc(tslot, G::kCols);
    tc::tmem_relinquish();
  }
  pdl_enter();
  const Walk w(a, b, seg, rev);
  const float dec = a.decay[h];
  const int dh = a.dh;
  const long long tok0 = (long long)b * a.T;
  const long long st = (long long)dh * dh;
  const bool have0 = p.s_in != nullptr || (a.nseg > 1 && seg != (rev ? a.nseg - 1 : 0));
  if (tid < 129) {
    const float x = decay_pow(dec, tid);
    pw[tid] = x;
    if (tid < 128) {
      pw[-tid] = x;
      pt[tid] = weight_terms(x);
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = *tslot;
  const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16);
  bool ok = true;  // no wait of this thread has run out
  auto wait = [&](uint64_t* x, int parity) { ok = ok && tc::mbar_wait(x, parity & 1, status); };

  if (warp >= 8) {
    reg_dec<DP == 64 ? 32 : 88>();
    if (tid == 256) {
      // ------------------------------------------------ loads and products
      constexpr uint32_t idA = tc::idesc_bf16(128, 128, 0, 0);
      constexpr uint32_t idO = tc::idesc_bf16(128, DP, 0, 1);
      int loaded = 0;
      auto load = [&]() {  // the next chunk of the walk
        const int i = loaded++;
        uint8_t* s = smem + (i & 1) * G::kStage;
        uint64_t* bf = &bar_full[i & 1];
        const int row = (int)(tok0 + w.start(i));
        tc::mbar_arrive_expect_tx(bf, 3 * G::kTile);
#pragma unroll
        for (int f = 0; f < G::kHalves; ++f) {
          tc::tma_load_3d(s + f * G::kHalf, &A.map[A.mq[ps]], bf, f * 64, h, row);
          tc::tma_load_3d(s + G::kTile + f * G::kHalf, &A.map[A.mk[ps]], bf, f * 64, h, row);
          tc::tma_load_3d(s + 2 * G::kTile + f * G::kHalf, &A.map[A.mv[ps]], bf, f * 64, h, row);
        }
      };
      if (w.nch > 0) load();
      if (w.nch > 1) load();
      for (int i = 0; i < w.nch; ++i) {
        uint8_t* sQ = smem + (i & 1) * G::kStage;
        uint8_t* sK = sQ + G::kTile;
        uint8_t* sV = sK + G::kTile;
        wait(&bar_full[i & 1], i >> 1);
        if (w.rows(i) < kRows) wait(bar_z, 0);
        if (i > 0) {  // P and, at DP = 64, P V share the scores' columns
          wait(bar_c, i - 1);
          wait(bar_o, i - 1);
        }
        tc::fence_after_sync();
        const uint64_t dq = tc::sdesc(tc::smem_u32(sQ), 16, 1024);
        if (ok) {
          const uint64_t dk = tc::sdesc(tc::smem_u32(sK), 16, 1024);
#pragma unroll
          for (int f = 0; f < G::kHalves; ++f)
            issue(tmem, dq + f * 1024, 2, dk + f * 1024, 2, idA, 4, f > 0 ? 1u : 0u);
        }
        tc::mma_commit(bar_a);
        wait(bar_s, i);
        // chunk i - 1 has had all its products: its stage takes chunk i + 1
        if (ok && i > 0 && loaded < w.nch) load();
        tc::fence_after_sync();
        if (ok && (i > 0 || have0)) {
          const uint64_t ds = tc::sdesc(tc::smem_u32(sS), DP * 128, 1024);
#pragma unroll
          for (int f = 0; f < G::kHalves; ++f)
            issue(tmem + G::cO2, dq + f * 1024, 2, ds + f * 512, 128, idO, 4, f > 0 ? 1u : 0u);
        }
        tc::mma_commit(bar_b);
        wait(bar_p, i);
        tc::fence_after_sync();
        if (ok) {
          const uint64_t dv = tc::sdesc(tc::smem_u32(sV), G::kHalf, 1024);
#pragma unroll 4
          for (int kk = 0; kk < kRows / 16; ++kk)
            mma_bf16_ts(tmem + G::cO1, tmem + kk * 8, dv + kk * 128, idO, kk > 0 ? 1u : 0u);
        }
        tc::mma_commit(bar_c);
        wait(bar_k, i);
        tc::fence_after_sync();
        if (ok) issue_state<DP>(tmem + G::cD, sQ, sK, sV);
        tc::mma_commit(bar_d);
      }
      if (!ok) {  // the loads in flight land before the CTA leaves
        for (int i = max(0, loaded - 2); i < loaded; ++i)
          tc::mbar_wait(&bar_full[i & 1], (i >> 1) & 1, status);
      }
    }
    __syncwarp();
  } else if (warp < 4) {
    // ------------------------------------------------------------- rows
    const bool wide = p.ldo % 16 == 0 && dh % 16 == 0 && (reinterpret_cast<uintptr_t>(p.o) & 31) == 0;
    for (int i = 0; i < w.nch; ++i) {
      const int t0 = w.start(i), m = w.rows(i);
      wait(bar_a, i);
      tc::fence_after_sync();
      // P, 32 columns at a time: block j of it covers half of the scores' block
      // j / 2, which has been read by then
#pragma unroll 1
      for (int j = 0; j < 4; ++j) {
        uint32_t pk[16];
        if (rev ? j >= q : j <= q) {
          uint32_t x[32];
          tc::tmem_ld32_issue(trow + 32 * j, x);
          const float* wt = pw + r - 32 * j;
          tc::tmem_wait();
#pragma unroll
          for (int e = 0; e < 32; e += 2)
            pk[e >> 1] = pack2(__uint_as_float(x[e]) * wt[-e], __uint_as_float(x[e + 1]) * wt[-e - 1]);
          if (j == q) {  // the diagonal block: column l is seen up to (rev: from) row l
            const uint32_t in = rev ? ~low_bits(lane) : low_bits(lane + 1);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              if (!((in >> (2 * e)) & 1u)) pk[e] &= 0xffff0000u;
              if (!((in >> (2 * e + 1)) & 1u)) pk[e] &= 0x0000ffffu;
            }
          }
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) pk[e] = 0u;
        }
        tmem_st16(trow + 16 * j, pk);
      }
      tmem_st_wait();
      warp_arrive(bar_p, lane);

      // ---- the chunk's output row
      wait(bar_c, i);  // C was issued after B: both are done
      tc::fence_after_sync();
      const bool have = i > 0 || have0;
      const float wq = r < m ? p.out_mul * pw[rev ? m - r - w.fresh(i) : r + 1] : 0.f;
      bf16* dst = (bf16*)p.o + (tok0 + t0 + r) * p.ldo + h * dh;
#pragma unroll 1
      for (int c0 = 0; c0 < DP; c0 += 16) {
        uint32_t x1[16], x2[16];
        tmem_ld16_issue(trow + G::cO1 + c0, x1);
        if (have) tmem_ld16_issue(trow + G::cO2 + c0, x2);
        tc::tmem_wait();
        if (c0 + 16 == DP) warp_arrive(bar_o, lane);
        float o[16];
        const float2 mul2 = make_float2(p.out_mul, p.out_mul), wq2 = make_float2(wq, wq);
#pragma unroll
        for (int c = 0; c < 16; c += 2) {
          float2 y = __fmul2_rn(make_float2(__uint_as_float(x1[c]), __uint_as_float(x1[c + 1])), mul2);
          if (have)
            y = __ffma2_rn(make_float2(__uint_as_float(x2[c]), __uint_as_float(x2[c + 1])), wq2, y);
          o[c] = y.x;
          o[c + 1] = y.y;
        }
        if (r < m && ok) {
          const uint4 u0 = pack8(o), u1 = pack8(o + 8);
          if (wide) {
            if (c0 < dh) store32(dst + c0, u0, u1);
          } else {
            if (c0 < dh) *reinterpret_cast<uint4*>(dst + c0) = u0;
            if (c0 + 8 < dh) *reinterpret_cast<uint4*>(dst + c0 + 8) = u1;
          }
        }
      }
    }
    // the rows past the sequence's end
    const int r0 = max(w.seg_lo, w.n), rows = w.seg_hi - r0, dv = dh / 8;
    for (int x = tid; x < rows * dv; x += 128) {
      const int rr = x / dv, u = x - rr * dv;
      *reinterpret_cast<uint4*>((bf16*)p.o + (tok0 + r0 + rr) * p.ldo + h * dh + u * 8) =
          make_uint4(0, 0, 0, 0);
    }
  } else {
    // ------------------------------------------------------------ state
    // thread: a row of the state; at DP = 64 the lower 64 threads keep the sums
    // of the keys' second terms
    reg_inc<DP == 64 ? 128 : 240>();
    const int t = tid - 128;
    const bool lo_part = DP == 64 && r < 64;
    const int srow = DP == 64 ? r & 63 : r;
    float S[DP];
#pragma unroll
    for (int c = 0; c < DP; ++c) S[c] = 0.f;
    const bool mine = !lo_part && srow < dh;
    if (have0) {
      // the incoming state, through the increment's TMEM columns: 16 columns of
      // the row at a time
      const float in_mul = w.n > 0 ? p.s_in_mul : 1.f;  // an empty sequence passes its state on
#pragma unroll 1
      for (int c0 = 0; c0 < DP; c0 += 16) {
        float v[16];
#pragma unroll
        for (int c = 0; c < 16; ++c) v[c] = 0.f;
        if (mine && a.nseg > 1 && a.joined) {
          const float* src = p.seg + ((long long)bh * a.nseg + seg) * st + srow * dh + c0;
#pragma unroll
          for (int c = 0; c < 16; c += 4)
            if (c0 + c < dh) load4(src + c, v + c);
        } else if (mine) {
          if (p.s_in) {
            const float* src = p.s_in + (long long)bh * st;
            const long si = p.s_in_t ? 1 : dh, sj = p.s_in_t ? dh : 1;
#pragma unroll
            for (int c = 0; c < 16; ++c)
              if (c0 + c < dh) v[c] = in_mul * src[srow * si + (c0 + c) * sj];
          }
          // the segments before this one, in walk order
#pragma unroll 1
          for (int s = rev ? a.nseg - 1 : 0; s != seg; s += rev ? -1 : 1) {
            const int ms = min(max(w.n - s * a.seg_len, 0), a.seg_len);
            if (ms == 0) continue;
            const bool fresh = rev && w.n <= s * a.seg_len + a.seg_len;
            const float f = decay_pow(dec, ms - (fresh ? 1 : 0));
            const float* src = p.seg + ((long long)bh * a.nseg + s) * st + srow * dh + c0;
#pragma unroll
            for (int c = 0; c < 16; c += 4)
              if (c0 + c < dh) {
                float x[4];
                load4(src + c, x);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[c + e] = fmaf(f, v[c + e], x[e]);
              }
          }
        }
        uint32_t u[16];
#pragma unroll
        for (int c = 0; c < 16; ++c) u[c] = __float_as_uint(v[c]);
        tmem_st16(trow + G::cD + c0, u);
      }
      tmem_st_wait();
    }
    float f = 0.f;
    for (int i = 0;; ++i) {
      // S <- f S + increment: the incoming state, then each chunk's
      if (i > 0 || have0) {
#pragma unroll
        for (int c0 = 0; c0 < DP; c0 += 32) {
          uint32_t d[32];
          tc::tmem_ld32_issue(trow + G::cD + c0, d);
          tc::tmem_wait();
          const float2 f2 = make_float2(f, f);
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            const float2 y =
                __ffma2_rn(f2, make_float2(S[c0 + c], S[c0 + c + 1]),
                           make_float2(__uint_as_float(d[c]), __uint_as_float(d[c + 1])));
            S[c0 + c] = y.x;
            S[c0 + c + 1] = y.y;
          }
        }
      }
      if (i == w.nch) break;
      if (!lo_part) {
#pragma unroll
        for (int u = 0; u < DP / 8; ++u)
          *reinterpret_cast<uint4*>(sS + (u >> 3) * (DP * 128) + tc::sw128_offset(srow, u & 7)) =
              pack8(S + 8 * u);
      }
      tc::fence_proxy_async_smem();
      warp_arrive(bar_s, lane);

      uint8_t* sQ = smem + (i & 1) * G::kStage;
      uint8_t* sK = sQ + G::kTile;
      const int m = w.rows(i);
      if (m < kRows) {
        // rows past the end may hold anything, and they meet zero weights only
        wait(&bar_full[i & 1], i >> 1);
        clear_rows<DP>(sK, m, t, 128);
        clear_rows<DP>(sK + G::kTile, m, t, 128);
        tc::fence_proxy_async_smem();
        warp_arrive(bar_z, lane);
      }
      wait(&bar_full[i & 1], i >> 1);
      wait(bar_b, i);  // the keys and the queries have been used
      const uint32_t* wr = rev ? pt : pt + m - 1;
#pragma unroll 4
      for (int x = 0; x < DP / 8; ++x) {
        const int idx = x * 128 + t, row = (idx >> 3) & 127;
        const uint32_t off = (idx >> 10) * G::kHalf + tc::sw128_offset(row, idx & 7);
        uint4 hi, lo;
        key_terms(*reinterpret_cast<const uint4*>(sK + off), row < m ? wr[rev ? row : -row] : 0u,
                  hi, lo);
        *reinterpret_cast<uint4*>(sK + off) = hi;
        *reinterpret_cast<uint4*>(sQ + off) = lo;
      }
      tc::fence_proxy_async_smem();
      warp_arrive(bar_k, lane);
      f = pw[m - w.fresh(i)];
      wait(bar_d, i);
      tc::fence_after_sync();
    }
    if (p.s_out && seg == (rev ? 0 : a.nseg - 1)) {  // uniform over the CTA
      float* dst = p.s_out + (long long)bh * st + srow * dh;
      const float mul = w.n > 0 ? p.s_out_mul * (rev ? dec : 1.f) : 1.f;
      if (DP == 64) {  // the two terms' sums, through the idle stages
        float* x = reinterpret_cast<float*>(smem);
        if (w.nch > 0) wait(bar_c, w.nch - 1);
        if (lo_part) {
#pragma unroll
          for (int c = 0; c < DP; ++c) x[srow * 65 + c] = S[c];
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (!lo_part) {
#pragma unroll
          for (int c = 0; c < DP; ++c) S[c] += x[srow * 65 + c];
        }
      }
      if (mine && ok) {
#pragma unroll
        for (int c = 0; c < DP; c += 4)
          if (c < dh) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = S[c + e] * mul;
            store4(dst + c, v);
          }
      }
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 8) tc::tmem_dealloc(tmem, G::kCols);
}

// ---------------------------------------------------------- segment states
// The state that a segment adds (from zero, before the segments' join): product
// D alone, its increments double-buffered in TMEM, so that the next chunk's K'
// is written under this one's product.  Reads K and V once: bandwidth-bound.
template <int DP>
__global__ void __launch_bounds__(288, DP == 64 ? 2 : 1)
    linattn_state_kernel(const __grid_constant__ LinTcArgs A, unsigned* status) {
  using G = TcGeo<DP>;
  constexpr int HC = DP / 2;  // columns of a state row that a thread holds
  constexpr uint32_t kCols = 2 * DP;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = align1024(smem_raw);
  float* pw = reinterpret_cast<float*>(smem + 2 * G::kStage + G::kState);  // a^0 .. a^128
  uint32_t* pt = reinterpret_cast<uint32_t*>(pw + 130);                    // in two bf16 terms
  uint64_t* bar = reinterpret_cast<uint64_t*>(pt + 128);
  uint64_t* bar_full = bar;   // (2)
  uint64_t* bar_d = bar + 2;  // (2)
  uint64_t* bar_k = bar + 4;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(bar + 5);

  const LinArgs& a = A.a;
  const int ps = blockIdx.y;
  const LinPass& p = a.pass[ps];
  const bool rev = p.rev != 0;
  // nobody needs the last segment's own contribution
  const int per = a.nseg - 1;
  const int bh = blockIdx.x / per, seg = blockIdx.x - bh * per + (rev ? 1 : 0);
  const int b = bh / a.H, h = bh - b * a.H;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3, g = (warp >> 2) & 1;
  const int r = q * 32 + lane;
  if (tid == 0) {
    for (int i = 0; i < 4; ++i) tc::mbar_init(&bar[i], 1);
    tc::mbar_init(bar_k, 8);
    tc::fence_mbar_init();
  }
  if (warp == 8) {
    if (lane < 2) tc::prefetch_tmap(&A.map[lane == 0 ? A.mk[ps] : A.mv[ps]]);
    tc::tmem_alloc(tslot, kCols);
    tc::tmem_relinquish();
  }
  pdl_enter();
  const Walk w(a, b, seg, rev);
  const float dec = a.decay[h];
  const int dh = a.dh;
  const long long tok0 = (long long)b * a.T;
  if (tid < 129) {
    const float x = decay_pow(dec, tid);
    pw[tid] = x;
    if (tid < 128) pt[tid] = weight_terms(x);
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = *tslot;
  const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16);
  bool ok = true;
  auto wait = [&](uint64_t* x, int parity) { ok = ok && tc::mbar_wait(x, parity & 1, status); };

  if (warp == 8) {
    if (lane == 0) {
      int loaded = 0;
      auto load = [&]() {
        const int i = loaded++;
        uint8_t* s = smem + (i & 1) * G::kStage;
        uint64_t* bf = &bar_full[i & 1];
        const int row = (int)(tok0 + w.start(i));
        tc::mbar_arrive_expect_tx(bf, 2 * G::kTile);
#pragma unroll
        for (int f = 0; f < G::kHalves; ++f) {
          tc::tma_load_3d(s + G::kTile + f * G::kHalf, &A.map[A.mk[ps]], bf, f * 64, h, row);
          tc::tma_load_3d(s + 2 * G::kTile + f * G::kHalf, &A.map[A.mv[ps]], bf, f * 64, h, row);
        }
      };
      if (w.nch > 0) load();
      if (w.nch > 1) load();
      for (int i = 0; i < w.nch; ++i) {
        uint8_t* sQ = smem + (i & 1) * G::kStage;
        wait(bar_k, i);
        tc::fence_after_sync();
        if (ok) issue_state<DP>(tmem + (i & 1) * DP, sQ, sQ + G::kTile, sQ + 2 * G::kTile);
        tc::mma_commit(&bar_d[i & 1]);
        if (loaded < w.nch) {
          wait(&bar_d[i & 1], i >> 1);  // the stage is free again
          if (ok) load();
        }
      }
      if (!ok) {
        for (int i = max(0, loaded - 2); i < loaded; ++i)
          tc::mbar_wait(&bar_full[i & 1], (i >> 1) & 1, status);
      }
    }
    __syncwarp();
  } else {
    const bool lo_part = DP == 64 && r < 64;
    const int srow = DP == 64 ? r & 63 : r;
    float S[HC];
#pragma unroll
    for (int c = 0; c < HC; ++c) S[c] = 0.f;
    auto add = [&](int i) {  // chunk i's increment
      wait(&bar_d[i & 1], i >> 1);
      tc::fence_after_sync();
      const float f = pw[w.rows(i)];
#pragma unroll
      for (int c0 = 0; c0 < HC; c0 += 32) {
        float d[32];
        tc::tmem_ld32(trow + (i & 1) * DP + g * HC + c0, d);
#pragma unroll
        for (int c = 0; c < 32; ++c) S[c0 + c] = fmaf(f, S[c0 + c], d[c]);
      }
    };
    for (int i = 0; i < w.nch; ++i) {
      uint8_t* sQ = smem + (i & 1) * G::kStage;
      uint8_t* sK = sQ + G::kTile;
      const int m = w.rows(i);
      wait(&bar_full[i & 1], i >> 1);
      if (m < kRows) {  // rows past the end may hold anything, and they meet zero weights only
        clear_rows<DP>(sK, m, tid, 256);
        clear_rows<DP>(sK + G::kTile, m, tid, 256);
        asm volatile("bar.sync 1, 256;" ::: "memory");
      }
      const uint32_t* wr = rev ? pt : pt + m - 1;
#pragma unroll 4
      for (int x = 0; x < DP / 16; ++x) {
        const int idx = x * 256 + tid, row = (idx >> 3) & 127;
        const uint32_t off = (idx >> 10) * G::kHalf + tc::sw128_offset(row, idx & 7);
        uint4 hi, lo;
        key_terms(*reinterpret_cast<const uint4*>(sK + off), row < m ? wr[rev ? row : -row] : 0u,
                  hi, lo);
        *reinterpret_cast<uint4*>(sK + off) = hi;
        *reinterpret_cast<uint4*>(sQ + off) = lo;
      }
      tc::fence_proxy_async_smem();
      warp_arrive(bar_k, lane);
      if (i > 0) add(i - 1);
    }
    if (w.nch > 0) add(w.nch - 1);
    float* dst = p.seg + ((long long)bh * a.nseg + seg) * dh * dh + srow * dh;
    if (DP == 64) {  // the two terms' sums, through the idle stages
      float* x = reinterpret_cast<float*>(smem);
      if (lo_part) {
#pragma unroll
        for (int c = 0; c < HC; ++c) x[srow * 65 + g * HC + c] = S[c];
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (!lo_part) {
#pragma unroll
        for (int c = 0; c < HC; ++c) S[c] += x[srow * 65 + g * HC + c];
      }
    }
    if (!lo_part && srow < dh && ok) {
#pragma unroll
      for (int c = 0; c < HC; c += 4)
        if (g * HC + c < dh) store4(dst + g * HC + c, S + c);
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 8) tc::tmem_dealloc(tmem, kCols);
}

// ---------------------------------------------------------------- host side
namespace {

template <int DP>
cudaError_t tc_launch(const Launch& lc, const LinTcArgs& A) {
  using G = TcGeo<DP>;
  static std::atomic<unsigned long long> opted{0}, opted_state{0};
  cudaError_t e = smem_opt_in(linattn_tc_kernel<DP>, G::kSmem, &opted);
  if (e != cudaSuccess) return e;
  const unsigned heads = (unsigned)A.a.B * A.a.H;
  if (A.a.nseg > 1) {
    if ((e = smem_opt_in(linattn_state_kernel<DP>, G::kSmem, &opted_state)) != cudaSuccess) return e;
    e = launch_k(linattn_state_kernel<DP>, dim3(heads * (A.a.nseg - 1), A.a.npass), dim3(288),
                 G::kSmem, lc.stream, A, lc.status);
    if (e != cudaSuccess) return e;
    if (A.a.joined && (e = linattn_combine(lc, A.a)) != cudaSuccess) return e;
  }
  e = launch_k(linattn_tc_kernel<DP>, dim3(heads * A.a.nseg, A.a.npass), dim3(384), G::kSmem,
               lc.stream, A, lc.status);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t linattn_tc(const Launch& lc, const LinArgs& a) {
  LinTcArgs A;
  A.a = a;
  // few segments: each CTA joins the states before its own; a state updated in
  // place is read before any CTA writes it only if a kernel of its own joins
  A.a.joined = a.nseg > 8 || (a.pass[0].s_in && a.pass[0].s_in == a.pass[0].s_out);
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
