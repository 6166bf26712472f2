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
// zero-padded by TMA) in two stages.  Roles of a CTA:
//  * one thread issues the loads, one the products: A = Q K^T, B = Q S, C = P V,
//    D = K'^T V, in that order for each chunk;
//  * "rows" (thread = token row) turn the scores into P, which goes back to TMEM
//    over the scores as the bf16 A operand of C, and store the output C + w B;
//  * "state" (thread = state row) keep S in fp32 registers, write its bf16 copy
//    (the B operand of Q S), and write K' over K, with its rounding error as a
//    second bf16 term over Q, so that the running state carries 16 bits of each
//    decayed key.  At DP = 64 the two terms are the halves of one M = 128 product,
//    at DP = 128 two accumulated products.
// Only D -> S -> B is sequential over the chunks; the rest of a chunk runs beside
// its neighbours' chain.
//
// Rounding: the scores times their decay, and S, are rounded to bf16 where they
// meet bf16 rows in a product, like any operand of the tensor cores (that gives
// the outputs the error of one more bf16 rounding: 0.23% for 0.17% in the root
// mean square).  S itself is a sum of up to T terms, in fp32 throughout.  States that
// the call returns have K' in three terms, by CTAs of their own (state_cta).
//
// What bounds it: at width 128 most of all shared memory (a chunk's loads, products'
// operands, K' and S's copy are 512 KB, 2.1 us at 128 bytes a cycle, of the 3.3 us
// that it takes; the tensor cores are busy for 28%); at width 64 the chain D -> S ->
// B of latencies.  4 sequences of 4095 tokens, 8 heads of 128, backward:
// 109 us, 197 TFLOP/s of the recurrence's own operations; 8 x 1024 tokens of 8
// heads of 64, forward: 23.5 us.
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
  int out;                  // the pass with an outgoing state, or -1
};

namespace {

constexpr int kRows = 128;  // tokens of a chunk

// Shared-memory matrix descriptors (128-byte swizzle, 8-row atoms of 1024 bytes)
// as their two words: the upper one is the same for every operand here, the
// lower one holds the address and the leading-dimension offset.  The issuing
// threads work on lower words and 32-bit addresses, to stay within the few
// registers they keep.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, uint32_t lbo) {
  return ((saddr & 0x3FFFFu) >> 4) | ((lbo >> 4) << 16);
}
// D[tmem] (+)= A B over `steps` 16-deep K steps, whose operands advance by da
// and db 16-byte units; the first step accumulates if acc0.
template <int steps>
__device__ __forceinline__ void issue(uint32_t d, uint32_t a, uint32_t da, uint32_t b, uint32_t db,
                                      uint32_t idesc, uint32_t acc0) {
#pragma unroll
  for (int kk = 0; kk < steps; ++kk)
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
        "r"(a + kk * da), "r"(b + kk * db), "r"(idesc), "r"(kk > 0 ? 1u : acc0), "r"(kDescHi)
        : "memory");
}
// The same with A in TMEM: bf16 pairs packed in 32-bit columns, lane = row.
template <int steps>
__device__ __forceinline__ void issue_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t db,
                                         uint32_t idesc) {
#pragma unroll
  for (int kk = 0; kk < steps; ++kk)
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 db;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 db, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d),
        "r"(a + kk * 8), "r"(b + kk * db), "r"(idesc), "r"(kk > 0 ? 1u : 0u), "r"(kDescHi)
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
// 32 bytes in one store (sm_100 and later); the address 32-byte aligned.
__device__ __forceinline__ void store32(void* p, const uint4& a, const uint4& b) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x),
               "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
               : "memory");
}
// a^n from log2 a (a = 0: the logarithm is -inf).  The product's rounding shifts
// the result by n |log2 a| 2^-24, below 2^-20 wherever a^n is above 2^-23.
__device__ __forceinline__ float decay_pow(float lg, int n) {
  return n == 0 ? 1.f : exp2f((float)n * lg);
}

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

// The same in three bf16 terms (hi, mid, lo: 24 bits), by fp32 arithmetic.  mid is
// multiplied by `half`.
__device__ __forceinline__ void key_terms3(const uint4& k, float w, float half, uint4& hi,
                                           uint4& mid, uint4& lo) {
  float v[8], t[8];
  unpack8(k, v);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= w;
  hi = pack8(v);
  unpack8(hi, t);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] -= t[e];
  mid = pack8(v);
  unpack8(mid, t);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] -= t[e];
    t[e] *= half;
  }
  mid = pack8(t);
  lo = pack8(v);
}

// What a CTA's first threads work out for the others.
struct Shared {
  uint32_t tmem;
  int b, h, seg, n, t_lo, t_hi, rev, have0;
};
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
  static constexpr int kSmem = 1024 + 2 * kStage + kState + 4 * 256 + 4 * 128 + 4 * 32 + 8 * 14 +
                               (int)sizeof(Shared);
};

}  // namespace

// The products of D: K'^T V into `acc`, K' in two terms over K and Q of the stage
// at shared address s.
template <int DP>
__device__ __forceinline__ void issue_state(uint32_t acc, uint32_t s) {
  using G = TcGeo<DP>;
  constexpr uint32_t id = tc::idesc_bf16(128, DP, 1, 1);
  const uint32_t q = desc_lo(s, G::kHalf), k = q + (G::kTile >> 4), v = k + (G::kTile >> 4);
  if (DP == 64) {  // rows 0..63 the second terms (over Q), rows 64..127 the first
    issue<kRows / 16>(acc, q, 128, v, 128, id, 0u);
  } else {
    issue<kRows / 16>(acc, k, 128, v, 128, id, 0u);
    issue<kRows / 16>(acc, q, 128, v, 128, id, 1u);
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

// A shared value, read where it is needed.
template <class T>
__device__ __forceinline__ T ld_once(const T* p) {
  return *const_cast<const volatile T*>(p);
}

// The tokens of a segment that one CTA walks.
struct Walk {
  int n, t_lo, t_hi, nch;
  bool rev;
  __device__ __forceinline__ Walk(const LinArgs& a, int b, int seg, bool r) : rev(r) {
    n = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
    t_lo = min(seg * a.seg_len, n);
    t_hi = min(min(a.T, seg * a.seg_len + a.seg_len), n);
    nch = (t_hi - t_lo + kRows - 1) / kRows;
  }
  __device__ __forceinline__ explicit Walk(const Shared* s)
      : n(ld_once(&s->n)), t_lo(ld_once(&s->t_lo)), t_hi(ld_once(&s->t_hi)),
        rev(ld_once(&s->rev) != 0) {
    nch = (t_hi - t_lo + kRows - 1) / kRows;
  }
  __device__ __forceinline__ int start(int i) const { return t_lo + (rev ? nch - 1 - i : i) * kRows; }
  __device__ __forceinline__ int rows(int i) const { return min(kRows, t_hi - start(i)); }
  // the chunk with fewer than kRows rows, or -1
  __device__ __forceinline__ int ragged() const {
    return (t_hi - t_lo) % kRows == 0 ? -1 : rev ? 0 : nch - 1;
  }
  // 1 where the incoming state is not decayed by the chunk's first token in walk order
  __device__ __forceinline__ int fresh(int i) const { return rev && start(i) + rows(i) == n; }
};

// ------------------------------------------------------------------ the pass
// Roles by warpgroup: NW of rows, NW of the state (a thread has 64 columns of its
// row in both), one that issues.  At DP = 128 a CTA fills an SM's shared memory
// (NW = 2), at DP = 64 two CTAs share it (NW = 1).
// Registers: the warpgroups start with an equal share (80 a thread at DP = 64, 96
// at DP = 128) and trade; the sums stay within what the CTA started with.
template <int DP>
struct Roles {
  static constexpr int NW = DP == 64 ? 1 : 2;
  static constexpr int kThreads = 128 * (2 * NW + 1);
  static constexpr int kRegLaunch = DP == 64 ? 80 : 96;
  static constexpr int kRegIssue = DP == 64 ? 48 : 64, kRegRows = DP == 64 ? 80 : 96,
                       kRegState = 112;
  static_assert(kRegIssue + NW * (kRegRows + kRegState) <= (2 * NW + 1) * kRegLaunch, "registers");
};

// What the roles share: shared-memory layout, barriers, the walk.  Each role reads
// it anew (nothing else is live across the split, so each keeps to the registers
// that it has).
template <int DP>
struct View {
  using G = TcGeo<DP>;
  uint8_t* smem;
  __device__ __forceinline__ View(uint8_t* raw) {
    uint32_t s = (tc::smem_u32(raw) + 1023u) & ~1023u;
    asm volatile("" : "+r"(s));  // a value of this role's own
    smem = static_cast<uint8_t*>(__cvta_shared_to_generic(s));
  }
  __device__ __forceinline__ uint8_t* state() const { return smem + 2 * G::kStage; }
  __device__ __forceinline__ float* pw() const {  // pw[d] = a^|d|, d = -127 .. 128
    return reinterpret_cast<float*>(state() + G::kState) + 127;
  }
  __device__ __forceinline__ uint32_t* pt() const {  // a^0 .. a^127 in two bf16 terms
    return reinterpret_cast<uint32_t*>(state() + G::kState + 4 * 256);
  }
  __device__ __forceinline__ float* cw() const {  // a^(distance of column l from the far end)
    return reinterpret_cast<float*>(state() + G::kState + 4 * 256 + 4 * 128);
  }
  __device__ __forceinline__ uint64_t* bars() const {
    return reinterpret_cast<uint64_t*>(state() + G::kState + 4 * 256 + 4 * 128 + 4 * 32);
  }
  __device__ __forceinline__ Shared* shared() const { return reinterpret_cast<Shared*>(bars() + 14); }
};
// Barriers: a stage's tiles have landed, products A and D done (two of each, for
// alternate chunks); B, C done; P written and C, B read (rows); K' written, the
// state's copy written, the rows past the end cleared and the joined state read
// from stage 1 (state).  A wait names
// a phase by its parity alone, so nobody may be able to complete two phases of a
// barrier before one of its waiters has looked at the first: where one role
// could run that far ahead of another, there are two barriers.
#define LINATTN_BARRIERS(v)                                                              \
  uint64_t* bar = (v).bars();                                                            \
  [[maybe_unused]] uint64_t *bar_full = bar, *bar_a = bar + 2, *bar_d = bar + 4,         \
                            *bar_b = bar + 6, *bar_c = bar + 7, *bar_p = bar + 8,        \
                            *bar_o = bar + 9, *bar_k = bar + 10, *bar_s = bar + 11,      \
                            *bar_z = bar + 12, *bar_j = bar + 13;                        \
  bool ok = true; /* no wait of this thread has run out */                               \
  auto wait = [&](uint64_t* x, int parity) { ok = ok && tc::mbar_wait(x, parity & 1, status); }

// One thread: the products.
template <int DP>
__device__ __forceinline__ void role_products(const LinTcArgs& A, uint8_t* raw, unsigned* status) {
  using G = TcGeo<DP>;
  const View<DP> vw(raw);
  uint8_t* smem = vw.smem;
  LINATTN_BARRIERS(vw);
  const Walk w(vw.shared());
  const uint32_t tmem = ld_once(&vw.shared()->tmem);
  const bool have0 = ld_once(&vw.shared()->have0) != 0;
  constexpr uint32_t idA = tc::idesc_bf16(128, 128, 0, 0);
  constexpr uint32_t idO = tc::idesc_bf16(128, DP, 0, 1);
  const uint32_t s0 = tc::smem_u32(smem);
  const int nch = w.nch, ragged = w.ragged();  // the chunk with rows to clear, or -1
  auto scores = [&](int i) {  // A of chunk i
    wait(&bar_full[i & 1], i >> 1);
    if (i == ragged) wait(bar_z, 0);
    tc::fence_after_sync();
    if (ok) {
      const uint32_t dq = desc_lo(s0 + (i & 1) * G::kStage, 16), dk = dq + (G::kTile >> 4);
#pragma unroll
      for (int f = 0; f < G::kHalves; ++f)
        issue<4>(tmem, dq + f * 1024, 2, dk + f * 1024, 2, idA, f > 0 ? 1u : 0u);
    }
    tc::mma_commit(&bar_a[i & 1]);
  };
  if (nch > 0) scores(0);
#pragma unroll 1
  for (int i = 0; i < nch; ++i) {
    const uint32_t s = s0 + (i & 1) * G::kStage;
    wait(bar_s, i);
    if (i > 0) wait(bar_o, i - 1);
    tc::fence_after_sync();
    if (ok && (i > 0 || have0)) {
      const uint32_t dq = desc_lo(s, 16), ds = desc_lo(s0 + 2 * G::kStage, DP * 128);
#pragma unroll
      for (int f = 0; f < G::kHalves; ++f)
        issue<4>(tmem + G::cO2, dq + f * 1024, 2, ds + f * 512, 128, idO, f > 0 ? 1u : 0u);
    }
    tc::mma_commit(bar_b);
    wait(bar_p, i);
    tc::fence_after_sync();
    if (ok)
      issue_ts<kRows / 16>(tmem + G::cO1, tmem, desc_lo(s + 2 * G::kTile, G::kHalf), 128, idO);
    tc::mma_commit(bar_c);
    if (i + 1 == nch) break;  // nobody reads the state after the last chunk
    wait(bar_k, i);
    tc::fence_after_sync();
    if (ok) issue_state<DP>(tmem + G::cD, s);
    tc::mma_commit(&bar_d[i & 1]);
    // the next chunk's scores replace P and, at DP = 64, C.  They come after D:
    // ahead of it they would hold it up until the next chunk's tiles are there
    wait(bar_c, i);
    if (DP == 64) wait(bar_o, i);
    scores(i + 1);
  }
  // no product is in flight when the CTA leaves, whatever ran out
  if (nch > 0) tc::mbar_wait(bar_c, (nch - 1) & 1, status);
}

// Loads chunk i of a walk of head h (the sequence's first token row: tok0).
template <int DP>
__device__ __forceinline__ void load_chunk(const LinTcArgs& A, const View<DP>& vw, const Walk& w,
                                           int ps, int h, int tok0, int i) {
  using G = TcGeo<DP>;
  uint8_t* s = vw.smem + (i & 1) * G::kStage;
  uint64_t* full = vw.bars() + (i & 1);
  const int row = tok0 + w.start(i);
  tc::mbar_arrive_expect_tx(full, 3 * G::kTile);
#pragma unroll
  for (int f = 0; f < G::kHalves; ++f) {
    tc::tma_load_3d(s + f * G::kHalf, &A.map[A.mq[ps]], full, f * 64, h, row);
    tc::tma_load_3d(s + G::kTile + f * G::kHalf, &A.map[A.mk[ps]], full, f * 64, h, row);
    tc::tma_load_3d(s + 2 * G::kTile + f * G::kHalf, &A.map[A.mv[ps]], full, f * 64, h, row);
  }
}

// One thread: the loads (the first chunk's is on its way).
template <int DP, bool kSegs>
__device__ __forceinline__ void role_loads(const LinTcArgs& A, uint8_t* raw, unsigned* status) {
  const View<DP> vw(raw);
  LINATTN_BARRIERS(vw);
  const Walk w(vw.shared());
  const int ps = blockIdx.y, h = ld_once(&vw.shared()->h);
  const int tok0 = ld_once(&vw.shared()->b) * A.a.T;
  int loaded = min(w.nch, 1);
  auto load = [&]() {  // the next chunk of the walk
    load_chunk<DP>(A, vw, w, ps, h, tok0, loaded);
    ++loaded;
  };
  if (w.nch > 1) {
    if (kSegs && !A.a.joined) wait(bar_j, 0);  // the joined state is there until then
    if (ok) load();
  }
  // D of chunk i is its last product: its stage takes chunk i + 2
  for (int i = 0; ok && loaded < w.nch; ++i) {
    wait(&bar_d[i & 1], i >> 1);
    if (!ok) break;
    load();
  }
  // the loads in flight land before the CTA leaves, however it went
  for (int i = max(0, loaded - 2); i < loaded; ++i)
    tc::mbar_wait(&bar_full[i & 1], (i >> 1) & 1, status);
}

// The state coming into segment seg of head bh, from the states of the segments
// before it, to shared memory (in their layout), and after the last segment the
// outgoing state (threads t of nt).  All threads of the CTA share it, 8 columns of
// a row at a time, so that a state takes one latency of L2.
__device__ __forceinline__ void join_states(const LinArgs& a, const LinPass& p, int bh, int seg,
                                            int n, float* to, int t, int nt) {
  const int dh = a.dh, st = dh * dh;
  const float dec = a.decay[bh % a.H], lg = log2f(dec);
  const bool last = p.s_out && seg == (p.rev ? 0 : a.nseg - 1);
  const int before = p.rev ? a.nseg - 1 - seg : seg;
  for (int e = t; e < st / 8; e += nt) {
    const int col = e / dh * 8, row = e - col / 8 * dh, at = col * dh + row * 4;
    float x[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) x[c] = 0.f;
    if (p.s_in) {
      const float* src = p.s_in + (long long)bh * st;
      const float mul = n > 0 ? p.s_in_mul : 1.f;  // an empty sequence passes its state on
#pragma unroll
      for (int c = 0; c < 8; ++c)
        x[c] = mul * (p.s_in_t ? src[(col + c) * dh + row] : src[row * dh + col + c]);
    }
    const int count = before + (last ? 1 : 0);
#pragma unroll 1
    for (int i0 = 0; i0 < count; i0 += 4) {  // in walk order, four segments' loads in flight
      float v[4][8];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = min(i0 + u, count - 1), s = p.rev ? a.nseg - 1 - i : i;
        const float* src = p.seg + ((long long)bh * a.nseg + s) * st + at;
        load4(src, v[u]);
        load4(src + dh * 4, v[u] + 4);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = i0 + u, s = p.rev ? a.nseg - 1 - i : i;
        if (i >= count) break;
        if (i == before) {
          store4(to + at, x);
          store4(to + at + dh * 4, x + 4);
        }
        const int m = min(max(n - s * a.seg_len, 0), a.seg_len);
        if (m == 0) continue;
        const bool fresh = p.rev && n <= s * a.seg_len + a.seg_len;  // holds the last valid token
        const float f = decay_pow(lg, m - (fresh ? 1 : 0));
#pragma unroll
        for (int c = 0; c < 8; ++c) x[c] = fmaf(f, x[c], v[u][c]);
      }
    }
    if (last) {
      const float mul = n > 0 ? p.s_out_mul * (p.rev ? dec : 1.f) : 1.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) x[c] *= mul;
      float* dst = p.s_out + (long long)bh * st + row * dh + col;
      store4(dst, x);
      store4(dst + 4, x + 4);
    } else {
      store4(to + at, x);
      store4(to + at + dh * 4, x + 4);
    }
  }
}

template <int DP>
__device__ __forceinline__ void role_rows(const LinTcArgs& A, uint8_t* raw, unsigned* status) {
  using G = TcGeo<DP>;
  const View<DP> vw(raw);
  LINATTN_BARRIERS(vw);
  const Walk w(vw.shared());
  const float* pw = vw.pw();
  const bool rev = w.rev, have0 = ld_once(&vw.shared()->have0) != 0;
  const LinArgs& a = A.a;
  const LinPass& p = a.pass[blockIdx.y];
  constexpr int NW = Roles<DP>::NW;
  const int tid = threadIdx.x, lane = tid & 31, g = tid >> 7, r = tid & 127, q = r >> 5, dh = a.dh;
  const float* cw = vw.cw();
  const int h = ld_once(&vw.shared()->h);
  const long long tok0 = (long long)ld_once(&vw.shared()->b) * a.T;
  const uint32_t trow = ld_once(&vw.shared()->tmem) + ((uint32_t)(q * 32) << 16);
  const bool wide = p.ldo % 16 == 0 && dh % 16 == 0 && (reinterpret_cast<uintptr_t>(p.o) & 31) == 0;
  // P of the scores' columns 16 hh .. 16 hh + 15
  auto weigh = [&](int hh, const uint32_t* x, uint32_t* pk) {
    const int j = hh >> 1, l0 = (hh & 1) * 16;
    if (j == q) {  // the diagonal block: column l is seen up to (rev: from) row l
      const float* wt = pw + lane - l0;
      const uint32_t in = (rev ? ~low_bits(lane) : low_bits(lane + 1)) >> l0;
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float v0 = __uint_as_float(x[e]) * wt[-e];
        const float v1 = __uint_as_float(x[e + 1]) * wt[-e - 1];
        pk[e >> 1] = pack2((in >> e) & 1u ? v0 : 0.f, (in >> (e + 1)) & 1u ? v1 : 0.f);
      }
    } else {  // a^(distance) as the row's distance from the block times the column's in it
      const float base = rev ? pw[32 * (j - q) - lane] : pw[32 * (q - j) + lane - 31];
      const float2 base2 = make_float2(base, base);
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        const float4 c4 = *reinterpret_cast<const float4*>(cw + l0 + e);
        const float2 v0 =
            __fmul2_rn(__fmul2_rn(make_float2(c4.x, c4.y), base2),
                       make_float2(__uint_as_float(x[e]), __uint_as_float(x[e + 1])));
        const float2 v1 =
            __fmul2_rn(__fmul2_rn(make_float2(c4.z, c4.w), base2),
                       make_float2(__uint_as_float(x[e + 2]), __uint_as_float(x[e + 3])));
        pk[e >> 1] = pack2(v0.x, v0.y);
        pk[(e >> 1) + 1] = pack2(v1.x, v1.y);
      }
    }
  };
  // the halves hh of blocks that the row sees
  const int h0 = rev ? 2 * q : 0, h1 = rev ? 8 : 2 * q + 2;
  for (int i = 0; i < w.nch; ++i) {
    const int t0 = w.start(i), m = w.rows(i);
    wait(&bar_a[i & 1], i >> 1);
    tc::fence_after_sync();
    if (NW == 1) {
      // half hh of P covers columns of the scores' half hh / 2, read by then; the
      // next half's scores are on their way under this one's arithmetic
      uint32_t x[2][16];
      tmem_ld16_issue(trow + 16 * h0, x[0]);
#pragma unroll 1
      for (int hh = h0; hh < h1; hh += 2) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          uint32_t pk[8];
          tc::tmem_wait();
          if (hh + y + 1 < h1) tmem_ld16_issue(trow + 16 * (hh + y + 1), x[1 - y]);
          weigh(hh + y, x[y], pk);
          tmem_st8(trow + 8 * (hh + y), pk);
        }
      }
    } else {
      // the quarter's two warps take every other half
      uint32_t pk[4][8];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int hh = h0 + g + 2 * y;
        if (hh >= h1) break;
        uint32_t x[16];
        tmem_ld16_issue(trow + 16 * hh, x);
        tc::tmem_wait();
        weigh(hh, x, pk[y]);
      }
      // both have read their scores: P may replace them
      tc::fence_before_sync();
      asm volatile("bar.sync %0, 64;" ::"r"(q + 1) : "memory");
      tc::fence_after_sync();
#pragma unroll
      for (int y = 0; y < 4; ++y)
        if (h0 + g + 2 * y < h1) tmem_st8(trow + 8 * (h0 + g + 2 * y), pk[y]);
    }
    {
      const uint32_t zero[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
#pragma unroll 1
      for (int hh = (rev ? 0 : h1) + g; hh < (rev ? h0 : 8); hh += NW) tmem_st8(trow + 8 * hh, zero);
    }
    tmem_st_wait();
    warp_arrive(bar_p, lane);

    // ---- the chunk's output row
    wait(bar_c, i);  // C was issued after B: both are done
    tc::fence_after_sync();
    const bool have = i > 0 || have0;
    const float wq = r < m ? p.out_mul * pw[rev ? m - r - w.fresh(i) : r + 1] : 0.f;
    const float2 mul2 = make_float2(p.out_mul, p.out_mul), wq2 = make_float2(wq, wq);
    bf16* dst = (bf16*)p.o + (tok0 + t0 + r) * p.ldo + h * dh;
#pragma unroll 1
    for (int c0 = g * 64; c0 < g * 64 + 64; c0 += 16) {
      uint32_t x1[16], x2[16];
      tmem_ld16_issue(trow + G::cO1 + c0, x1);
      if (have) tmem_ld16_issue(trow + G::cO2 + c0, x2);
      tc::tmem_wait();
      if ((c0 & 48) == 48) warp_arrive(bar_o, lane);
#pragma unroll
      for (int c = 0; c < 16; c += 2) {
        float2 y = __fmul2_rn(make_float2(__uint_as_float(x1[c]), __uint_as_float(x1[c + 1])), mul2);
        if (have)
          y = __ffma2_rn(make_float2(__uint_as_float(x2[c]), __uint_as_float(x2[c + 1])), wq2, y);
        x1[c >> 1] = pack2(y.x, y.y);
      }
      if (r < m && ok) {
        const uint4 u0 = make_uint4(x1[0], x1[1], x1[2], x1[3]);
        const uint4 u1 = make_uint4(x1[4], x1[5], x1[6], x1[7]);
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
  const int seg_lo = ld_once(&vw.shared()->seg) * a.seg_len, seg_hi = min(a.T, seg_lo + a.seg_len);
  const int r0 = max(seg_lo, w.n), rows = seg_hi - r0, dv = dh / 8;
  for (int x = tid; x < rows * dv; x += 128 * NW) {
    const int rr = x / dv, u = x - rr * dv;
    *reinterpret_cast<uint4*>((bf16*)p.o + (tok0 + r0 + rr) * p.ldo + h * dh + u * 8) =
        make_uint4(0, 0, 0, 0);
  }
}

// 4 NW warps, thread = 64 columns of a row of the state; at DP = 64 the lower 64
// threads keep the sums of the keys' second terms.
template <int DP, bool kSegs>
__device__ __forceinline__ void role_state(const LinTcArgs& A, uint8_t* raw, unsigned* status) {
  using G = TcGeo<DP>;
  constexpr int NW = Roles<DP>::NW;
  const View<DP> vw(raw);
  uint8_t *smem = vw.smem, *sS = vw.state();
  LINATTN_BARRIERS(vw);
  const Walk w(vw.shared());
  const float* pw = vw.pw();
  const uint32_t* pt = vw.pt();
  const bool rev = w.rev;
  const LinArgs& a = A.a;
  const LinPass& p = a.pass[blockIdx.y];
  const int dh = a.dh, seg = ld_once(&vw.shared()->seg);
  const int bh = ld_once(&vw.shared()->b) * a.H + ld_once(&vw.shared()->h);
  const long long st = (long long)dh * dh;
  const int tid = threadIdx.x, lane = tid & 31, r = tid & 127, q = r >> 5;
  const int t = tid - 128 * NW, g = t >> 7, c64 = g * 64;
  const bool lo_part = DP == 64 && r < 64;
  const int srow = DP == 64 ? r & 63 : r;
  float S[64];
#pragma unroll
  for (int c = 0; c < 64; ++c) S[c] = 0.f;
  const bool mine = !lo_part && srow < dh;
  const uint32_t tinc =
      ld_once(&vw.shared()->tmem) + ((uint32_t)(q * 32) << 16) + G::cD + c64;
  // the incoming state: joined in shared memory or by a kernel of its own (in
  // 4-column groups), or the call's
  const bool here = kSegs && !a.joined;
  if (mine) {
    constexpr bool grouped = kSegs;
    const float* src = here      ? reinterpret_cast<const float*>(smem + G::kStage) + srow * 4
                       : grouped ? p.seg + ((long long)bh * a.nseg + seg) * st + srow * 4
                       : p.s_in  ? p.s_in + (long long)bh * st
                                 : nullptr;
    if (src && (grouped || !p.s_in_t)) {
      src += grouped ? c64 * dh : srow * dh + c64;
      const int step = grouped ? dh : 1;
#pragma unroll
      for (int c = 0; c < 64; c += 4)
        if (c64 + c < dh) load4(src + c * step, S + c);
    } else if (src) {
#pragma unroll
      for (int c = 0; c < 64; ++c)
        if (c64 + c < dh) S[c] = src[(c64 + c) * dh + srow];
    }
    // an empty sequence passes its state on as it is
    if (!grouped && p.s_in_mul != 1.f && w.n > 0) {
#pragma unroll
      for (int c = 0; c < 64; ++c) S[c] *= p.s_in_mul;
    }
  }
  if (here) {  // the stage may be loaded
    tc::fence_proxy_async_smem();
    warp_arrive(bar_j, lane);
  }
  float f = 0.f;
  for (int i = 0;; ++i) {
    if (i > 0) {  // S <- f S + the last chunk's increment
#pragma unroll
      for (int c0 = 0; c0 < 64; c0 += 32) {
        uint32_t d[32];
        tc::tmem_ld32_issue(tinc + c0, d);
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
    uint8_t* copy = sS + g * (DP * 128);
    if (DP == 64 && i > 0) {  // the second terms' sums join, by way of the copy's place
      if (lo_part) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          *reinterpret_cast<uint4*>(copy + tc::sw128_offset(srow, u)) = pack8(S + 8 * u);
      }
      asm volatile("bar.sync 1, 128;" ::: "memory");
    }
    if (!lo_part) {
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        uint4* to = reinterpret_cast<uint4*>(copy + tc::sw128_offset(srow, u));
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
        if (DP == 64 && i > 0) unpack8(*to, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += S[8 * u + e];
        *to = pack8(v);
      }
    }
    tc::fence_proxy_async_smem();
    warp_arrive(bar_s, lane);

    uint8_t* sQ = smem + (i & 1) * G::kStage;
    uint8_t* sK = sQ + G::kTile;
    const int m = w.rows(i);
    wait(&bar_full[i & 1], i >> 1);
    if (m < kRows) {
      // rows past the end may hold anything, and they meet zero weights only
      clear_rows<DP>(sK, m, t, 128 * NW);
      clear_rows<DP>(sK + G::kTile, m, t, 128 * NW);
      tc::fence_proxy_async_smem();
      warp_arrive(bar_z, lane);
    }
    if (i + 1 == w.nch) break;
    wait(&bar_a[i & 1], i >> 1);  // the keys have been used
    const uint32_t* wr = rev ? pt : pt + m - 1;
    uint4 lo[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const int idx = x * (128 * NW) + t, row = (idx >> 3) & 127;
      const uint32_t off = (idx >> 10) * G::kHalf + tc::sw128_offset(row, idx & 7);
      uint4 hi;
      key_terms(*reinterpret_cast<const uint4*>(sK + off), row < m ? wr[rev ? row : -row] : 0u, hi,
                lo[x]);
      *reinterpret_cast<uint4*>(sK + off) = hi;
    }
    wait(bar_b, i);  // and so have the queries
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const int idx = x * (128 * NW) + t, row = (idx >> 3) & 127;
      *reinterpret_cast<uint4*>(sQ + (idx >> 10) * G::kHalf + tc::sw128_offset(row, idx & 7)) =
          lo[x];
    }
    tc::fence_proxy_async_smem();
    warp_arrive(bar_k, lane);
    f = pw[m - w.fresh(i)];
    wait(&bar_d[i & 1], i >> 1);
    tc::fence_after_sync();
  }
}

// The outputs of the walk that are not finite, again, from the recurrence token by
// token in fp32 (the rows' threads, at the CTA's end).  In a product over 128 tokens
// an infinity or NaN of v meets the zero weights of the rows before it, and 0 * inf
// is NaN: those rows get here what the definition gives them.  Such a value stays in
// the state, so that one look at the state's last copy and at the last chunk's v finds
// it in any chunk.  A thread keeps half of a column of the state in shared memory, over
// the tiles.  The look costs a walk up to 0.4 us, the rest 0.6 us a token.
template <int DP, bool kSegs>
__device__ __noinline__ void redo_rows(const LinTcArgs& A, uint8_t* raw) {
  using G = TcGeo<DP>;
  constexpr int NT = 128 * Roles<DP>::NW;
  static_assert(NT == 2 * DP && DP * DP * 4 <= G::kStage, "two threads a column, the state in a stage");
  const View<DP> vw(raw);
  const Walk w(vw.shared());
  if (w.nch == 0) return;
  const int tid = threadIdx.x;
  __nv_bfloat162 z = __float2bfloat162_rn(0.f);  // 0 * x: 0 or NaN
  auto look = [&](const uint8_t* at) {
    const uint4 v = *reinterpret_cast<const uint4*>(at);
    const uint32_t vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      z = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&vv[e]), __float2bfloat162_rn(0.f), z);
  };
  // (rows past the end have been cleared)
  const uint8_t* sV = vw.smem + ((w.nch - 1) & 1) * G::kStage + 2 * G::kTile;
#pragma unroll
  for (int x = tid * 16; x < (int)G::kTile; x += NT * 16) look(sV + x);
#pragma unroll
  for (int x = tid * 16; x < (int)G::kState; x += NT * 16) look(vw.state() + x);
  // true for all threads if it is for one; a barrier between them
  auto any = [&](bool x) {
    uint32_t r = x;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %0, 0;\n\t"
        "barrier.cta.red.or.pred q, 1, %1, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "+r"(r)
        : "n"(NT)
        : "memory");
    return r != 0;
  };
  if (!any(!(__low2float(z) + __high2float(z) == 0.f))) return;
  const LinArgs& a = A.a;
  const LinPass& p = a.pass[blockIdx.y];
  const int dh = a.dh, st = dh * dh, h = ld_once(&vw.shared()->h), b = ld_once(&vw.shared()->b);
  const int seg = ld_once(&vw.shared()->seg), bh = b * a.H + h;
  const float dec = a.decay[h], lg = log2f(dec);
  float* S = reinterpret_cast<float*>(vw.smem);  // [dh][dh]
  float* part = reinterpret_cast<float*>(vw.smem + G::kStage);
  const float* segs = p.seg + (long long)bh * a.nseg * st;
#pragma unroll 1
  for (int e = tid; e < st; e += NT) {  // the state coming into the segment
    const int i = e / dh, j = e - i * dh, at = (j >> 2) * dh * 4 + i * 4 + (j & 3);
    float x = 0.f;
    if (kSegs && a.joined) {
      x = segs[seg * st + at];
    } else {
      if (p.s_in)
        x = (w.n > 0 ? p.s_in_mul : 1.f) * p.s_in[(long long)bh * st + (p.s_in_t ? j * dh + i : e)];
#pragma unroll 1
      for (int y = 0; kSegs && y < (w.rev ? a.nseg - 1 - seg : seg); ++y) {
        const int s = w.rev ? a.nseg - 1 - y : y, m = min(max(w.n - s * a.seg_len, 0), a.seg_len);
        const bool fresh = w.rev && w.n <= s * a.seg_len + a.seg_len;
        if (m > 0) x = fmaf(decay_pow(lg, m - (fresh ? 1 : 0)), x, segs[s * st + at]);
      }
    }
    S[e] = x;
  }
  any(false);
  const int j = tid % DP, mid = (dh / 2 + 7) / 8 * 8;
  const bool first = tid < DP;
  const bf16 *q = (const bf16*)p.q, *k = (const bf16*)p.k, *v = (const bf16*)p.v;
  float y = 0.f;
#pragma unroll 1
  for (int x = 0; x < w.t_hi - w.t_lo; ++x) {
    // a column whose state is not finite gives no finite output any more
    if (x % 32 == 31 && !any(j < dh && isfinite(y))) return;
    const int t = w.rev ? w.t_hi - 1 - x : w.t_lo + x;
    const long long tok = (long long)b * a.T + t;
    const float f = w.rev && t == w.n - 1 ? 1.f : dec;
    float acc = 0.f;
    if (j < dh) {
      const float vj = to_f(v[tok * p.ldv + h * dh + j]);
#pragma unroll 1
      for (int i = first ? 0 : mid; i < (first ? mid : dh); i += 8) {
        float kk[8], qq[8], s[8];
        load8(k + tok * p.ldk + h * dh + i, kk);
        load8(q + tok * p.ldq + h * dh + i, qq);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = S[(i + e) * dh + j];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y = fmaf(f, s[e], kk[e] * vj);
          S[(i + e) * dh + j] = y;
          acc = fmaf(qq[e], y, acc);
        }
      }
      if (!first) part[(x & 1) * DP + j] = acc;
    }
    any(false);
    if (j < dh && first) {
      bf16* o = (bf16*)p.o + tok * p.ldo + h * dh + j;
      if (!isfinite(to_f(*o))) *o = from_f<bf16>((acc + part[(x & 1) * DP + j]) * p.out_mul);
    }
  }
}

// ------------------------------------------------------------------ states
// The state that a segment adds (from zero, before the segments' join) or, with
// one segment, the outgoing state: product D alone.  A state that the call returns
// is made to fp32 accuracy, with K' in three bf16 terms (24 bits of each decayed
// key); one that is only a bf16 operand of the outputs has two, as in the walk.
// The second and third terms have a tile each, K and V two stages; the halves of
// a chunk's tokens are products of their own, so that one half's terms are written
// under the other's product, and the increments alternate between two accumulators.
// DP = 64: the terms are the 64-row halves of products, [mid | hi] and [lo | mid]
// with half of the second term in mid; DP = 128: a product for each term.
// A segment's state is stored with the 4-column groups of all rows together: the
// threads of a warp hold a row each, and their accesses are consecutive (row-major
// states made the joins of 8 x 1024 tokens of 8 heads of 64 take 4 us more).
// Bound by shared memory (K read once, three terms written, six operands read, by
// count of bytes 1.6 us a chunk at DP = 128) and the making of the terms: 2.2 us.
// The first 4 DP threads hold the state (32 columns of a row each), the warp after
// them issues.
template <int DP>
__device__ __forceinline__ void state_cta(const LinTcArgs& A, int ps, int bh, int seg,
                                          uint8_t* smem_raw, unsigned* status) {
  using G = TcGeo<DP>;
  constexpr int HC = 32, NT = 4 * DP, kIssue = NT / 32;
  uint8_t* smem = align1024(smem_raw);
  uint8_t *sLo = smem, *sMid = smem + G::kTile, *stages = smem + 2 * G::kTile;
  float* pw = reinterpret_cast<float*>(smem + 6 * G::kTile);  // a^0 .. a^128
  uint64_t* bar = reinterpret_cast<uint64_t*>(pw + 130);
  uint64_t* bar_full = bar;   // K and V have landed (2)
  uint64_t* bar_d = bar + 2;  // D of a half done (2)
  uint64_t* bar_k = bar + 4;  // K' of a half written (2)
  uint32_t* tslot = reinterpret_cast<uint32_t*>(bar + 6);

  const LinArgs& a = A.a;
  const LinPass& p = a.pass[ps];
  const bool rev = p.rev != 0;
  const bool three = p.s_out != nullptr;
  const int b = bh / a.H, h = bh - b * a.H;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = warp & 3, g = warp >> 2;
  const int r = q * 32 + lane;
  if (tid == 0) {
    for (int i = 0; i < 4; ++i) tc::mbar_init(&bar[i], 1);
    for (int i = 4; i < 6; ++i) tc::mbar_init(&bar[i], NT / 32);
    tc::fence_mbar_init();
  }
  if (warp == kIssue) {
    if (lane < 2) tc::prefetch_tmap(&A.map[lane == 0 ? A.mk[ps] : A.mv[ps]]);
    tc::tmem_alloc(tslot, 2 * DP);
    tc::tmem_relinquish();
  }
  pdl_enter();
  const Walk w(a, b, seg, rev);
  const int dh = a.dh;
  if (tid < 129) pw[tid] = tid == 1 ? a.decay[h] : decay_pow(log2f(a.decay[h]), tid);
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  bool ok = true;
  auto wait = [&](uint64_t* x, int parity) { ok = ok && tc::mbar_wait(x, parity & 1, status); };

  if (warp >= kIssue) {
    if (tid == NT) {
      const uint32_t tmem = ld_once(tslot);
      int loaded = 0;
      const int tok0 = b * a.T;
      auto load = [&]() {
        const int i = loaded++;
        uint8_t* s = stages + (i & 1) * 2 * G::kTile;
        uint64_t* bf = &bar_full[i & 1];
        const int row = tok0 + w.start(i);
        tc::mbar_arrive_expect_tx(bf, 2 * G::kTile);
#pragma unroll
        for (int f = 0; f < G::kHalves; ++f) {
          tc::tma_load_3d(s + f * G::kHalf, &A.map[A.mk[ps]], bf, f * 64, h, row);
          tc::tma_load_3d(s + G::kTile + f * G::kHalf, &A.map[A.mv[ps]], bf, f * 64, h, row);
        }
      };
      if (w.nch > 0) load();
      if (w.nch > 1) load();
      constexpr uint32_t id = tc::idesc_bf16(128, DP, 1, 1);
#pragma unroll 1
      for (int i = 0; i < w.nch; ++i) {
        const uint32_t lo = tc::smem_u32(sLo), mid = tc::smem_u32(sMid),
                       k = tc::smem_u32(stages) + (i & 1) * 2 * G::kTile, v = k + G::kTile,
                       acc = tmem + (i & 1) * DP;
#pragma unroll 1
        for (int x = 0; x < 2; ++x) {
          wait(&bar_k[x], i);
          tc::fence_after_sync();
          const uint32_t o = x * 4 * 128, dv = desc_lo(v, G::kHalf) + o;
          if (ok && DP == 64) {
            issue<4>(acc, desc_lo(mid, k - mid) + o, 128, dv, 128, id, x);
            if (three) issue<4>(acc, desc_lo(lo, mid - lo) + o, 128, dv, 128, id, 1u);
          } else if (ok) {
            issue<4>(acc, desc_lo(k, G::kHalf) + o, 128, dv, 128, id, x);
            issue<4>(acc, desc_lo(mid, G::kHalf) + o, 128, dv, 128, id, 1u);
            if (three) issue<4>(acc, desc_lo(lo, G::kHalf) + o, 128, dv, 128, id, 1u);
          }
          tc::mma_commit(&bar_d[x]);
        }
        if (loaded < w.nch || i + 1 == w.nch) wait(&bar_d[1], i);  // the stage is free again
        if (ok && loaded < w.nch) load();
      }
      if (!ok) {  // the loads in flight land before the CTA leaves
        for (int i = max(0, loaded - 2); i < loaded; ++i)
          tc::mbar_wait(&bar_full[i & 1], (i >> 1) & 1, status);
      }
    }
    __syncwarp();
  } else {
    const uint32_t trow = ld_once(tslot) + ((uint32_t)(q * 32) << 16) + g * HC;
    const bool lo_part = DP == 64 && r < 64;
    const int srow = DP == 64 ? r & 63 : r;
    const bool mine = !lo_part && srow < dh;
    const bool whole = a.nseg == 1;  // the outgoing state
    float S[HC];
#pragma unroll
    for (int c = 0; c < HC; ++c) S[c] = 0.f;
    if (whole && mine && p.s_in) {  // (not transposed: no pass has s_in_t and s_out)
      const float* src = p.s_in + (long long)bh * dh * dh;
      const float mul = w.n > 0 ? p.s_in_mul : 1.f;
#pragma unroll
      for (int c = 0; c < HC; c += 4)
        if (g * HC + c < dh) load4(src + srow * dh + g * HC + c, S + c);
#pragma unroll
      for (int c = 0; c < HC; ++c) S[c] *= mul;
    }
    auto add = [&](int i) {  // chunk i's increment
      wait(&bar_d[1], i);
      tc::fence_after_sync();
      const float f = pw[w.rows(i) - (whole ? w.fresh(i) : 0)];
      float d[HC];
      tc::tmem_ld32(trow + (i & 1) * DP, d);
#pragma unroll
      for (int c = 0; c < HC; ++c) S[c] = fmaf(f, S[c], d[c]);
    };
#pragma unroll 1
    for (int i = 0; i < w.nch; ++i) {
      uint8_t* sK = stages + (i & 1) * 2 * G::kTile;
      const int m = w.rows(i);
      wait(&bar_full[i & 1], i >> 1);
      if (m < kRows) {  // rows past the end may hold anything, and they meet zero weights only
        clear_rows<DP>(sK, m, tid, NT);
        clear_rows<DP>(sK + G::kTile, m, tid, NT);
        asm volatile("bar.sync 1, %0;" ::"n"(NT) : "memory");
      }
#pragma unroll 1
      for (int x = 0; x < 2; ++x) {
        // the last chunk's product has used this half's second and third terms
        if (i > 0 && x == 0) wait(&bar_d[0], i - 1);
        if (i > 0 && x == 1) add(i - 1);
        uint4 k[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int idx = u * NT + tid, row = x * 64 + ((idx >> 3) & 63);
          k[u] = *reinterpret_cast<const uint4*>(sK + (idx >> 9) * G::kHalf +
                                                 tc::sw128_offset(row, idx & 7));
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int idx = u * NT + tid, row = x * 64 + ((idx >> 3) & 63);
          const uint32_t off = (idx >> 9) * G::kHalf + tc::sw128_offset(row, idx & 7);
          const float wt = row < m ? pw[rev ? row : m - 1 - row] : 0.f;
          uint4 hi, mid, lo;
          if (three) {
            key_terms3(k[u], wt, DP == 64 ? 0.5f : 1.f, hi, mid, lo);
            *reinterpret_cast<uint4*>(sLo + off) = lo;
          } else {
            key_terms(k[u], weight_terms(wt), hi, mid);
          }
          *reinterpret_cast<uint4*>(sK + off) = hi;
          *reinterpret_cast<uint4*>(sMid + off) = mid;
        }
        tc::fence_proxy_async_smem();
        warp_arrive(&bar_k[x], lane);
      }
    }
    if (w.nch > 0) add(w.nch - 1);
    if (DP == 64) {  // the halves' sums, through the idle tiles
      float* x = reinterpret_cast<float*>(smem);
      if (lo_part) {
#pragma unroll
        for (int c = 0; c < HC; ++c) x[srow * 65 + g * HC + c] = S[c];
      }
      asm volatile("bar.sync 1, %0;" ::"n"(NT) : "memory");
      if (!lo_part) {
#pragma unroll
        for (int c = 0; c < HC; ++c) S[c] += x[srow * 65 + g * HC + c];
      }
    }
    float* dst = whole ? p.s_out + (long long)bh * dh * dh + srow * dh
                       : p.seg + ((long long)bh * a.nseg + seg) * dh * dh + srow * 4;
    const int step = whole ? 1 : dh;
    const float mul = whole && w.n > 0 ? p.s_out_mul * (rev ? pw[1] : 1.f) : 1.f;
    if (mine && ok) {
#pragma unroll
      for (int c = 0; c < HC; c += 4)
        if (g * HC + c < dh) {
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = S[c + e] * mul;
          store4(dst + (g * HC + c) * step, v);
        }
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == kIssue) tc::tmem_dealloc(ld_once(tslot), 2 * DP);
}

// The segments' states (the last one's own contribution is needed for the outgoing
// state only), or the outgoing state after a walk that reads the same buffer.
template <int DP>
__global__ void __launch_bounds__(4 * DP + 32, DP == 64 ? 2 : 1)
    linattn_state_kernel(const __grid_constant__ LinTcArgs A, unsigned* status) {
  extern __shared__ uint8_t smem_raw[];
  const int ps = blockIdx.y, nseg = A.a.nseg;
  const int bh = blockIdx.x / nseg, seg = blockIdx.x - bh * nseg;
  if (!A.a.pass[ps].s_out && seg == (A.a.pass[ps].rev ? 0 : nseg - 1)) return;
  state_cta<DP>(A, ps, bh, seg, smem_raw, status);
}

// kSegs: the heads are cut into segments (their join), or not (the outgoing state's
// CTAs).  A kernel each keeps their code short: as one, the backward of 4 x 4095 tokens
// of 8 heads of 128 took 115 us for 107.
template <int DP, bool kSegs>
__global__ void __launch_bounds__(Roles<DP>::kThreads, DP == 64 ? 2 : 1)
    linattn_tc_kernel(const __grid_constant__ LinTcArgs A, unsigned* status) {
  using G = TcGeo<DP>;
  using R = Roles<DP>;
  constexpr int NW = R::NW;
  extern __shared__ uint8_t smem_raw[];
  if (!kSegs && blockIdx.y == A.a.npass) {  // the outgoing state, beside the walks
    state_cta<DP>(A, A.out, blockIdx.x, 0, smem_raw, status);
    return;
  }
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  {
    const View<DP> vw(smem_raw);
    uint64_t* bar = vw.bars();
    if (tid == 0) {
      for (int i = 0; i < 8; ++i) tc::mbar_init(&bar[i], 1);
      for (int i = 8; i < 14; ++i) tc::mbar_init(&bar[i], 4 * NW);
      tc::fence_mbar_init();
    }
    const int ps = blockIdx.y;
    if (warp == 8 * NW) {
      if (lane < 3) tc::prefetch_tmap(&A.map[lane == 0 ? A.mq[ps] : lane == 1 ? A.mk[ps] : A.mv[ps]]);
      tc::tmem_alloc(&vw.shared()->tmem, G::kCols);
      tc::tmem_relinquish();
    }
    pdl_enter();
    const LinArgs& a = A.a;
    const int seg = blockIdx.x % a.nseg, bh = blockIdx.x / a.nseg, b = bh / a.H, h = bh - b * a.H;
    const bool rev = a.pass[ps].rev != 0;
    if (tid == 0) {
      const Walk w(a, b, seg, rev);
      if (w.nch > 0) load_chunk<DP>(A, vw, w, ps, h, b * a.T, 0);
    }
    if (tid == 32) {
      Shared* sh = vw.shared();
      sh->b = b;
      sh->h = h;
      sh->seg = seg;
      sh->rev = rev;
      sh->have0 = a.pass[ps].s_in != nullptr || (a.nseg > 1 && seg != (rev ? a.nseg - 1 : 0));
      const Walk w(a, b, seg, rev);
      sh->n = w.n;
      sh->t_lo = w.t_lo;
      sh->t_hi = w.t_hi;
      check_decay(a.decay[h], status);
    }
    if (tid >= 64 && tid < 193) {
      const int d = tid - 64;
      const float x = decay_pow(log2f(a.decay[h]), d);
      vw.pw()[d] = d == 1 ? a.decay[h] : x;
      if (d < 128) {
        vw.pw()[-d] = x;
        vw.pt()[d] = weight_terms(x);
        if (d < 32) vw.cw()[rev ? d : 31 - d] = d == 1 ? a.decay[h] : x;
      }
    }
    if (kSegs && !a.joined)
      join_states(a, a.pass[ps], bh, seg, a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T,
                  reinterpret_cast<float*>(vw.smem + G::kStage), tid, R::kThreads);
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  if (warp >= 8 * NW) {
    reg_dec<R::kRegIssue>();
    if (tid == 256 * NW) role_products<DP>(A, smem_raw, status);
    if (tid == 256 * NW + 32) role_loads<DP, kSegs>(A, smem_raw, status);
    __syncwarp();
  } else if (warp < 4 * NW) {
    reg_dec<R::kRegRows>();
    role_rows<DP>(A, smem_raw, status);
  } else {
    reg_inc<R::kRegState>();
    role_state<DP, kSegs>(A, smem_raw, status);
  }
  tc::fence_before_sync();
  __syncthreads();
  if (warp == 8 * NW) tc::tmem_dealloc(View<DP>(smem_raw).shared()->tmem, G::kCols);
  if (warp < 4 * NW) redo_rows<DP, kSegs>(A, smem_raw);
}

// ---------------------------------------------------------------- host side
namespace {

template <int DP>
cudaError_t tc_launch(const Launch& lc, const LinTcArgs& A) {
  using G = TcGeo<DP>;
  static std::atomic<unsigned long long> opted{0}, opted_segs{0}, opted_state{0};
  cudaError_t e = smem_opt_in(linattn_tc_kernel<DP, false>, G::kSmem, &opted);
  if (e == cudaSuccess) e = smem_opt_in(linattn_tc_kernel<DP, true>, G::kSmem, &opted_segs);
  if (e != cudaSuccess) return e;
  const unsigned heads = (unsigned)A.a.B * A.a.H;
  if ((e = smem_opt_in(linattn_state_kernel<DP>, G::kSmem, &opted_state)) != cudaSuccess) return e;
  auto states = [&](int passes) {
    return launch_k(linattn_state_kernel<DP>, dim3(heads * A.a.nseg, passes), dim3(4 * DP + 32), G::kSmem,
                    lc.stream, A, lc.status);
  };
  if (A.a.nseg > 1) {
    if ((e = states(A.a.npass)) != cudaSuccess) return e;
    if (A.a.joined && (e = linattn_combine(lc, A.a)) != cudaSuccess) return e;
  }
  // One segment: the outgoing state is a product of its own, by CTAs beside the
  // walks, or after them where it overwrites the state that they read
  const bool whole = A.out >= 0 && A.a.nseg == 1;
  bool after = false;
  for (int i = 0; whole && i < A.a.npass; ++i)
    after = after || A.a.pass[i].s_in == A.a.pass[A.out].s_out;
  e = launch_k(A.a.nseg > 1 ? linattn_tc_kernel<DP, true> : linattn_tc_kernel<DP, false>,
               dim3(heads * A.a.nseg, A.a.npass + (whole && !after ? 1 : 0)),
               dim3(Roles<DP>::kThreads), G::kSmem, lc.stream, A, lc.status);
  if (e != cudaSuccess) return e;
  if (after && (e = states(A.out + 1)) != cudaSuccess) return e;
  return cudaGetLastError();
}

}  // namespace

cudaError_t linattn_tc(const Launch& lc, const LinArgs& a) {
  LinTcArgs A;
  A.a = a;
  // few segments: each CTA joins the states before its own; a state updated in
  // place is read before any CTA writes it only if a kernel of its own joins
  A.a.grouped = 1;
  A.out = -1;
  for (int i = 0; i < a.npass; ++i)
    if (a.pass[i].s_out) A.out = i;
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
