// Verify attention over paged K / V of 8-bit floats (e4m3, one scale per block of tokens and kv head)
// on the 5th-generation tensor cores, without widening a single cached byte.
//
// The 8-bit MMA multiplies e4m3 by e5m2, so K and V are its B operands as they lie in the pages (TMA
// page gathers, as in the 16-bit kernels), and the accuracy lost nowhere is kept on the other side:
//   * a query row, scaled by a power of two so that its largest element lies in [2^7, 2^8), is the sum
//     of an e4m3 and an e5m2 piece, each rounded to nearest: 4 significant bits and 3 more of the remainder, with its sign
//     bfloat16's 8, exact for elements down to 2^-13 of the row's largest; those below are off by 2^-21 of it at most;
//   * S = (Q1 + Q2) K^T accumulates in fp32; K's scale multiplies the score of its token;
//   * a weight times V's scale, x_t = p_t v_t, is rounded to binary16 and cut into three e5m2 pieces (e5m2 is the upper
//     byte of binary16, so a piece is a byte of the remainder), the third rounded to nearest: 9 significant bits, off by
//     2^-9 at most, 2^-10.9 in the mean square with the rounding to binary16 (bfloat16, which the 16-bit kernels round P to:
//     2^-8 and 2^-9.3), O += (P1 + P2 + P3) V.
// The MMAs of one B tile are weight-stationary and share it: it stays in the collector, 27 cycles an MMA at 32 rows
// back to back, against 44 when each loads its own.  A tile's 8 score and 12 value MMAs come from two warps (by
// elect.sync in a converged warp; a branch on one thread costs 46 cycles an MMA), 550 of the 1,420 cycles in which
// its 32 KB can come from memory.
//
// What bounds it (one call, the plan and the combine kernel included, 12 us of it): the Llama-3-8B layer shape (64
// requests of 512 to 4096 tokens, 320 MB of K and V) takes 85 to 89 us from one board to another, 81 with the softmax
// arithmetic taken out: the stream of tiles, 5 TB/s between the first and the last (the 16-bit kernel, whose copies are
// twice as large, reaches 5.5 on this shape; what holds this one is not shown); the 70B shape (128 requests, a pool in token
// order, 469 MB) 128 to 135 us.  Contexts of 32,768 at 36 rows, 300 to 344 us by the clock the power limit leaves, are bound
// by the softmax groups, whose tiles are 64 rows wide there (211 us without their arithmetic).
//
// binary16 has no exponents to spare for V's scales, so a row's reference m' is the maximum of s_t + log2 v_t
// instead of s_t: y_t = 2^(10 + s_t - m') goes into the row's sum and x_t = y_t v_t into P, both under
// the one reference.  It is taken from an entry's first tile and kept: the tiles after it need no maximum,
// and their warps no agreement, before the weights.  They look at the x they make.  One above 2^13 has the
// group take the next tile's maximum again; one above 2^15 is past what P can hold, and the
// group takes the maximum and makes the same tile's weights again: scores and scales are held until the tile's
// verdict is read, and the issuer of the value MMAs reads it before it goes on.  m' moves, and O is rescaled, when a tile's
// maximum passes it by a factor of 16.  The least x with a bit left is 2^-26 of the row's largest (a V scale below 2^-90
// counted as 2^-90).  Where V's scales are zero or that small the x do not tell how large the y are (and 0 times a y
// past fp32 is NaN): a thread's sum of a tile above 2^112 is past the range as well.  Sums add up to 2^111 a tile then,
// 65,000 tiles of an entry before they leave fp32.
//
// Roles of the 512 threads: warps 0 and 13 TMA producers of K and of V, warp 1 issuer of the score MMAs, warp 12 of the
// value MMAs, warp 2 scales of the next tiles, warps 3, 14 and 15 query pieces of the next entry, warps 4-7 and 8-11 two softmax groups
// that take the tiles in turn, each with its own reference, sum and O, merged in the entry's epilogue: a tile's
// chain (scores, weights, pieces) is some 2,000 cycles long, and two tiles in it at a time keep up with memory.
// The plan, its work entries, partial results and bounded waits are those of the 16-bit kernels.
#pragma once
#include <cstddef>

#include "attn_tc4.cuh"

namespace spx {

constexpr int kE8Threads = 512;
constexpr int kE8QueryWarps = 3;   // 3, 14, 15
constexpr int kE8GroupWarps = 4;   // softmax warps of a group
constexpr int kE8ScaleSlots = 4;   // tiles whose scales are staged
constexpr int kE8RowSlots = 8;     // entries whose row factors are kept: the scores run four tiles (entries, at most) ahead of the softmax, the query pieces one more
constexpr int kE8NanSlots = 8;
constexpr float kE8Shift = 10.f;
constexpr float kE8Rescale = 4.f;   // under a fresh reference x <= 2^(10 + 4)
constexpr uint32_t kE8Warn = 0x7000u, kE8Redo = 0x7800u;   // 2^13, 2^15 as binary16 (its largest: 65504)
constexpr float kE8MinLog2 = -90.f;  // smaller V scales (zero too) count as this in m': under a fresh reference y <= 2^(10 + 4 + 90)
constexpr float kE8SumRedo = 5.19229686e33f;   // 2^112: 128 tokens of such y are 2^111

template <int D, int MROWS>
struct E8Cfg {
  static constexpr int kSplit = 128 / MROWS;                       // token blocks of a tile (the accumulator layout of the M = MROWS MMA): warps that share a row
  static constexpr int kTokPerThread = kTileTokens / kSplit;       // 32, 64, 128
  static constexpr int kTileBytes = kTileTokens * D;
  static constexpr int kPiece = MROWS * 128;                       // one piece of Q (D <= 128 columns) or of P (128 tokens), 128-byte rows
  static constexpr int kQBufs = MROWS == 128 ? 1 : 2, kPBufs = MROWS == 128 ? 1 : 2, kOBufs = MROWS == 128 && D == 128 ? 1 : 2;
  // The rings of K and of V: what they hold is in flight or waits, so they take all the memory that is left.  K is done
  // with as soon as its scores are issued, V waits for the softmax: two more of it.
  static constexpr int kStagesK = D == 64 ? 6 : MROWS == 32 ? 4 : 3, kStagesV = D == 64 ? 8 : MROWS == 32 ? 6 : MROWS == 64 ? 5 : 4;
  static constexpr int kColBlock = D / kSplit / 2;                 // columns of O a thread finishes
  static constexpr int kSCols = kTileTokens / kSplit, kOCols = D / kSplit;
  static constexpr int kSBufs = MROWS == 128 ? 2 : 4;              // score buffers: the scores run that many tiles ahead
  static constexpr int kColS = 0, kColO = kSBufs * kSCols;         // then kOBufs pairs of O (one of each group)
  static constexpr int kTmemNeed = kColO + 2 * kOBufs * kOCols;
  static constexpr int kTmemCols = kTmemNeed <= 128 ? 128 : kTmemNeed <= 256 ? 256 : 512;
  static_assert(kTmemNeed <= 512, "tensor memory");
  // byte offsets into shared memory, after rounding its base up to 1024
  static constexpr int kOffK = 0, kOffV = kOffK + kStagesK * kTileBytes, kOffQ = kOffV + kStagesV * kTileBytes, kOffP = kOffQ + kQBufs * 2 * kPiece;
  static constexpr int kOffKs = kOffP + kPBufs * 3 * kPiece, kOffVs = kOffKs + kE8ScaleSlots * 512, kOffLv = kOffVs + kE8ScaleSlots * 512;
  static constexpr int kOffMx = kOffLv + kE8ScaleSlots * 512, kOffL = kOffMx + 2 * 1024;
  static constexpr int kOffRef = kOffL + 2 * 1024, kOffRow = kOffRef + 2 * 2 * MROWS * 4, kOffNan = kOffRow + kE8RowSlots * MROWS * 4;
  static constexpr int kOffBar = kOffNan + kE8NanSlots * 128 * 4;
  static constexpr int kSmemBytes = kOffBar + 640 + 1024;
  static_assert(kSmemBytes <= 232448, "shared memory");
};

struct E8Barriers {
  uint64_t k_full[8], v_full[8], k_empty[8], v_empty[8], sc_full[kE8ScaleSlots], sc_empty[kE8ScaleSlots];
  uint64_t s_full[4], p_full[2], q_full[2], q_empty[2], pv_done[2], o_full[2], o_free[2], item_done[2], e_bar[2], redo_ack[2];
  uint32_t tmem_base;
  volatile int32_t abort;
  int32_t nan_any[kE8NanSlots];
  int32_t verdict[2][4];   // of a group's last weights, by phase of p_full: 0 fine, 1 near the end of P's range, 2 past it
  int32_t *dev_status;
};
static_assert(sizeof(E8Barriers) <= 640, "barrier area");

namespace e8 {

using namespace tc;

// Bounded wait of a converged warp.  What does not find the barrier completed goes on out of line: with
// the polling loops in line in some twenty places the kernel was 180 KB of code, and its warps waited for
// instructions more than for anything else.  For the same reason the outcome is not handed back: when
// a wait gives up it raises SPX_DEV_TIMEOUT and the CTA's abort flag, which ends every other wait as well, and
// every role's loop looks at the flag once a tile.
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// (the warp may sleep in it for some microseconds: polling warps take issue slots from the working ones)
__device__ __forceinline__ bool try_wait_long(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3; selp.u32 %0, 1, 0, p; }"
               : "=r"(ok) : "r"(bar), "r"(parity), "r"(20000) : "memory");
  return ok != 0;
}
__device__ __noinline__ void wait_slow(uint32_t bar, uint32_t parity, E8Barriers *bars) {
  const long long t0 = clock64();
#pragma unroll 1
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (__all_sync(0xffffffffu, try_wait_long(bar, parity))) return;
    if (__any_sync(0xffffffffu, bars->abort)) return;
    if (__any_sync(0xffffffffu, clock64() - t0 > kWaitLimitCycles)) {
      bars->abort = 1;
      atomicOr(bars->dev_status, SPX_DEV_TIMEOUT);
      return;
    }
  }
}
__device__ __forceinline__ void warp_wait(uint32_t bar, uint32_t parity, E8Barriers *bars) {
  if (!__all_sync(0xffffffffu, try_wait(bar, parity))) wait_slow(bar, parity, bars);
}
__device__ __forceinline__ void expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tma_page(uint32_t dst, const CUtensorMap *map, uint32_t bar, int c1, int c2, int page) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(map), "r"(bar), "r"(0), "r"(c1), "r"(c2), "r"(page) : "memory");
}
__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

__device__ __forceinline__ bool elect_lane() {
  uint32_t r;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(r));
  return r != 0;
}
// Weight-stationary MMAs; those in a row that multiply one B tile share it through collector buffer kBuf:
// kUse 0 fills it, 1 uses it, 2 is the last to.
#define SPX_E8_MMA(OP)                                                                                                      \
  asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.ws.cta_group::1.kind::f8f6f4" OP " [%0], %1, %2, %3, p; }" \
               ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc) : "memory")
template <int kBuf, int kUse>
__device__ __forceinline__ void mma_piece(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  if constexpr (kBuf == 0) {
    if constexpr (kUse == 0) SPX_E8_MMA(".collector::b0::fill");
    else if constexpr (kUse == 1) SPX_E8_MMA(".collector::b0::use");
    else SPX_E8_MMA(".collector::b0::lastuse");
  } else {
    if constexpr (kUse == 0) SPX_E8_MMA(".collector::b1::fill");
    else if constexpr (kUse == 1) SPX_E8_MMA(".collector::b1::use");
    else SPX_E8_MMA(".collector::b1::lastuse");
  }
}
#undef SPX_E8_MMA
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// D fp32, A e4m3 or e5m2 K-major, B e4m3
__host__ __device__ constexpr uint32_t idesc_f8(uint32_t m, uint32_t n, bool a_e5m2, bool b_mn_major) {
  return (1u << 4) | (a_e5m2 ? 1u << 7 : 0u) | (b_mn_major ? (1u << 16) : 0u) | ((n >> 3) << 17) | ((m >> 4) << 24);
}
// rows of D bytes: 128-byte swizzle for 128 columns, 64-byte swizzle for 64
template <int D>
__device__ __forceinline__ uint64_t kv_desc(uint32_t saddr) {
  constexpr uint64_t layout = D == 128 ? 2 : 4;
  return (uint64_t)((saddr >> 4) & 0x3fff) | ((uint64_t)1 << 16) | ((uint64_t)(8 * D >> 4) << 32) | ((uint64_t)1 << 46) | (layout << 61);
}
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t taddr, uint32_t (&r)[N]) {
  if constexpr (N == 8) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
  } else {
    tmem_ld<N>(taddr, r);
  }
}
template <int N>
__device__ __forceinline__ void tmem_store(uint32_t taddr, const uint32_t (&r)[N]) {
  if constexpr (N == 8) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
  } else {
    tmem_st<N>(taddr, r);
  }
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// two fp32 operations in one instruction
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint32_t max_f16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Four values, as two binary16 pairs, as the sums of an e4m3 and an e5m2 value, each rounded to nearest.
__device__ __forceinline__ void cut2(uint32_t h01, uint32_t h23, uint32_t &w1, uint32_t &w2) {
  uint16_t a, b;
  uint32_t u, v;
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(a) : "r"(h01));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(b) : "r"(h23));
  w1 = (uint32_t)a | ((uint32_t)b << 16);
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(u) : "h"(a));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(v) : "h"(b));
  u = sub_f16x2(h01, u);
  v = sub_f16x2(h23, v);
  asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(a) : "r"(u));
  asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(b) : "r"(v));
  w2 = (uint32_t)a | ((uint32_t)b << 16);
}
// Four values, as two binary16 pairs, cut into three e5m2 pieces of four bytes each.
__device__ __forceinline__ void cut3(uint32_t h01, uint32_t h23, uint32_t &w1, uint32_t &w2, uint32_t &w3) {
  w1 = __byte_perm(h01, h23, 0x7531);
  h01 = sub_f16x2(h01, h01 & 0xff00ff00u);
  h23 = sub_f16x2(h23, h23 & 0xff00ff00u);
  w2 = __byte_perm(h01, h23, 0x7531);
  h01 = sub_f16x2(h01, h01 & 0xff00ff00u);
  h23 = sub_f16x2(h23, h23 & 0xff00ff00u);
  uint16_t a, b;
  asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(a) : "r"(h01));
  asm("cvt.rn.satfinite.e5m2x2.f16x2 %0, %1;" : "=h"(b) : "r"(h23));
  w3 = (uint32_t)a | ((uint32_t)b << 16);
}

}  // namespace e8

template <int D, int MROWS>
__global__ void __launch_bounds__(kE8Threads, 1)
attn_e4m3_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, AttnParams p) {
  SPX_TL_SCOPE(kTlAttention);
  using Cfg = E8Cfg<D, MROWS>;
  using namespace e8;
  constexpr int kSplit = Cfg::kSplit, TPT = Cfg::kTokPerThread, CB = Cfg::kColBlock;
  extern __shared__ __align__(1024) unsigned char smem_dyn[];
  unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
  unsigned char *sK = smem + Cfg::kOffK, *sV = smem + Cfg::kOffV, *sQ = smem + Cfg::kOffQ, *sP = smem + Cfg::kOffP;
  float *sKs = reinterpret_cast<float *>(smem + Cfg::kOffKs), *sVs = reinterpret_cast<float *>(smem + Cfg::kOffVs);
  float *sLv = reinterpret_cast<float *>(smem + Cfg::kOffLv);      // log2 of V's scales
  float *sMx = reinterpret_cast<float *>(smem + Cfg::kOffMx);   // [2 tiles][group][kSplit][MROWS]
  float *sL = reinterpret_cast<float *>(smem + Cfg::kOffL);        // [2 entries][group][kSplit][MROWS]
  float *sRef = reinterpret_cast<float *>(smem + Cfg::kOffRef);    // [2 entries][group][MROWS]
  float *sRow = reinterpret_cast<float *>(smem + Cfg::kOffRow);    // [kE8RowSlots][MROWS]
  uint32_t *sNan = reinterpret_cast<uint32_t *>(smem + Cfg::kOffNan);  // [kE8NanSlots][128]
  E8Barriers *bars = reinterpret_cast<E8Barriers *>(smem + Cfg::kOffBar);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
#pragma unroll 1
    for (int s = 0; s < 8; ++s) { mbar_init(&bars->k_full[s], 1); mbar_init(&bars->v_full[s], 1); mbar_init(&bars->k_empty[s], 1); mbar_init(&bars->v_empty[s], 1); }
#pragma unroll 1
    for (int s = 0; s < kE8ScaleSlots; ++s) { mbar_init(&bars->sc_full[s], 1); mbar_init(&bars->sc_empty[s], kE8GroupWarps); }
#pragma unroll 1
    for (int b = 0; b < 2; ++b) {
      mbar_init(&bars->s_full[b], 1); mbar_init(&bars->s_full[b + 2], 1); mbar_init(&bars->p_full[b], kE8GroupWarps); mbar_init(&bars->q_full[b], kE8QueryWarps); mbar_init(&bars->q_empty[b], 1);
      mbar_init(&bars->pv_done[b], 1); mbar_init(&bars->o_full[b], 1); mbar_init(&bars->o_free[b], 2 * kE8GroupWarps);
      mbar_init(&bars->item_done[b], 2 * kE8GroupWarps); mbar_init(&bars->e_bar[b], kE8GroupWarps);
      mbar_init(&bars->redo_ack[b], 1);
      for (int i = 0; i < 4; ++i) bars->verdict[b][i] = 0;
    }
    bars->abort = 0;
    bars->dev_status = p.dev_status;
    for (int i = 0; i < kE8NanSlots; ++i) bars->nan_any[i] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
#pragma unroll 1
  for (int i = tid; i < kE8NanSlots * 128; i += kE8Threads) sNan[i] = 0;
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)), "n"(Cfg::kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = bars->tmem_base;

  // Everything above touched only this CTA's own resources; the plan, and what the caller's kernels before it
  // wrote, is read from here on.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // the combine kernel may take its places now, and not before: it reads the plan ahead of its own wait
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // this CTA's range of the plan: entries cta_off[c] .. cta_off[c+1] of the work list, in order
  const bool planned = !p.hdr->overflow && (int)blockIdx.x < p.hdr->n_cta;
  const int item_begin = planned ? p.cta_off[blockIdx.x] : 0;
  const int item_end = planned ? p.cta_off[blockIdx.x + 1] : 0;
  auto item_index = [&](int it) -> int { return item_begin + it < item_end ? item_begin + it : -1; };
  const int pages_per_tile = kTileTokens >> p.log2P;
  const uint32_t bar0 = smem_u32(bars);
  auto warp_wait = [&](uint32_t bar, uint32_t parity) { e8::warp_wait(bar, parity, bars); };
#define SPX_E8_BAR(member, i) (bar0 + (uint32_t)offsetof(E8Barriers, member) + 8u * (uint32_t)(i))

  if (warp == 0 || warp == 13) {
    // ------------------------------------------------------------------ producers: K (warp 0), V (warp 13)
    // One warp for both was what the tiles waited for: the copies of a tile's pages are issued one after the other,
    // some 60 cycles each, sixteen to a tile with pages of 16 tokens.
    const bool keys = warp == 0;
    const CUtensorMap *map = keys ? &kmap : &vmap;
    const uint32_t bar_full = keys ? SPX_E8_BAR(k_full, 0) : SPX_E8_BAR(v_full, 0), bar_empty = keys ? SPX_E8_BAR(k_empty, 0) : SPX_E8_BAR(v_empty, 0);
    const uint32_t ring = smem_u32(keys ? sK : sV), stages = keys ? Cfg::kStagesK : Cfg::kStagesV;
    // Tiles are walked in groups of 32/pages_per_tile so that every lane owns one page of the group:
    // one coalesced block-table read per group, a group ahead of the copies (the next entry one ahead).
    const int tiles_per_group = 32 / pages_per_tile;
    const int my_tile = lane / pages_per_tile, my_page = lane % pages_per_tile;
    struct GCursor { int it, tile0; WorkEntry e, e_next; bool valid; };
    auto open = [&](GCursor &c, int it) {
      c.it = it;
      c.valid = item_index(it) >= 0;
      if (c.valid) {
        c.tile0 = c.e.tile_begin;
        const int idx_next = item_index(it + 1);
        if (idx_next >= 0) c.e_next = p.work[idx_next];
      }
    };
    auto advance = [&](GCursor &c) {
      c.tile0 += tiles_per_group;
      if (c.tile0 >= c.e.tile_end) { c.e = c.e_next; open(c, c.it + 1); }
    };
    auto load_page = [&](const GCursor &c) -> int {
      const int tile = c.tile0 + my_tile;
      if (!c.valid || tile >= c.e.tile_end) return -1;
      const int ntok = min(kTileTokens, c.e.L - tile * kTileTokens);
      if (my_page * p.P >= ntok) return -1;
      int page = p.block_table[(int64_t)c.e.req * p.max_pages_per_req + tile * pages_per_tile + my_page];
      if (page < 0 || page >= p.num_pages) {
        page = 0;  // keep the copy in bounds; the request is flagged and its rows are voided
        atomicOr(p.dev_status, SPX_DEV_BAD_PAGE);
        p.req_bad[c.e.req] = 1;
      }
      return page;
    };
    GCursor la;
    if (item_index(0) >= 0) la.e = p.work[item_index(0)];
    open(la, 0);
    int page_la = load_page(la);
    uint32_t tc_ = 0;
    while (la.valid && !bars->abort) {
      const GCursor cur = la;
      const int page = page_la;
      advance(la);
      page_la = load_page(la);
      const int g = cur.e.g;
      for (int ti = 0; ti < tiles_per_group && cur.tile0 + ti < cur.e.tile_end; ++ti, ++tc_) {
        const int tile = cur.tile0 + ti;
        const int slot = tc_ % stages;
        const uint32_t ph = (tc_ / stages) & 1;
        const int ntok = min(kTileTokens, cur.e.L - tile * kTileTokens);
        const uint32_t bytes = (uint32_t)(((ntok + p.P - 1) >> p.log2P) << p.log2P) * D;
        const bool mine = (my_tile == ti) && page >= 0;
        warp_wait(bar_empty + 8 * slot, ph ^ 1);
        if (lane == 0) expect_tx(bar_full + 8 * slot, bytes);
        __syncwarp();
        if (mine) tma_page(ring + slot * Cfg::kTileBytes + my_page * p.P * D, map, bar_full + 8 * slot, p.head_inner ? g : 0, p.head_inner ? 0 : g, page);
      }
    }
  } else if (warp == 1 || warp == 12) {
    // ------------------------------------------------------------------ MMA issuers: scores (warp 1), values (warp 12)
    // One warp for both was the kernel's longest chain (waits, descriptors and commits included, some 46 cycles an MMA).
    const bool scores = warp == 1;
    int it = 0;
    auto tiles_of = [&](int i) -> int {
      const int idx = item_index(i);
      if (idx < 0) return 0;
      return p.work[idx].tile_end - p.work[idx].tile_begin;
    };
    int n_tiles = tiles_of(0), n_next = tiles_of(1), i = 0;
    uint32_t phase0 = 0, phase1 = 0;   // of p_full: as many as a group made weights, those it took back included
#pragma unroll 1
    for (uint32_t t = 0; item_index(it) >= 0 && !bars->abort; ++t) {
      const uint32_t stages = scores ? Cfg::kStagesK : Cfg::kStagesV;
      const int slot = t % stages;
      const uint32_t ph = (t / stages) & 1;
      const bool last = i + 1 >= n_tiles;
      if (scores) {
        constexpr uint32_t kIdesc0 = idesc_f8(MROWS, kTileTokens, false, false), kIdesc1 = idesc_f8(MROWS, kTileTokens, true, false);
        const uint32_t qb = Cfg::kQBufs == 2 ? (it & 1) : 0;
        if (i == 0) warp_wait(SPX_E8_BAR(q_full, qb), (Cfg::kQBufs == 2 ? (it >> 1) : it) & 1);
        warp_wait(SPX_E8_BAR(k_full, slot), ph);
        // the tile whose scores the buffer holds is settled when its scales are handed back
        if (t >= Cfg::kSBufs) {
          const uint32_t u = t - Cfg::kSBufs;
          warp_wait(SPX_E8_BAR(sc_empty, u % kE8ScaleSlots), (u / kE8ScaleSlots) & 1);
        }
        fence_after();
        const uint64_t qa = smem_desc(smem_u32(sQ + qb * 2 * Cfg::kPiece), 16, 1024), ka = kv_desc<D>(smem_u32(sK + slot * Cfg::kTileBytes));
        const uint32_t ts = tmem + Cfg::kColS + (t % Cfg::kSBufs) * Cfg::kSCols;
        if (elect_lane()) {
#pragma unroll
          for (int k = 0; k < D / 32; k += 2) {   // descriptors count 16-byte units: 32 columns are 2
            mma_piece<0, 0>(ts, qa + k * 2, ka + k * 2, kIdesc0, k > 0);
            mma_piece<0, 2>(ts, qa + k * 2 + (Cfg::kPiece >> 4), ka + k * 2, kIdesc1, 1);
            mma_piece<1, 0>(ts, qa + k * 2 + 2, ka + k * 2 + 2, kIdesc0, 1);
            mma_piece<1, 2>(ts, qa + k * 2 + 2 + (Cfg::kPiece >> 4), ka + k * 2 + 2, kIdesc1, 1);
          }
          commit(SPX_E8_BAR(s_full, t % Cfg::kSBufs));
          commit(SPX_E8_BAR(k_empty, slot));
          if (last) commit(SPX_E8_BAR(q_empty, qb));
        }
      } else {
        constexpr uint32_t kIdesc = idesc_f8(MROWS, D, true, true);
        constexpr int kStep = 32 * D >> 4;   // 32 tokens are 32 * D bytes of V, 32 bytes of P
        // O's buffers were last used kOBufs entries ago
        if (i == 0 && it >= Cfg::kOBufs)
          warp_wait(SPX_E8_BAR(o_free, Cfg::kOBufs == 2 ? (it & 1) : 0), (Cfg::kOBufs == 2 ? (it >> 1) - 1 : it - 1) & 1);
        warp_wait(SPX_E8_BAR(v_full, slot), ph);
        // the tile's weights: the first its group does not take back
#pragma unroll 1
        for (;;) {
          const uint32_t g = t & 1, n = g ? phase1++ : phase0++;
          warp_wait(SPX_E8_BAR(p_full, g), n & 1);
          if (*reinterpret_cast<volatile int32_t *>(&bars->verdict[g][n & 3]) != 2 || bars->abort) break;
          __syncwarp();
          if (lane == 0) arrive(SPX_E8_BAR(redo_ack, g));   // seen: the group may complete another phase
        }
        fence_after();
        const uint64_t pa = smem_desc(smem_u32(sP + (Cfg::kPBufs == 2 ? (t & 1) : 0) * 3 * Cfg::kPiece), 16, 1024), va = kv_desc<D>(smem_u32(sV + slot * Cfg::kTileBytes));
        const uint32_t to = tmem + Cfg::kColO + ((Cfg::kOBufs == 2 ? (it & 1) * 2 : 0) + (t & 1)) * Cfg::kOCols;
        if (elect_lane()) {
#pragma unroll
          for (int k = 0; k < kTileTokens / 32; k += 2) {
            mma_piece<0, 0>(to, pa + k * 2, va + k * kStep, kIdesc, (i > 1) || (k > 0));   // an entry's first two tiles begin their group's O
            mma_piece<0, 1>(to, pa + k * 2 + (Cfg::kPiece >> 4), va + k * kStep, kIdesc, 1);
            mma_piece<0, 2>(to, pa + k * 2 + 2 * (Cfg::kPiece >> 4), va + k * kStep, kIdesc, 1);
            mma_piece<1, 0>(to, pa + k * 2 + 2, va + (k + 1) * kStep, kIdesc, 1);
            mma_piece<1, 1>(to, pa + k * 2 + 2 + (Cfg::kPiece >> 4), va + (k + 1) * kStep, kIdesc, 1);
            mma_piece<1, 2>(to, pa + k * 2 + 2 + 2 * (Cfg::kPiece >> 4), va + (k + 1) * kStep, kIdesc, 1);
          }
          commit(SPX_E8_BAR(v_empty, slot));
          commit(SPX_E8_BAR(pv_done, t & 1));
          if (last) commit(SPX_E8_BAR(o_full, it & 1));
        }
      }
      __syncwarp();
      ++i;
      if (last) { ++it; i = 0; n_tiles = n_next; n_next = tiles_of(it + 1); }
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------------ scales, one float per token and tile
    // A lane owns four consecutive tokens (of one page: pages hold eight at least).  The chain table ->
    // scale of a tile is spread over two rounds, so that no load is waited for but an entry's own (the ring is
    // four tiles deep).
    int it = -1, tile = 0, tile_end = 0, req = 0, g = 0, L = 0;
    auto advance = [&]() -> bool {
      if (++tile >= tile_end) {
        const int idx = item_index(++it);
        if (idx < 0) return false;
        const WorkEntry e = p.work[idx];
        req = e.req; g = e.g; L = e.L; tile = e.tile_begin; tile_end = e.tile_end;
      }
      return true;
    };
    int page = -1, base_t = 0, base_g = 0, base_L = 0;   // of the tile whose scales are fetched next
    bool have_page = false, have_scales = false;
    float ks[4], vs[4];
#pragma unroll 1
    for (uint32_t t = 0; !bars->abort;) {
      float kn[4], vn[4];
      {
        const int left = have_page && page >= 0 ? base_L - base_t : 0;   // tokens past the end have scale zero
        const int64_t base = ((int64_t)page * p.Hkv + base_g) << (p.log2P - p.log2SB);
        const int slot = base_t & (p.P - 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          kn[i] = vn[i] = 0.f;
          if (i < left) {
            const int64_t at = base + ((slot + i) >> p.log2SB);
            kn[i] = __ldg(p.k_scales + at);
            vn[i] = __ldg(p.v_scales + at);
          }
        }
      }
      const bool next_scales = have_page;
      have_page = it < 0 || item_index(it) >= 0 ? advance() : false;
      if (have_page) {
        base_t = tile * kTileTokens + lane * 4; base_g = g; base_L = L;
        page = -1;
        if (base_t < L) {
          page = p.block_table[(int64_t)req * p.max_pages_per_req + (base_t >> p.log2P)];
          if (page < 0 || page >= p.num_pages) page = 0;   // (flagged by the producer)
        }
      }
      if (have_scales) {
        const int slot = t % kE8ScaleSlots;
        if (t >= kE8ScaleSlots) warp_wait(SPX_E8_BAR(sc_empty, slot), ((t / kE8ScaleSlots) - 1) & 1);
        float lv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) lv[i] = fmaxf(__log2f(vs[i]), kE8MinLog2);
        *reinterpret_cast<float4 *>(sKs + slot * 128 + lane * 4) = make_float4(ks[0], ks[1], ks[2], ks[3]);
        *reinterpret_cast<float4 *>(sVs + slot * 128 + lane * 4) = make_float4(vs[0], vs[1], vs[2], vs[3]);
        *reinterpret_cast<float4 *>(sLv + slot * 128 + lane * 4) = make_float4(lv[0], lv[1], lv[2], lv[3]);
        __syncwarp();
        if (lane == 0) arrive(SPX_E8_BAR(sc_full, slot));
        ++t;
      }
      if (!next_scales && !have_page) break;
      have_scales = next_scales;
#pragma unroll
      for (int i = 0; i < 4; ++i) { ks[i] = kn[i]; vs[i] = vn[i]; }
    }
  } else if (warp == 3 || warp > 13) {
    // ------------------------------------------------------------------ query pieces, an entry ahead
    // A lane owns 8 columns of a row: a pass of one warp covers 2 rows of 128 columns or 4 of 64.  Three warps,
    // each with six passes' loads in flight, turn 36 rows in one trip to memory; a single warp took 8,500
    // cycles an entry of 32 rows, the time of six tiles.
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;
    const int q_warp = warp == 3 ? 0 : warp - 13;
    const int c = lane % kLanes;
    const __nv_bfloat16 *q = reinterpret_cast<const __nv_bfloat16 *>(p.q);
    WorkEntry e, e_next;
    if (item_index(0) >= 0) e = p.work[item_index(0)];
    for (int it = 0; item_index(it) >= 0 && !bars->abort; ++it) {
      const int idx_next = item_index(it + 1);
      if (idx_next >= 0) e_next = p.work[idx_next];
      const int qb = Cfg::kQBufs == 2 ? (it & 1) : 0, uses = Cfg::kQBufs == 2 ? (it >> 1) : it;
      const int R = e.m * p.G;
      float *rows_out = sRow + (it % kE8RowSlots) * MROWS;
      unsigned char *dst = sQ + qb * 2 * Cfg::kPiece;
      auto load = [&](int row) -> uint4 {
        if (row >= R) return make_uint4(0, 0, 0, 0);
        const int j = row / p.G, hg = row - j * p.G;
        return __ldg(reinterpret_cast<const uint4 *>(q + ((int64_t)(e.q0 + j) * p.Hq + e.g * p.G + hg) * D + c * 8));
      };
      constexpr int kAhead = 6;   // passes whose loads are in flight together
      bool waited = false;
      for (int row0 = q_warp * kAhead * kRows; row0 < R || !waited; row0 += kE8QueryWarps * kAhead * kRows) {
        uint4 v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) v[u] = load(row0 + u * kRows + lane / kLanes);
        if (!waited) {
          waited = true;
          if (uses >= 1) warp_wait(SPX_E8_BAR(q_empty, qb), (uses - 1) & 1);
        }
#pragma unroll 1
        for (int u = 0; u < kAhead; ++u) {
          const int row = row0 + u * kRows + lane / kLanes;
          uint4 x = v[0];
#pragma unroll
          for (int w = 1; w < kAhead; ++w) x = u == w ? v[w] : x;
          const uint32_t w[4] = {x.x, x.y, x.z, x.w};
          uint32_t a = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) a = __vmaxu2(a, w[i] & 0x7fff7fffu);
          a = max(a & 0xffffu, a >> 16);
#pragma unroll
          for (int o = 1; o < kLanes; o <<= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
          // 2^f puts the row's largest element into [2^7, 2^8); a row that is not finite becomes NaN through its factor
          const bool finite = a < 0x7f80u;
          const int field = a == 0 ? 127 : min(261 - (int)(a >> 7), 253);
          const float mult = finite ? __uint_as_float((uint32_t)field << 23) : 0.f;
          uint32_t h[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) h[i] = finite ? pack_f16(__uint_as_float(w[i] << 16) * mult, __uint_as_float(w[i] & 0xffff0000u) * mult) : 0u;
          uint2 piece[2];
          cut2(h[0], h[1], piece[0].x, piece[1].x);
          cut2(h[2], h[3], piece[0].y, piece[1].y);
          if (row < R) {
            unsigned char *at = dst + (row >> 3) * 1024 + (row & 7) * 128 + (((c >> 1) ^ (row & 7)) << 4) + (c & 1) * 8;
#pragma unroll
            for (int i = 0; i < 2; ++i) *reinterpret_cast<uint2 *>(at + i * Cfg::kPiece) = piece[i];
            // (never zero: a hidden score is -inf, and times zero it would be NaN)
            if (c == 0) rows_out[row] = finite ? fmaxf(ldexpf(p.scale_log2, 127 - field), 1.17549435e-38f) : __int_as_float(0x7fc00000);
          }
        }
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) arrive(SPX_E8_BAR(q_full, qb));
      e = e_next;
    }
  } else {
    // ------------------------------------------------------------------ softmax / epilogue
    const int quad = warp & 3, grp = (warp - 4) >> 2;
    // the accumulator layouts of the M = 32 / 64 / 128 weight-stationary MMAs: quadrant -> (row group,
    // token block); the same split applies to the columns of O
    const int rgrp = kSplit == 4 ? 0 : kSplit == 2 ? (quad & 1) : quad;
    const int part = kSplit == 4 ? quad : kSplit == 2 ? (quad >> 1) : 0;
    const int row = rgrp * 32 + lane;                       // packed query row
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const int sm_tid = tid - 128, g_tid = sm_tid & 127;
    const int row_j = row / p.G, row_h = row - row_j * p.G;
    __nv_bfloat16 *out = reinterpret_cast<__nv_bfloat16 *>(p.out);

    uint32_t ec = 0;
    // An entry's epilogue needs both groups' sums (item_done) and both O's (o_full); it is deferred behind
    // the group's next tile, so that neither is waited for.  All eight warps run it once per entry, in
    // order and before they report the next entry done; each takes half of its quadrant's columns.
    struct Pending { bool valid; WorkEntry e; uint32_t t_first; int it; } pend;
    pend.valid = false;
    auto run_epilogue = [&]() {
      const WorkEntry &J = pend.e;
      const int it = pend.it;
      warp_wait(SPX_E8_BAR(item_done, it & 1), (it >> 1) & 1);
      warp_wait(SPX_E8_BAR(o_full, it & 1), (it >> 1) & 1);
      fence_after();
      uint32_t o[CB], o2[CB];
      const uint32_t to = tmem + Cfg::kColO + (Cfg::kOBufs == 2 ? (it & 1) * 2 : 0) * Cfg::kOCols + grp * CB + lane_addr;
      tmem_load<CB>(to, o);
      tmem_load<CB>(to + Cfg::kOCols, o2);
      wait_ld();
      // O has been read: a later entry may overwrite the buffers
      fence_before();
      __syncwarp();
      if (lane == 0) arrive(SPX_E8_BAR(o_free, Cfg::kOBufs == 2 ? (it & 1) : 0));
      float l0 = 0.f, l1 = 0.f;
      const float *sl = sL + (it & 1) * 256;
#pragma unroll
      for (int i = 0; i < kSplit; ++i) { l0 += sl[i * MROWS + row]; l1 += sl[128 + i * MROWS + row]; }
      const float ref0 = sRef[(it & 1) * 2 * MROWS + row], ref1 = sRef[(it & 1) * 2 * MROWS + MROWS + row];
      // the groups' tiles: those of parity 0 and 1 among t_first .. t_first + n - 1; an O without one is nobody's
      const bool one_tile = J.tile_end - J.tile_begin == 1;
      const bool use0 = !one_tile || (pend.t_first & 1) == 0, use1 = !one_tile || (pend.t_first & 1) == 1;
      float ref = fmaxf(ref0, ref1);
      const float w0 = ref0 == -INFINITY ? 0.f : fast_exp2(ref0 - ref), w1 = ref1 == -INFINITY ? 0.f : fast_exp2(ref1 - ref);
      // (a group without a reference has a sum of zero, or NaN)
      const float l_row = rescaled_sum(l0, ref0 == -INFINITY ? -INFINITY : ref0 - ref) + rescaled_sum(l1, ref1 == -INFINITY ? -INFINITY : ref1 - ref);
      if (l_row != l_row) ref = 0.f;   // a NaN row stays one where its chunks are merged
#pragma unroll
      for (int i = 0; i < CB; ++i) {
        const float a = use0 ? w0 * __uint_as_float(o[i]) : 0.f;
        o[i] = __float_as_uint(use1 ? fmaf(w1, __uint_as_float(o2[i]), a) : a);
      }
      const int col0 = part * Cfg::kOCols + grp * CB;
      const int nan_slot = it % kE8NanSlots;
      if (bars->nan_any[nan_slot]) {
        // columns of V with a NaN at a new position: into the rows that see it
        uint64_t hit = 0;
#pragma unroll 1
        for (int i = 0; i < CB; ++i) hit |= (uint64_t)((sNan[nan_slot * 128 + col0 + i] & ((1u << row_j) - 1)) != 0) << i;
#pragma unroll
        for (int i = 0; i < CB; ++i)
          if ((hit >> i) & 1) o[i] = 0x7fc00000u;
      }
      if (row < J.m * p.G) {
        if (J.part_slot < 0) {
          const float inv = 1.f / l_row;
          const int64_t at = (int64_t)(J.q0 + row_j) * p.Hq + J.g * p.G + row_h;
          __nv_bfloat16 *dst = out + at * D + col0;
#pragma unroll
          for (int v = 0; v < CB / 8; ++v) {
            uint4 u;
            u.x = pack_bf16(__uint_as_float(o[8 * v + 0]) * inv, __uint_as_float(o[8 * v + 1]) * inv);
            u.y = pack_bf16(__uint_as_float(o[8 * v + 2]) * inv, __uint_as_float(o[8 * v + 3]) * inv);
            u.z = pack_bf16(__uint_as_float(o[8 * v + 4]) * inv, __uint_as_float(o[8 * v + 5]) * inv);
            u.w = pack_bf16(__uint_as_float(o[8 * v + 6]) * inv, __uint_as_float(o[8 * v + 7]) * inv);
            *reinterpret_cast<uint4 *>(dst + v * 8) = u;
          }
          if (col0 == 0 && p.lse) p.lse[at] = (ref - kE8Shift + log2f(l_row)) * kLn2;
        } else {
          const int64_t slot = (int64_t)J.part_slot * p.rows_cap + row;
          float *dst = p.part_o + slot * D + col0;
#pragma unroll
          for (int v = 0; v < CB / 4; ++v)
            *reinterpret_cast<uint4 *>(dst + v * 4) = make_uint4(o[4 * v], o[4 * v + 1], o[4 * v + 2], o[4 * v + 3]);
          if (col0 == 0) p.part_ml[slot] = make_float2(ref - kE8Shift, l_row);
        }
      }
      // the slot of the fourth entry from here: nobody can be that far ahead, nor still behind its last user
      const int clear = (it + 4) % kE8NanSlots;
      if (sm_tid < 128) sNan[clear * 128 + sm_tid] = 0;
      if (sm_tid == 128) bars->nan_any[clear] = 0;
      pend.valid = false;
    };
    // One step of the loop: the verdict on the last tile's weights, then this group's next tile of the current entry (or
    // the last one again), then the epilogue of the entry before; behind the entry's last tile its sums and
    // the next entry.
    WorkEntry e, e_next;
    int it = 0;
    bool have = item_index(0) >= 0;
    if (have) e = p.work[item_index(0)];
    if (item_index(1) >= 0) e_next = p.work[item_index(1)];
    uint32_t t_first = 0;                          // the entry's first tile in the CTA's sequence
    int tile = have ? e.tile_begin + grp : 0;
    float x_ref = -INFINITY, l_sum = 0.f, row_f = 0.f;   // the reference is the same in all parts of a row
    bool first = true, need_max = true, check = false, again = false;
    uint32_t n_phase = 0, n_redo = 0;                    // p_full phases completed by this group, tiles taken back
    uint32_t last_slot = 0;
    float l_before = 0.f;
#pragma unroll 1
    while (!bars->abort) {
      if (check) {
        check = false;
        warp_wait(SPX_E8_BAR(p_full, grp), (n_phase - 1) & 1);   // (all four warps' verdicts are in)
        const int verdict = *reinterpret_cast<volatile int32_t *>(&bars->verdict[grp][(n_phase - 1) & 3]);
        if (verdict == 2) {
          warp_wait(SPX_E8_BAR(redo_ack, grp), n_redo & 1);
          ++n_redo;
          tile -= 2;
          l_sum = l_before;
          again = true;   // (once: under a fresh reference nothing passes 2^14 but what is not finite)
        } else {
          again = false;
          __syncwarp();
          if (lane == 0) arrive(SPX_E8_BAR(sc_empty, last_slot));
        }
        need_max |= verdict != 0;
      }
      // with a single pair of O's the entry's first value MMAs wait for the last epilogue, and the other
      // group's may be what this tile's P waits for: nothing is deferred there
      if (Cfg::kOBufs == 1 && pend.valid) run_epilogue();
      const bool work = have && tile < e.tile_end;
      if (work) {
        const bool valid_row = row < e.m * p.G;
        const int limit = e.L - e.m + row_j;         // last visible token of this row
        const uint32_t tc_ = t_first + (uint32_t)(tile - e.tile_begin);
        const int sc_slot = tc_ % kE8ScaleSlots;
        const int t0 = tile * kTileTokens + part * TPT;  // first token of this thread
        const bool mask_tile = tile * kTileTokens + kTileTokens - 1 > e.L - e.m;
        warp_wait(SPX_E8_BAR(sc_full, sc_slot), (tc_ / kE8ScaleSlots) & 1);
        warp_wait(SPX_E8_BAR(s_full, tc_ % Cfg::kSBufs), (tc_ / Cfg::kSBufs) & 1);
        fence_after();
        if (first) row_f = sRow[(it % kE8RowSlots) * MROWS + row];
        // 32 tokens a thread stay in registers; more are taken in chunks of 32, twice (the scores stay in tensor memory)
        constexpr int CH = 32, NCH = TPT / CH;
        uint64_t v[CH / 2];
        auto load_scores = [&](int ch) {
          uint32_t r[CH];
          tmem_load<CH>(tmem + Cfg::kColS + (tc_ % Cfg::kSBufs) * Cfg::kSCols + ch * CH + lane_addr, r);
          wait_ld();
#pragma unroll
          for (int i = 0; i < CH / 2; ++i) v[i] = pair(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
          const ulonglong2 *ks4 = reinterpret_cast<const ulonglong2 *>(sKs + sc_slot * 128 + part * TPT + ch * CH);
#pragma unroll
          for (int i = 0; i < CH / 4; ++i) {
            const ulonglong2 s = ks4[i];
            v[2 * i] = mul2(v[2 * i], s.x);
            v[2 * i + 1] = mul2(v[2 * i + 1], s.y);
          }
          if (mask_tile) {
#pragma unroll
            for (int i = 0; i < CH / 2; ++i) {
              float a, b;
              unpair(v[i], a, b);
              const int t = t0 + ch * CH + 2 * i;
              v[i] = pair(t <= limit ? a : -INFINITY, t + 1 <= limit ? b : -INFINITY);
            }
          }
        };
        float alpha = 1.f;
        if (NCH == 1 || need_max) load_scores(0);
        if (need_max) {
          float x_tile = -INFINITY;
          const uint64_t f2 = pair(row_f, row_f);
#pragma unroll 1
          for (int ch = 0;;) {
            const ulonglong2 *lv4 = reinterpret_cast<const ulonglong2 *>(sLv + sc_slot * 128 + part * TPT + ch * CH);
#pragma unroll
            for (int i = 0; i < CH / 4; ++i) {
              const ulonglong2 lv = lv4[i];
              float a, b, c, d;
              unpair(fma2(v[2 * i], f2, lv.x), a, b);
              unpair(fma2(v[2 * i + 1], f2, lv.y), c, d);
              x_tile = fmaxf(x_tile, fmaxf(fmaxf(a, b), fmaxf(c, d)));
            }
            if (++ch >= NCH) break;
            load_scores(ch);
          }
          if constexpr (kSplit > 1) {
            // agree on the row's maximum over the whole tile
            float *sm = sMx + ((ec & 1) ? 2 * 128 : 0) + grp * 128;
            sm[part * MROWS + row] = x_tile;
            __syncwarp();
            if (lane == 0) arrive(SPX_E8_BAR(e_bar, grp));
            warp_wait(SPX_E8_BAR(e_bar, grp), ec & 1);
            ++ec;
            x_tile = -INFINITY;
#pragma unroll
            for (int i = 0; i < kSplit; ++i) x_tile = fmaxf(x_tile, sm[i * MROWS + row]);
          }
          // the reference moves when it is passed by a factor of sixteen; a row without one adopts the tile's
          // (its O and its sum are zero)
          if (x_ref == -INFINITY) {
            x_ref = x_tile;
          } else if (x_tile > x_ref + kE8Rescale) {
            alpha = fast_exp2(x_ref - x_tile);
            l_sum = rescaled_sum(l_sum, x_ref - x_tile);
            x_ref = x_tile;
          }
          need_max = false;
        }
        // this group's last value MMA: its P is rewritten, its O perhaps rescaled
        if (tc_ >= 2) {
          warp_wait(SPX_E8_BAR(pv_done, grp), ((tc_ - 2) >> 1) & 1);
        }
        if (Cfg::kPBufs == 1 && tc_ >= 1) {   // one P for both groups
          warp_wait(SPX_E8_BAR(pv_done, grp ^ 1), ((tc_ - 1) >> 1) & 1);
        }
        if (__any_sync(0xffffffffu, valid_row && alpha != 1.f)) {
          fence_after();
          const uint32_t to = tmem + Cfg::kColO + ((Cfg::kOBufs == 2 ? (it & 1) * 2 : 0) + grp) * Cfg::kOCols + lane_addr;
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            uint32_t o[CB];
            tmem_load<CB>(to + h * CB, o);
            wait_ld();
#pragma unroll
            for (int i = 0; i < CB; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
            tmem_store<CB>(to + h * CB, o);
          }
          wait_st();
        }
        const float shift = x_ref == -INFINITY ? 0.f : kE8Shift - x_ref;
        unsigned char *pr = sP + (Cfg::kPBufs == 2 ? grp : 0) * 3 * Cfg::kPiece + (row >> 3) * 1024 + (row & 7) * 128;
        const uint64_t row_f2 = pair(row_f, row_f), shift2 = pair(shift, shift);
        uint64_t sum2 = 0;
        uint32_t h_max = 0;
#pragma unroll 1
        for (int ch = 0; ch < NCH; ++ch) {
          if (NCH > 1) load_scores(ch);
          const ulonglong2 *vs4 = reinterpret_cast<const ulonglong2 *>(sVs + sc_slot * 128 + part * TPT + ch * CH);
#pragma unroll
          for (int c = 0; c < CH / 16; ++c) {
            uint32_t w[3][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const ulonglong2 s = vs4[4 * c + i];
              uint32_t h[2];
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                float y0, y1;
                unpair(fma2(v[8 * c + 2 * i + u], row_f2, shift2), y0, y1);
                const uint64_t y = pair(fast_exp2(y0), fast_exp2(y1));
                sum2 = add2(sum2, y);
                unpair(mul2(y, u ? s.y : s.x), y0, y1);
                h[u] = pack_f16(y0, y1);
                h_max = max_f16x2(h_max, h[u]);
              }
              cut3(h[0], h[1], w[0][i], w[1][i], w[2][i]);
            }
            const int chunk = (part * TPT + ch * CH) / 16 + c;   // 16-byte chunk of the row: 16 tokens
#pragma unroll
            for (int i = 0; i < 3; ++i)
              *reinterpret_cast<uint4 *>(pr + i * Cfg::kPiece + ((chunk ^ (row & 7)) << 4)) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
          }
        }
        float sum_lo, sum_hi;
        unpair(sum2, sum_lo, sum_hi);
        const float y_sum = sum_lo + sum_hi;
        l_before = l_sum;
        l_sum += y_sum;
        // the verdict: x is not negative, so binary16 patterns order like values (NaNs do not count)
        const uint32_t x_top = y_sum > kE8SumRedo ? 0xffffu : max(h_max & 0xffffu, h_max >> 16);
        const bool past = __any_sync(0xffffffffu, valid_row && x_top > kE8Redo), near = __any_sync(0xffffffffu, valid_row && x_top > kE8Warn);
        if (lane == 0 && near) atomicMax(&bars->verdict[grp][n_phase & 3], past && !again ? 2 : 1);
        if (g_tid == 0) bars->verdict[grp][(n_phase + 2) & 3] = 0;   // read by everybody: the group is two phases on
        if (mask_tile) {
          // V at the end of the request, as its value MMA must see it: slots past the end are zero (they
          // hold an earlier tile's or nobody's bytes, and 0 * NaN is NaN), and a NaN at a position that some
          // rows do not see is taken out and left to the epilogue of those that do
          const int ntok = min(kTileTokens, e.L - tile * kTileTokens);
          const int hidden = max(0, e.L - e.m + 1 - tile * kTileTokens);   // first token of the tile not seen by every row
          const int slot = tc_ % Cfg::kStagesV;
          warp_wait(SPX_E8_BAR(v_full, slot), (tc_ / Cfg::kStagesV) & 1);
          unsigned char *vt = sV + slot * Cfg::kTileBytes;
#pragma unroll 1
          for (int i = g_tid; i < (kTileTokens - ntok) * (D / 16); i += 128)
            *reinterpret_cast<uint4 *>(vt + ntok * D + i * 16) = make_uint4(0, 0, 0, 0);
#pragma unroll 1
          for (int i = g_tid; i < (ntok - hidden) * (D / 16); i += 128) {
            const int tok = hidden + i / (D / 16), ch = i % (D / 16);
            uint4 *at = reinterpret_cast<uint4 *>(vt + tok * D + ch * 16);
            const uint4 v = *at;
            const uint32_t any = __vcmpeq4(v.x & 0x7f7f7f7fu, 0x7f7f7f7fu) | __vcmpeq4(v.y & 0x7f7f7f7fu, 0x7f7f7f7fu) |
                                 __vcmpeq4(v.z & 0x7f7f7f7fu, 0x7f7f7f7fu) | __vcmpeq4(v.w & 0x7f7f7f7fu, 0x7f7f7f7fu);
            if (any) {
              // logical columns of this chunk under the swizzle
              const int col = (D == 128 ? ch ^ (tok & 7) : ch ^ ((tok >> 1) & 3)) * 16;
              const uint32_t bit = 1u << (tile * kTileTokens + tok - (e.L - e.m + 1));   // rows j > this position's index see it
              unsigned char *bytes = reinterpret_cast<unsigned char *>(at);
#pragma unroll 1
              for (int k = 0; k < 16; ++k)
                if ((bytes[k] & 0x7f) == 0x7f) {
                  bytes[k] = 0;
                  atomicOr(&sNan[(it % kE8NanSlots) * 128 + col + k], bit);
                }
              bars->nan_any[it % kE8NanSlots] = 1;
            }
          }
        }
        fence_async_smem();
        fence_before();
        __syncwarp();
        if (lane == 0) arrive(SPX_E8_BAR(p_full, grp));
        ++n_phase;
        check = true;
        last_slot = sc_slot;
        first = false;
        tile += 2;
      }
      if (Cfg::kOBufs == 2 && pend.valid) run_epilogue();
      if (!have) break;
      if (!work) {
        sL[(it & 1) * 256 + grp * 128 + part * MROWS + row] = l_sum;
        if (part == 0) sRef[(it & 1) * 2 * MROWS + grp * MROWS + row] = x_ref;
        __syncwarp();
        if (lane == 0) arrive(SPX_E8_BAR(item_done, it & 1));
        pend.valid = true; pend.e = e; pend.t_first = t_first; pend.it = it;
        t_first += (uint32_t)(e.tile_end - e.tile_begin);
        ++it;
        have = item_index(it) >= 0;
        e = e_next;
        if (item_index(it + 1) >= 0) e_next = p.work[item_index(it + 1)];
        if (have) tile = e.tile_begin + (int)((t_first ^ (uint32_t)grp) & 1);
        x_ref = -INFINITY; l_sum = 0.f;
        first = need_max = true;
      }
    }
  }

#undef SPX_E8_BAR
  // ---------------------------------------------------------------------- teardown
  __syncwarp();
  if (bars->abort) {
#pragma unroll 1
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  }
  fence_before();
  __syncthreads();
  if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Cfg::kTmemCols) : "memory");
  }
}

}  // namespace spx
