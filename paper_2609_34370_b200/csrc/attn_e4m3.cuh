// Verify attention over paged K / V of 8-bit floats (e4m3, one scale per block of tokens and kv head)
// on the 5th-generation tensor cores, without widening a single cached byte.
//
// The 8-bit MMA multiplies e4m3 by e5m2, so K and V are its B operands as they lie in the pages (TMA
// page gathers, as in the 16-bit kernels), and the accuracy lost nowhere is kept on the other side:
//   * a query row, scaled by a power of two so that its largest element lies in [2^14, 2^15), is the
//     exact sum of three e5m2 pieces: e5m2 is the upper byte of binary16, so each piece is a byte of
//     the remainder, and 8 significant bits are 3 + 3 + 2 (elements below 2^-24 of the largest lose
//     bits that its products round away);
//   * S = (Q1 + Q2 + Q3) K^T accumulates in fp32; K's scale multiplies the score of its token;
//   * a weight times V's scale, x_t = p_t v_t, is rounded to binary16 and cut the same way, the third
//     piece rounded to nearest: 9 significant bits and a sign, half a step off by 2^-10 at most
//     (bfloat16, which the 16-bit kernels round P to: 2^-9), O += (P1 + P2 + P3) V.
// Three weight-stationary MMAs share one B tile, which stays in the collector: 27 cycles an MMA at
// 32 rows, against 44 when each loads its own, and against 46 when they are issued from a branch on
// one thread instead of by elect.sync in a converged warp.  24 of them take 650 of the 1,420 cycles a tile's
// 32 KB need from memory: the kernel stays bound by HBM.
//
// binary16 has no exponents to spare for V's scales, so a row keeps two references: m for the sum of
// the weights, and m' for x, the running maximum of s_t + log2 v_t: x_t = 2^13 * 2^(s_t + log2 v_t - m').
// Within a tile whose scales lie within a factor of 16 of each other the bound max s + max log2 v
// stands for the maximum; other tiles take it element by element.  m' moves when it is passed by a
// factor of 4, which rescales O.  The least weight with a byte left is then 2^-29 of the largest.
//
// Roles of the 384 threads: warp 0 TMA producer, warp 1 MMA issuer, warp 2 scales of the next tiles,
// warp 3 query pieces of the next entry, warps 4-11 softmax: a lane quadrant belongs to two warps, each
// with half of the quadrant's tokens.  The plan, its work entries, partial results and bounded waits
// are those of the 16-bit kernels.
#pragma once
#include "attn_tc4.cuh"

namespace spx {

constexpr int kE8Threads = 384;
constexpr int kE8SoftmaxWarps = 8;
constexpr int kE8ScaleSlots = 4;   // tiles whose scales are staged
constexpr int kE8RowSlots = 8;     // entries whose row factors are kept: the query warp is at most four entries ahead of the softmax
constexpr int kE8NanSlots = 4;
constexpr float kE8Shift = 13.f;   // x <= 2^(13 + 2) stays below binary16's 65504
constexpr float kE8Rescale = 2.f;
constexpr float kE8MinLog2 = -110.f;  // smaller V scales count as this in m', so that 2^(13 + m - m') stays finite

template <int D, int MROWS>
struct E8Cfg {
  static constexpr int kSplit = 128 / MROWS;                       // token blocks of a tile (the accumulator layout of the M = MROWS MMA)
  static constexpr int kParts = 2 * kSplit;                        // softmax warps that share a row
  static constexpr int kTokPerThread = kTileTokens / kParts;       // 16, 32, 64
  static constexpr int kTileBytes = kTileTokens * D;
  static constexpr int kPiece = MROWS * 128;                       // one piece of Q (D <= 128 columns) or of P (128 tokens), 128-byte rows
  static constexpr int kQBufs = MROWS == 128 ? 1 : 2, kPBufs = MROWS == 128 ? 1 : 2;
  static constexpr int kStages = MROWS == 32 ? 4 : 3;
  static constexpr int kColBlock = D / kSplit / 2;                 // columns of O a thread holds
  static constexpr int kSCols = kTileTokens / kSplit, kOCols = D / kSplit;
  static constexpr int kColS = 0, kColO = 2 * kSCols;
  static constexpr int kTmemCols = kColO + 2 * kOCols <= 128 ? 128 : kColO + 2 * kOCols <= 256 ? 256 : 512;
  // byte offsets into shared memory, after rounding its base up to 1024
  static constexpr int kOffK = 0, kOffV = kOffK + kStages * kTileBytes, kOffQ = kOffV + kStages * kTileBytes, kOffP = kOffQ + kQBufs * 3 * kPiece;
  static constexpr int kOffKs = kOffP + kPBufs * 3 * kPiece, kOffVs = kOffKs + kE8ScaleSlots * 512, kOffVr = kOffVs + kE8ScaleSlots * 512;
  static constexpr int kOffMx = kOffVr + kE8ScaleSlots * 16, kOffMx2 = kOffMx + 2 * 1024, kOffL = kOffMx2 + 2 * 1024;
  static constexpr int kOffRow = kOffL + 2 * 1024, kOffNan = kOffRow + kE8RowSlots * MROWS * 4, kOffBar = kOffNan + kE8NanSlots * 128 * 4;
  static constexpr int kSmemBytes = kOffBar + 512 + 1024;
  static_assert(kSmemBytes <= 232448, "shared memory");
};

struct E8Barriers {
  uint64_t k_full[4], v_full[4], k_empty[4], v_empty[4], sc_full[kE8ScaleSlots], sc_empty[kE8ScaleSlots];
  uint64_t s_full[2], p_full[2], q_full[2], q_empty[2], pv_done[2], o_free[2], e_bar;
  uint32_t tmem_base;
  volatile int32_t abort;
  int32_t nan_any[kE8NanSlots];
};
static_assert(sizeof(E8Barriers) <= 512, "barrier area");

namespace e8 {

using namespace tc;

// Bounded wait of a converged warp; the outcome is shared, so that a warp never diverges around the
// .sync.aligned instructions.  What does not find the barrier completed goes on out of line: with the
// polling loops in line in some twenty places the kernel was 180 KB of code, and its warps waited for
// instructions more than for anything else.
__device__ __noinline__ bool wait_slow(uint64_t *b, uint32_t parity, E8Barriers *bars, int32_t *dev_status) {
  const long long t0 = clock64();
#pragma unroll 1
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (__all_sync(0xffffffffu, mbar_try_wait(b, parity))) return true;
    if (__any_sync(0xffffffffu, bars->abort)) return false;
    if (__any_sync(0xffffffffu, clock64() - t0 > kWaitLimitCycles)) {
      bars->abort = 1;
      atomicOr(dev_status, SPX_DEV_TIMEOUT);
      return false;
    }
  }
}
__device__ __forceinline__ bool warp_wait(uint64_t *b, uint32_t parity, E8Barriers *bars, int32_t *dev_status) {
  if (__all_sync(0xffffffffu, mbar_try_wait(b, parity))) return true;
  return wait_slow(b, parity, bars, dev_status);
}

// Weight-stationary MMA, A e5m2, B e4m3; three of them in a row multiply one B tile, which the first
// leaves in collector buffer kBuf.  One elected lane issues.
__device__ __forceinline__ bool elect_lane() {
  uint32_t r;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(r));
  return r != 0;
}
#define SPX_E8_MMA(OP)                                                                                                      \
  asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.ws.cta_group::1.kind::f8f6f4" OP " [%0], %1, %2, %3, p; }" \
               ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(acc) : "memory")
template <int kBuf, int kPieceIdx>
__device__ __forceinline__ void mma_piece(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  if constexpr (kBuf == 0) {
    if constexpr (kPieceIdx == 0) SPX_E8_MMA(".collector::b0::fill");
    else if constexpr (kPieceIdx == 1) SPX_E8_MMA(".collector::b0::use");
    else SPX_E8_MMA(".collector::b0::lastuse");
  } else {
    if constexpr (kPieceIdx == 0) SPX_E8_MMA(".collector::b1::fill");
    else if constexpr (kPieceIdx == 1) SPX_E8_MMA(".collector::b1::use");
    else SPX_E8_MMA(".collector::b1::lastuse");
  }
}
#undef SPX_E8_MMA
// D fp32, A e5m2 K-major, B e4m3
__host__ __device__ constexpr uint32_t idesc_f8(uint32_t m, uint32_t n, bool b_mn_major) {
  return (1u << 4) | (1u << 7) | (b_mn_major ? (1u << 16) : 0u) | ((n >> 3) << 17) | ((m >> 4) << 24);
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
  // the combine kernel may take its places now (see attn_tc4_kernel)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  using Cfg = E8Cfg<D, MROWS>;
  using namespace e8;
  constexpr int kSplit = Cfg::kSplit, kParts = Cfg::kParts, TPT = Cfg::kTokPerThread, CB = Cfg::kColBlock;
  extern __shared__ __align__(1024) unsigned char smem_dyn[];
  unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
  unsigned char *sK = smem + Cfg::kOffK, *sV = smem + Cfg::kOffV, *sQ = smem + Cfg::kOffQ, *sP = smem + Cfg::kOffP;
  float *sKs = reinterpret_cast<float *>(smem + Cfg::kOffKs), *sVs = reinterpret_cast<float *>(smem + Cfg::kOffVs);
  float2 *sVr = reinterpret_cast<float2 *>(smem + Cfg::kOffVr);    // per tile: (log2 of the largest V scale, 1 if all are within a factor of 16)
  float *sMx = reinterpret_cast<float *>(smem + Cfg::kOffMx), *sMx2 = reinterpret_cast<float *>(smem + Cfg::kOffMx2);   // [2 tiles][kParts][MROWS]
  float *sL = reinterpret_cast<float *>(smem + Cfg::kOffL);        // [2 entries][kParts][MROWS]
  float *sRow = reinterpret_cast<float *>(smem + Cfg::kOffRow);    // [kE8RowSlots][MROWS]
  uint32_t *sNan = reinterpret_cast<uint32_t *>(smem + Cfg::kOffNan);  // [kE8NanSlots][128]
  E8Barriers *bars = reinterpret_cast<E8Barriers *>(smem + Cfg::kOffBar);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
#pragma unroll 1
    for (int s = 0; s < 4; ++s) { mbar_init(&bars->k_full[s], 1); mbar_init(&bars->v_full[s], 1); mbar_init(&bars->k_empty[s], 1); mbar_init(&bars->v_empty[s], 1); }
#pragma unroll 1
    for (int s = 0; s < kE8ScaleSlots; ++s) { mbar_init(&bars->sc_full[s], 1); mbar_init(&bars->sc_empty[s], kE8SoftmaxWarps); }
#pragma unroll 1
    for (int b = 0; b < 2; ++b) {
      mbar_init(&bars->s_full[b], 1); mbar_init(&bars->p_full[b], kE8SoftmaxWarps); mbar_init(&bars->q_full[b], 1); mbar_init(&bars->q_empty[b], 1);
      mbar_init(&bars->pv_done[b], 1); mbar_init(&bars->o_free[b], kE8SoftmaxWarps);
    }
    mbar_init(&bars->e_bar, kE8SoftmaxWarps);
    bars->abort = 0;
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

  // this CTA's range of the plan: entries cta_off[c] .. cta_off[c+1] of the work list, in order
  const bool planned = !p.hdr->overflow && (int)blockIdx.x < p.hdr->n_cta;
  const int item_begin = planned ? p.cta_off[blockIdx.x] : 0;
  const int item_end = planned ? p.cta_off[blockIdx.x + 1] : 0;
  auto item_index = [&](int it) -> int { return item_begin + it < item_end ? item_begin + it : -1; };
  const int pages_per_tile = kTileTokens >> p.log2P;
  auto warp_wait = [&](uint64_t *bar, uint32_t parity) -> bool { return e8::warp_wait(bar, parity, bars, p.dev_status); };

  if (warp == 0) {
    // ------------------------------------------------------------------ producer
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
    bool ok = true;
    while (la.valid && ok && !bars->abort) {
      const GCursor cur = la;
      const int page = page_la;
      advance(la);
      page_la = load_page(la);
      const int g = cur.e.g;
      for (int ti = 0; ti < tiles_per_group && cur.tile0 + ti < cur.e.tile_end; ++ti, ++tc_) {
        const int tile = cur.tile0 + ti;
        const int slot = tc_ % Cfg::kStages;
        const uint32_t ph = (tc_ / Cfg::kStages) & 1;
        const int ntok = min(kTileTokens, cur.e.L - tile * kTileTokens);
        const uint32_t bytes = (uint32_t)(((ntok + p.P - 1) >> p.log2P) << p.log2P) * D;
        const bool mine = (my_tile == ti) && page >= 0;
        ok = warp_wait(&bars->k_empty[slot], ph ^ 1);
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(&bars->k_full[slot], bytes);
        if (mine) tma_load_4d(smem_u32(sK + slot * Cfg::kTileBytes + my_page * p.P * D), &kmap, &bars->k_full[slot], 0, p.head_inner ? g : 0, p.head_inner ? 0 : g, page);
        ok = warp_wait(&bars->v_empty[slot], ph ^ 1);
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(&bars->v_full[slot], bytes);
        if (mine) tma_load_4d(smem_u32(sV + slot * Cfg::kTileBytes + my_page * p.P * D), &vmap, &bars->v_full[slot], 0, p.head_inner ? g : 0, p.head_inner ? 0 : g, page);
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (the whole warp, converged)
    constexpr uint32_t kIdescQK = idesc_f8(MROWS, kTileTokens, false);
    constexpr uint32_t kIdescPV = idesc_f8(MROWS, D, true);
    // two cursors over the CTA's flat tile sequence: the score MMAs run one tile ahead of the value
    // MMAs, across entries too
    struct Cursor { int it, n_tiles, n_tiles_next, i; uint32_t t; bool valid; };
    auto tiles_of = [&](int it) -> int {
      const int idx = item_index(it);
      if (idx < 0) return 0;
      return p.work[idx].tile_end - p.work[idx].tile_begin;
    };
    auto open_item = [&](Cursor &c) {
      c.valid = item_index(c.it) >= 0;
      c.i = 0;
      c.n_tiles_next = tiles_of(c.it + 1);
    };
    auto advance = [&](Cursor &c) {
      ++c.t;
      if (++c.i >= c.n_tiles) { ++c.it; c.n_tiles = c.n_tiles_next; open_item(c); }
    };
    Cursor qk{0, 0, 0, 0, 0, false}, pv{0, 0, 0, 0, 0, false};
    qk.n_tiles = pv.n_tiles = tiles_of(0);
    open_item(qk);
    open_item(pv);
    bool ok = true;
    auto issue_qk = [&]() -> bool {
      const uint32_t t = qk.t, qb = Cfg::kQBufs == 2 ? (qk.it & 1) : 0;
      if (qk.i == 0 && !warp_wait(&bars->q_full[qb], (Cfg::kQBufs == 2 ? (qk.it >> 1) : qk.it) & 1)) return false;
      const int slot = t % Cfg::kStages;
      if (!warp_wait(&bars->k_full[slot], (t / Cfg::kStages) & 1)) return false;
      fence_after();
      const uint64_t qa = smem_desc(smem_u32(sQ + qb * 3 * Cfg::kPiece), 16, 1024), ka = kv_desc<D>(smem_u32(sK + slot * Cfg::kTileBytes));
      const uint32_t ts = tmem + Cfg::kColS + (t & 1) * Cfg::kSCols;
      if (elect_lane()) {
#pragma unroll
      for (int k = 0; k < D / 32; k += 2) {   // descriptors count 16-byte units: 32 columns are 2
        mma_piece<0, 0>(ts, qa + k * 2, ka + k * 2, kIdescQK, k > 0);
        mma_piece<0, 1>(ts, qa + k * 2 + (Cfg::kPiece >> 4), ka + k * 2, kIdescQK, 1);
        mma_piece<0, 2>(ts, qa + k * 2 + 2 * (Cfg::kPiece >> 4), ka + k * 2, kIdescQK, 1);
        mma_piece<1, 0>(ts, qa + k * 2 + 2, ka + k * 2 + 2, kIdescQK, 1);
        mma_piece<1, 1>(ts, qa + k * 2 + 2 + (Cfg::kPiece >> 4), ka + k * 2 + 2, kIdescQK, 1);
        mma_piece<1, 2>(ts, qa + k * 2 + 2 + 2 * (Cfg::kPiece >> 4), ka + k * 2 + 2, kIdescQK, 1);
      }
      mma_commit(&bars->s_full[t & 1]);
      mma_commit(&bars->k_empty[slot]);
      if (qk.i + 1 >= qk.n_tiles) mma_commit(&bars->q_empty[qb]);  // last score MMA of the entry
      }
      __syncwarp();
      advance(qk);
      return true;
    };
    if (qk.valid) ok = issue_qk();
    while (ok && pv.valid && !bars->abort) {
      if (qk.valid) ok = issue_qk();
      if (!ok) break;
      const uint32_t t = pv.t;
      ok = warp_wait(&bars->p_full[t & 1], (t >> 1) & 1);
      // the O buffer of this entry's parity was last used two entries ago
      if (ok && pv.i == 0 && pv.it >= 2) ok = warp_wait(&bars->o_free[pv.it & 1], ((pv.it >> 1) - 1) & 1);
      const int slot = t % Cfg::kStages;
      if (ok) ok = warp_wait(&bars->v_full[slot], (t / Cfg::kStages) & 1);
      if (!ok) break;
      fence_after();
      const uint64_t pa = smem_desc(smem_u32(sP + (Cfg::kPBufs == 2 ? (t & 1) : 0) * 3 * Cfg::kPiece), 16, 1024), va = kv_desc<D>(smem_u32(sV + slot * Cfg::kTileBytes));
      const uint32_t to = tmem + Cfg::kColO + (pv.it & 1) * Cfg::kOCols;
      if (elect_lane()) {
#pragma unroll
      for (int k = 0; k < kTileTokens / 32; k += 2) {   // 32 tokens are 32 * D bytes of V, 32 bytes of P
        constexpr int kStep = 32 * D >> 4;
        mma_piece<0, 0>(to, pa + k * 2, va + k * kStep, kIdescPV, (pv.i > 0) || (k > 0));
        mma_piece<0, 1>(to, pa + k * 2 + (Cfg::kPiece >> 4), va + k * kStep, kIdescPV, 1);
        mma_piece<0, 2>(to, pa + k * 2 + 2 * (Cfg::kPiece >> 4), va + k * kStep, kIdescPV, 1);
        mma_piece<1, 0>(to, pa + k * 2 + 2, va + (k + 1) * kStep, kIdescPV, 1);
        mma_piece<1, 1>(to, pa + k * 2 + 2 + (Cfg::kPiece >> 4), va + (k + 1) * kStep, kIdescPV, 1);
        mma_piece<1, 2>(to, pa + k * 2 + 2 + 2 * (Cfg::kPiece >> 4), va + (k + 1) * kStep, kIdescPV, 1);
      }
      mma_commit(&bars->v_empty[slot]);
      mma_commit(&bars->pv_done[t & 1]);
      }
      __syncwarp();
      advance(pv);
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------------ scales, one float per token and tile
    // A lane owns four consecutive tokens (of one page: pages hold eight at least).  The chain table ->
    // scale of a tile is spread over two iterations, so that no load is waited for.
    struct TCursor { int it, tile; WorkEntry e, e_next; bool valid; };
    auto open = [&](TCursor &c, int it) {
      c.it = it;
      c.valid = item_index(it) >= 0;
      if (c.valid) {
        c.tile = c.e.tile_begin;
        const int idx_next = item_index(it + 1);
        if (idx_next >= 0) c.e_next = p.work[idx_next];
      }
    };
    auto advance = [&](TCursor &c) {
      if (!c.valid) return;
      if (++c.tile >= c.e.tile_end) { c.e = c.e_next; open(c, c.it + 1); }
    };
    auto load_page = [&](const TCursor &c) -> int {
      const int t = c.tile * kTileTokens + lane * 4;
      if (!c.valid || t >= c.e.L) return -1;
      const int page = p.block_table[(int64_t)c.e.req * p.max_pages_per_req + (t >> p.log2P)];
      return page < 0 || page >= p.num_pages ? 0 : page;   // (flagged by the producer)
    };
    auto load_scales = [&](const TCursor &c, int page, float (&ks)[4], float (&vs)[4]) {
      const int t = c.tile * kTileTokens + lane * 4;
      const int64_t base = ((int64_t)page * p.Hkv + c.e.g) << (p.log2P - p.log2SB);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ks[i] = vs[i] = 0.f;   // tokens past the end
        if (page >= 0 && t + i < c.e.L) {
          const int64_t at = base + (((t + i) & (p.P - 1)) >> p.log2SB);
          ks[i] = __ldg(p.k_scales + at);
          vs[i] = __ldg(p.v_scales + at);
        }
      }
    };
    TCursor cur;
    if (item_index(0) >= 0) cur.e = p.work[item_index(0)];
    open(cur, 0);
    float ks[4], vs[4], ks_next[4], vs_next[4];
    const int page0 = load_page(cur);
    TCursor next = cur;
    advance(next);
    int page_next = load_page(next);
    load_scales(cur, page0, ks, vs);
    bool valid = cur.valid;
    for (uint32_t t = 0; valid && !bars->abort; ++t) {
      const bool valid_next = next.valid;
      load_scales(next, page_next, ks_next, vs_next);
      advance(next);
      page_next = load_page(next);
      const int slot = t % kE8ScaleSlots;
      if (t >= kE8ScaleSlots && !warp_wait(&bars->sc_empty[slot], ((t / kE8ScaleSlots) - 1) & 1)) break;
      *reinterpret_cast<float4 *>(sKs + slot * 128 + lane * 4) = make_float4(ks[0], ks[1], ks[2], ks[3]);
      *reinterpret_cast<float4 *>(sVs + slot * 128 + lane * 4) = make_float4(vs[0], vs[1], vs[2], vs[3]);
      // positive floats order like their patterns
      uint32_t hi = 0, lo = 0xffffffffu;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t b = __float_as_uint(vs[i]);
        hi = max(hi, b);
        if (b != 0) lo = min(lo, b);
      }
      const float v_max = __uint_as_float(__reduce_max_sync(0xffffffffu, hi)), v_min = __uint_as_float(__reduce_min_sync(0xffffffffu, lo));
      if (lane == 0) sVr[slot] = make_float2(fmaxf(__log2f(v_max), kE8MinLog2), v_max == 0.f || v_max * 0.0625f <= v_min ? 1.f : 0.f);
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->sc_full[slot]);
      valid = valid_next;
#pragma unroll
      for (int i = 0; i < 4; ++i) { ks[i] = ks_next[i]; vs[i] = vs_next[i]; }
    }
  } else if (warp == 3) {
    // ------------------------------------------------------------------ query pieces, an entry ahead
    // A lane owns 8 columns of a row: a pass covers 2 rows of 128 columns or 4 of 64.
    constexpr int kLanes = D / 8, kRows = 32 / kLanes;
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
      unsigned char *dst = sQ + qb * 3 * Cfg::kPiece;
      auto load = [&](int row) -> uint4 {
        if (row >= R) return make_uint4(0, 0, 0, 0);
        const int j = row / p.G, hg = row - j * p.G;
        return __ldg(reinterpret_cast<const uint4 *>(q + ((int64_t)(e.q0 + j) * p.Hq + e.g * p.G + hg) * D + c * 8));
      };
      constexpr int kAhead = 4;   // passes whose loads are in flight together
      bool waited = false;
      for (int row0 = 0; row0 < R; row0 += kAhead * kRows) {
        uint4 v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) v[u] = load(row0 + u * kRows + lane / kLanes);
        if (!waited) {
          waited = true;
          if (uses >= 1 && !warp_wait(&bars->q_empty[qb], (uses - 1) & 1)) break;
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          const int row = row0 + u * kRows + lane / kLanes;
          const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
          uint32_t a = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) a = __vmaxu2(a, w[i] & 0x7fff7fffu);
          a = max(a & 0xffffu, a >> 16);
#pragma unroll
          for (int o = 1; o < kLanes; o <<= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
          // 2^f puts the row's largest element into [2^14, 2^15); a row that is not finite becomes NaN through its factor
          const bool finite = a < 0x7f80u;
          const int field = a == 0 ? 127 : min(268 - (int)(a >> 7), 253);
          const float mult = finite ? __uint_as_float((uint32_t)field << 23) : 0.f;
          uint32_t h[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) h[i] = finite ? pack_f16(__uint_as_float(w[i] << 16) * mult, __uint_as_float(w[i] & 0xffff0000u) * mult) : 0u;
          uint2 piece[3];
          cut3(h[0], h[1], piece[0].x, piece[1].x, piece[2].x);
          cut3(h[2], h[3], piece[0].y, piece[1].y, piece[2].y);
          if (row < R) {
            unsigned char *at = dst + (row >> 3) * 1024 + (row & 7) * 128 + (((c >> 1) ^ (row & 7)) << 4) + (c & 1) * 8;
#pragma unroll
            for (int i = 0; i < 3; ++i) *reinterpret_cast<uint2 *>(at + i * Cfg::kPiece) = piece[i];
            // (never zero: a hidden score is -inf, and times zero it would be NaN)
            if (c == 0) rows_out[row] = finite ? fmaxf(ldexpf(p.scale_log2, 127 - field), 1.17549435e-38f) : __int_as_float(0x7fc00000);
          }
        }
      }
      if (bars->abort) break;
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->q_full[qb]);
      e = e_next;
    }
  } else {
    // ------------------------------------------------------------------ softmax / epilogue
    const int quad = warp & 3, half = (warp - 4) >> 2;
    // the accumulator layouts of the M = 32 / 64 / 128 weight-stationary MMAs: quadrant -> (row group,
    // token block); the same split applies to the columns of O.  Two warps halve a quadrant's columns.
    const int rgrp = kSplit == 4 ? 0 : kSplit == 2 ? (quad & 1) : quad;
    const int tblk = kSplit == 4 ? quad : kSplit == 2 ? (quad >> 1) : 0;
    const int row = rgrp * 32 + lane;                       // packed query row
    const int part = tblk * 2 + half;                       // this warp's share of the row: tokens and output columns
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const int sm_tid = tid - 128;                           // 0 .. 255
    __nv_bfloat16 *out = reinterpret_cast<__nv_bfloat16 *>(p.out);

    uint32_t tc_ = 0, qc = 0, ec = 0;
    bool ok = true;
    // bounded barrier among the softmax warps (a named barrier could not time out)
    auto softmax_sync = [&]() -> bool {
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->e_bar);
      const bool r = warp_wait(&bars->e_bar, ec & 1);
      ++ec;
      return r;
    };
    // The sums of a row's parts are merged through sL (written at the end of the entry's last tile, visible
    // after the next bounded barrier); each thread then finishes its columns.
    struct Pending { bool valid; WorkEntry e; float m_ref, x_ref; uint32_t last_tc, qc; } pend;
    pend.valid = false;
    auto run_epilogue = [&]() -> bool {
      const WorkEntry &J = pend.e;
      const float *sl = sL + (pend.qc & 1) * 256;
      float l_row = 0.f;
#pragma unroll
      for (int i = 0; i < kParts; ++i) l_row += sl[i * MROWS + row];
      if (!warp_wait(&bars->pv_done[pend.last_tc & 1], (pend.last_tc >> 1) & 1)) return false;
      fence_after();
      uint32_t o[CB];
      tmem_load<CB>(tmem + Cfg::kColO + (pend.qc & 1) * Cfg::kOCols + half * CB + lane_addr, o);
      wait_ld();
      // O has been read: the entry after next may overwrite this buffer
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars->o_free[pend.qc & 1]);
      const int j = row / p.G, hg = row - j * p.G;
      const int nan_slot = pend.qc % kE8NanSlots;
      if (bars->nan_any[nan_slot]) {
        // columns of V with a NaN at a new position: into the rows that see it
#pragma unroll
        for (int i = 0; i < CB; ++i)
          if (sNan[nan_slot * 128 + part * CB + i] & ((1u << j) - 1)) o[i] = 0x7fc00000u;
      }
      if (row < J.m * p.G) {
        // from x's reference to the weights' (a row with no value above zero so far: its O is zero)
        const float f = pend.x_ref == -INFINITY ? 0.f : exp2f(pend.x_ref - kE8Shift - pend.m_ref);
        if (J.part_slot < 0) {
          const float inv = f / l_row;
          __nv_bfloat16 *dst = out + ((int64_t)(J.q0 + j) * p.Hq + J.g * p.G + hg) * D + part * CB;
#pragma unroll
          for (int v = 0; v < CB / 8; ++v) {
            uint4 u;
            u.x = pack_bf16(__uint_as_float(o[8 * v + 0]) * inv, __uint_as_float(o[8 * v + 1]) * inv);
            u.y = pack_bf16(__uint_as_float(o[8 * v + 2]) * inv, __uint_as_float(o[8 * v + 3]) * inv);
            u.z = pack_bf16(__uint_as_float(o[8 * v + 4]) * inv, __uint_as_float(o[8 * v + 5]) * inv);
            u.w = pack_bf16(__uint_as_float(o[8 * v + 6]) * inv, __uint_as_float(o[8 * v + 7]) * inv);
            *reinterpret_cast<uint4 *>(dst + v * 8) = u;
          }
          if (part == 0 && p.lse) p.lse[(int64_t)(J.q0 + j) * p.Hq + J.g * p.G + hg] = (pend.m_ref + log2f(l_row)) * kLn2;
        } else {
          const int64_t slot = (int64_t)J.part_slot * p.rows_cap + row;
          float *dst = p.part_o + slot * D + part * CB;
#pragma unroll
          for (int v = 0; v < CB / 4; ++v)
            *reinterpret_cast<float4 *>(dst + v * 4) = make_float4(__uint_as_float(o[4 * v]) * f, __uint_as_float(o[4 * v + 1]) * f,
                                                                  __uint_as_float(o[4 * v + 2]) * f, __uint_as_float(o[4 * v + 3]) * f);
          if (part == 0) p.part_ml[slot] = make_float2(pend.m_ref, l_row);
        }
      }
      // the slot of the entry after next: its last user's epilogue lies at least one barrier back, its
      // next user's first look at V at least one ahead
      const int clear = (pend.qc + 2) % kE8NanSlots;
      if (sm_tid < 128) sNan[clear * 128 + sm_tid] = 0;
      if (sm_tid == 128) bars->nan_any[clear] = 0;
      pend.valid = false;
      return true;
    };
    WorkEntry e, e_next;
    if (item_index(0) >= 0) e = p.work[item_index(0)];
    for (int it = 0; item_index(it) >= 0 && ok; ++it, ++qc) {
      if (bars->abort) break;
      const int idx_next = item_index(it + 1);
      if (idx_next >= 0) e_next = p.work[idx_next];
      const bool valid_row = row < e.m * p.G;
      float m_ref = -INFINITY, x_ref = -INFINITY, l_sum = 0.f, row_f = 0.f;   // the references are the same in all parts of a row
      const int limit = e.L - e.m + row / p.G;  // last visible token of this row
      for (int tile = e.tile_begin; tile < e.tile_end && ok; ++tile, ++tc_) {
        const uint32_t b = tc_ & 1;
        const int sc_slot = tc_ % kE8ScaleSlots;
        const int t0 = tile * kTileTokens + part * TPT;  // first token of this thread
        const bool mask_tile = tile * kTileTokens + kTileTokens - 1 > e.L - e.m;
        ok = warp_wait(&bars->sc_full[sc_slot], (tc_ / kE8ScaleSlots) & 1) && warp_wait(&bars->s_full[b], (tc_ >> 1) & 1);
        if (!ok) break;
        fence_after();
        if (tile == e.tile_begin) row_f = sRow[(it % kE8RowSlots) * MROWS + row];
        uint32_t r[TPT];
        tmem_load<TPT>(tmem + Cfg::kColS + b * Cfg::kSCols + half * TPT + lane_addr, r);
        wait_ld();
        const float4 *ks4 = reinterpret_cast<const float4 *>(sKs + sc_slot * 128 + part * TPT);
        const float4 *vs4 = reinterpret_cast<const float4 *>(sVs + sc_slot * 128 + part * TPT);
        const float2 v_range = sVr[sc_slot];
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < TPT / 4; ++i) {
          const float4 s = ks4[i];
          r[4 * i] = __float_as_uint(__uint_as_float(r[4 * i]) * s.x);
          r[4 * i + 1] = __float_as_uint(__uint_as_float(r[4 * i + 1]) * s.y);
          r[4 * i + 2] = __float_as_uint(__uint_as_float(r[4 * i + 2]) * s.z);
          r[4 * i + 3] = __float_as_uint(__uint_as_float(r[4 * i + 3]) * s.w);
        }
        if (mask_tile) {
#pragma unroll
          for (int i = 0; i < TPT; ++i) r[i] = (t0 + i <= limit) ? r[i] : 0xff800000u;  // -inf
        }
#pragma unroll
        for (int i = 0; i < TPT; ++i) mx = fmaxf(mx, __uint_as_float(r[i]));
        // agree on the row's maxima over the whole tile
        const bool narrow = v_range.y != 0.f;
        sMx[(b * kParts + part) * MROWS + row] = mx * row_f;
        if (!narrow) {
          float mx2 = -INFINITY;
          const float *vs1 = reinterpret_cast<const float *>(vs4);
#pragma unroll
          for (int i = 0; i < TPT; ++i) mx2 = fmaxf(mx2, fmaf(__uint_as_float(r[i]), row_f, fmaxf(__log2f(vs1[i]), kE8MinLog2)));
          sMx2[(b * kParts + part) * MROWS + row] = mx2;
        }
        ok = softmax_sync();
        if (!ok) break;
        float m_tile = -INFINITY, x_tile = -INFINITY;
#pragma unroll
        for (int i = 0; i < kParts; ++i) m_tile = fmaxf(m_tile, sMx[(b * kParts + i) * MROWS + row]);
        if (narrow) {
          x_tile = m_tile + v_range.x;
        } else {
#pragma unroll
          for (int i = 0; i < kParts; ++i) x_tile = fmaxf(x_tile, sMx2[(b * kParts + i) * MROWS + row]);
        }
        if (m_tile > m_ref) {
          l_sum *= m_ref == -INFINITY ? 0.f : fast_exp2(m_ref - m_tile);
          m_ref = m_tile;
        }
        // x's reference moves when it is passed by a factor of four; a row without one adopts the
        // tile's (its O is zero)
        float alpha = 1.f;
        bool need_scale = false;
        if (x_ref == -INFINITY) {
          x_ref = x_tile;
        } else if (x_tile > x_ref + kE8Rescale) {
          alpha = fast_exp2(x_ref - x_tile);
          x_ref = x_tile;
          need_scale = valid_row;
        }
        if (__any_sync(0xffffffffu, need_scale)) {
          // this warp's columns of O hold earlier tiles: wait for the last value MMA, scale
          ok = warp_wait(&bars->pv_done[(tc_ - 1) & 1], ((tc_ - 1) >> 1) & 1);
          if (!ok) break;
          fence_after();
          uint32_t o[CB];
          const uint32_t to = tmem + Cfg::kColO + (qc & 1) * Cfg::kOCols + half * CB + lane_addr;
          tmem_load<CB>(to, o);
          wait_ld();
#pragma unroll
          for (int i = 0; i < CB; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
          tmem_store<CB>(to, o);
          wait_st();
        }
        const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
        const float gain = x_ref == -INFINITY ? 0.f : fast_exp2(kE8Shift + m_use - x_ref);
        // P's buffer is free once the value MMAs that read it last are done
        if (tc_ >= (uint32_t)Cfg::kPBufs) {
          const uint32_t u = tc_ - Cfg::kPBufs;
          ok = warp_wait(&bars->pv_done[u & 1], (u >> 1) & 1);
          if (!ok) break;
        }
        unsigned char *pr = sP + (Cfg::kPBufs == 2 ? b : 0) * 3 * Cfg::kPiece + (row >> 3) * 1024 + (row & 7) * 128;
        float sum = 0.f;
#pragma unroll
        for (int c = 0; c < TPT / 16; ++c) {
          uint32_t w[3][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 s = vs4[4 * c + i];
            const int at = 16 * c + 4 * i;
            const float p0 = fast_exp2(fmaf(__uint_as_float(r[at]), row_f, -m_use));
            const float p1 = fast_exp2(fmaf(__uint_as_float(r[at + 1]), row_f, -m_use));
            const float p2 = fast_exp2(fmaf(__uint_as_float(r[at + 2]), row_f, -m_use));
            const float p3 = fast_exp2(fmaf(__uint_as_float(r[at + 3]), row_f, -m_use));
            sum += (p0 + p1) + (p2 + p3);
            cut3(pack_f16(p0 * s.x * gain, p1 * s.y * gain), pack_f16(p2 * s.z * gain, p3 * s.w * gain), w[0][i], w[1][i], w[2][i]);
          }
          const int chunk = part * (TPT / 16) + c;   // 16-byte chunk of the row: 16 tokens
#pragma unroll
          for (int i = 0; i < 3; ++i)
            *reinterpret_cast<uint4 *>(pr + i * Cfg::kPiece + ((chunk ^ (row & 7)) << 4)) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
        }
        l_sum += sum;
        if (mask_tile) {
          // V at the end of the request, as its value MMA must see it: slots past the end are zero (they
          // hold an earlier tile's or nobody's bytes, and 0 * NaN is NaN), and a NaN at a position that some
          // rows do not see is taken out and left to the epilogue of those that do
          const int ntok = min(kTileTokens, e.L - tile * kTileTokens);
          const int hidden = max(0, e.L - e.m + 1 - tile * kTileTokens);   // first token of the tile not seen by every row
          const int slot = tc_ % Cfg::kStages;
          ok = warp_wait(&bars->v_full[slot], (tc_ / Cfg::kStages) & 1);
          if (!ok) break;
          unsigned char *vt = sV + slot * Cfg::kTileBytes;
#pragma unroll 1
          for (int i = sm_tid; i < (kTileTokens - ntok) * (D / 16); i += 256)
            *reinterpret_cast<uint4 *>(vt + ntok * D + i * 16) = make_uint4(0, 0, 0, 0);
#pragma unroll 1
          for (int i = sm_tid; i < (ntok - hidden) * (D / 16); i += 256) {
            const int tok = hidden + i / (D / 16), ch = i % (D / 16);
            uint4 *at = reinterpret_cast<uint4 *>(vt + tok * D + ch * 16);
            uint4 v = *at;
            uint32_t *w = &v.x;
            uint32_t any = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) any |= __vcmpeq4(w[k] & 0x7f7f7f7fu, 0x7f7f7f7fu);
            if (any) {
              // logical columns of this chunk under the swizzle
              const int col = (D == 128 ? ch ^ (tok & 7) : ch ^ ((tok >> 1) & 3)) * 16;
              const uint32_t bit = 1u << (tile * kTileTokens + tok - (e.L - e.m + 1));   // rows j > this position's index see it
#pragma unroll 1
              for (int k = 0; k < 16; ++k)
                if (((w[k >> 2] >> (8 * (k & 3))) & 0x7f) == 0x7f) {
                  w[k >> 2] &= ~(0xffu << (8 * (k & 3)));
                  atomicOr(&sNan[(qc % kE8NanSlots) * 128 + col + k], bit);
                }
              *at = v;
              bars->nan_any[qc % kE8NanSlots] = 1;
            }
          }
        }
        fence_async_smem();
        fence_before();
        __syncwarp();
        if (lane == 0) { mbar_arrive(&bars->p_full[b]); mbar_arrive(&bars->sc_empty[sc_slot]); }
        if (pend.valid) ok = run_epilogue();  // previous entry (its sL became visible at this tile's barrier)
      }
      if (!ok) break;
      // the entry's epilogue is deferred: it runs after the first tile of the next one
      sL[((qc & 1) * kParts + part) * MROWS + row] = l_sum;
      pend.valid = true; pend.e = e; pend.m_ref = m_ref; pend.x_ref = x_ref; pend.last_tc = tc_ - 1; pend.qc = qc;
      e = e_next;
    }
    if (ok && pend.valid && !bars->abort) {
      ok = softmax_sync();  // make the last entry's row sums visible
      if (ok) ok = run_epilogue();
    }
  }

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
