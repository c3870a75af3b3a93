// Attention of many query rows on the 5th-generation tensor cores (tcgen05 + TMEM), fed by TMA page gathers.
//
// An item is up to 256 packed rows of one kv head: two groups of 128 rows, the M of a score and a value MMA, that share every K and
// V tile.  One persistent CTA per SM, warp-specialised:
//   warps 0-3, 4-7  softmax of group 0 and 1: a thread holds one row's 128 scores of a tile in registers (one read
//                   of tensor memory, no exchange between threads), keeps the row's maximum and sum, and writes
//                   its weights over the scores as bf16, the A operand of the value MMA;
//   warp 8          producer: takes entries of the plan, copies query rows, and K and V tiles, page by page, into a ring;
//   warps 9, 10     issuers of the MMAs of group 0 and 1 (one warp for both was the bound: 12 waits, elections and commits
//                   a tile, 200 cycles each).  While one group is at its softmax the other's MMAs run;
//   warp 11         looks after the V tiles at the edge of what rows see (below); over 8-bit pools it fetches scales,
//                   and warps 12-15 turn the codes into bf16 tiles.
// Tensor memory is full: two score buffers of 128 columns and two outputs of D.
//
// Two prompts of 8192 tokens, 32/8 heads of 128: 907 us (1.21 PFLOP/s), 1064 on boards whose clock falls under the load; 24 of up to 2000 tokens 283
// to 325; six of up to 4000 over 8-bit pools 480 to 500.  No unit alone bounds it (MMA pipe 53 % busy, exponentials 50 %), but the chain between them.
//
// The running maximum of a row is a reference that moves only when weights under it grow past 2^8 or so (the output
// is then rescaled by the row's own thread).  Weights are rounded to bf16 (half a step of 2^-8 each, the type V has to be multiplied in); their sum is
// taken in fp32 before that.
//
// What rows do not see must not reach them.  Scores are masked before the maximum.  A weight of zero does not
// mask an infinity or a NaN in V, so in the tiles at the edge (some row of the item does not see all of them) V is
// looked through: rows past the last one seen become zero, and elements that are not finite become zero and are noted; the rows that
// do see one get it (an infinity of its sign, NaN otherwise) at the end.
#pragma once
#include <type_traits>

#include "attn_e4m3.cuh"
#include "attn_tc.cuh"
#include "attn_tc4.cuh"
#include "prompt_plan.cuh"

namespace spx {

// Threads, and registers of a softmax warp, of warps 8-11, of the converting warps 12-15: together what 65536 registers give each thread at launch.
template <bool kCodes>
struct PtSplit {
  static constexpr int kThreads = kCodes ? 512 : 384;
  static constexpr int kSoftmax = kCodes ? 176 : 192, kOther = kCodes ? 96 : 120, kConvert = 64;
  static constexpr int kLaunch = 65536 / kThreads / 8 * 8;
  static_assert(2 * kSoftmax + kOther + (kCodes ? kConvert : 0) == kLaunch * (kThreads / 128), "what is given is what is there");
};
constexpr int kPtScaleSlots = 4;   // tiles whose scales are staged

template <int D, bool kCodes>
struct PtCfg {
  static constexpr int kHalves = D / 64;
  static constexpr int kHalfBytes = 128 * 128;             // 128 rows of 64 elements: a half of a tile, or of a group's query rows
  static constexpr int kTileBytes = kHalves * kHalfBytes;
  static constexpr int kSlots = kCodes ? (D == 128 ? 3 : 6) : (D == 128 ? 5 : 8);
  static constexpr int kRawBytes = kTileTokens * D, kRawSlots = D == 128 ? 3 : 6;   // 8-bit pools: tiles as they lie there
  static constexpr int kOffKv = 2 * kTileBytes;            // behind the query rows of the two groups
  static constexpr int kOffRaw = kOffKv + kSlots * kTileBytes;
  static constexpr int kOffScale = kOffRaw + (kCodes ? kRawSlots * kRawBytes : 0);      // [slot][K, V][128]
  static constexpr int kOffBar = kOffScale + (kCodes ? kPtScaleSlots * 1024 : 0);
  static constexpr int kSmemBytes = kOffBar + 1024 + 1024;
  static_assert(kSmemBytes <= 232448, "shared memory");
  static constexpr int kColS = 0, kColO = 256;             // group x: S at 128 x, O at 256 + D x
};

struct PtBars {
  uint64_t kv_full[8], kv_empty[8], q_full[2], q_empty[2], s_full[2][2], p_full[2][2], h_done[2], o_full[2], o_free[2], item_full[2], item_empty[2], v_ask, v_clean, item_clean[2];
  uint64_t turn[2][4];
  uint64_t raw_full[6], raw_empty[6], sc_full[kPtScaleSlots], sc_empty[kPtScaleSlots];
  PromptEntry item[2];
  int32_t notes[2];
  int32_t general[kPtScaleSlots];   // some scale of the tile is no power of two
  uint32_t tmem_base;
  volatile int32_t abort;
  int32_t *dev_status;
};
static_assert(sizeof(PtBars) <= 1024, "barrier area");

namespace pt {

using namespace tc;
using e8::add2;
using e8::arrive;
using e8::commit;
using e8::elect_lane;
using e8::expect_tx;
using e8::fma2;
using e8::pair;
using e8::try_wait;
using e8::try_wait_long;
using e8::unpair;

// Bounded wait of a converged warp; the outcome is told by the abort flag alone, which every role's loop looks at once a tile.
// (In line: a call's convention and a split of the registers among the warps do not go together.)
__device__ __forceinline__ void wait(uint64_t *b, uint32_t parity, PtBars *bars) {
  const uint32_t bar = smem_u32(b);
  if (__all_sync(0xffffffffu, try_wait(bar, parity & 1))) return;
  const long long t0 = clock64();
#pragma unroll 1
  while (!__all_sync(0xffffffffu, try_wait_long(bar, parity & 1))) {
    const bool late = clock64() - t0 > kWaitLimitCycles;
    if (late) {
      bars->abort = 1;
      atomicOr(bars->dev_status, SPX_DEV_TIMEOUT);
    }
    if (__any_sync(0xffffffffu, late || bars->abort)) return;
  }
}
// (volatile: a batch of them is issued in a row, while the one before is made use of)
__device__ __forceinline__ float exp2_in_turn(float x) {
  float y;
  asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 32 bytes: a whole sector, where the address allows it
__device__ __forceinline__ void store_sector(void *at, const uint32_t (&r)[8], bool aligned) {
  if (!aligned) {
    *reinterpret_cast<uint4 *>(at) = make_uint4(r[0], r[1], r[2], r[3]);
    *(reinterpret_cast<uint4 *>(at) + 1) = make_uint4(r[4], r[5], r[6], r[7]);
    return;
  }
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// one arrival for the warp, behind what its lanes did
__device__ __forceinline__ void warp_arrive(uint64_t *b, int lane) {
  __syncwarp();
  if (lane == 0) arrive(smem_u32(b));
}

// Looks through a V row that some rows do not see: what is not finite becomes zero and is noted.
template <int D>
__device__ __forceinline__ void look_through(unsigned char *row_at, int tok, int token, PromptNote *notes, int32_t *count) {
  constexpr int kHalfBytes = 128 * 128;
  const uint4 *row = reinterpret_cast<const uint4 *>(row_at);
  // 0 * x is zero for a finite x, NaN otherwise
  const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
  __nv_bfloat162 acc = zero;
#pragma unroll
  for (int i = 0; i < D / 8; ++i) {
    const uint4 w = row[(i >> 3) * (kHalfBytes / 16) + (i & 7)];
    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&w.x), zero, acc);
    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&w.y), zero, acc);
    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&w.z), zero, acc);
    acc = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&w.w), zero, acc);
  }
  if ((*reinterpret_cast<const uint32_t *>(&acc) & 0x7fff7fffu) == 0) return;
  const int note = atomicAdd(count, 1);
  if (note >= kPtNotes) return;                   // (cannot be: a token for each position but the first)
  notes[note].token = token;
#pragma unroll 1
  for (int b = 0; b < 4; ++b) {                   // 32 columns
    uint32_t plus = 0, minus = 0;
    if (b < D / 32) {
#pragma unroll 1
      for (int c = 0; c < 32; ++c) {
        const int col = b * 32 + c, chunk = (col & 63) >> 3;
        uint16_t *at = reinterpret_cast<uint16_t *>(row_at + (col >> 6) * kHalfBytes + ((chunk ^ (tok & 7)) << 4)) + (col & 7);
        const uint16_t x = *at;
        if ((x & 0x7f80u) != 0x7f80u) continue;
        const bool nan = (x & 0x7fu) != 0;
        if (nan || !(x & 0x8000u)) plus |= 1u << c;
        if (nan || (x & 0x8000u)) minus |= 1u << c;
        *at = 0;
      }
    }
    notes[note].plus[b] = plus; notes[note].minus[b] = minus;
  }
}

}  // namespace pt

template <int D, bool kCodes>
__global__ void __launch_bounds__(PtSplit<kCodes>::kThreads, 1)
prompt_tc_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CUtensorMap qmap,
                 PromptParams p) {
  SPX_TL_SCOPE(kTlAttention);
  using Cfg = PtCfg<D, kCodes>;
  using Split = PtSplit<kCodes>;
  using namespace pt;
  extern __shared__ __align__(1024) unsigned char smem_dyn[];
  unsigned char *smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_dyn) + 1023) & ~uintptr_t(1023));
  unsigned char *sQ = smem, *sKv = smem + Cfg::kOffKv;
  PtBars *bars = reinterpret_cast<PtBars *>(smem + Cfg::kOffBar);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
#pragma unroll 1
    for (int s = 0; s < 8; ++s) { mbar_init(&bars->kv_full[s], kCodes ? 4 : 1); mbar_init(&bars->kv_empty[s], 2); }
    if (kCodes) {
#pragma unroll 1
      for (int s = 0; s < 6; ++s) { mbar_init(&bars->raw_full[s], 1); mbar_init(&bars->raw_empty[s], 4); }
#pragma unroll 1
      for (int s = 0; s < kPtScaleSlots; ++s) { mbar_init(&bars->sc_full[s], 1); mbar_init(&bars->sc_empty[s], 12); }   // eight softmax, four converting warps
    }
#pragma unroll 1
    for (int b = 0; b < 2; ++b) {
      mbar_init(&bars->q_full[b], 1); mbar_init(&bars->q_empty[b], 1); mbar_init(&bars->s_full[b][0], 1); mbar_init(&bars->s_full[b][1], 1);
      mbar_init(&bars->p_full[b][0], 4); mbar_init(&bars->p_full[b][1], 4); mbar_init(&bars->h_done[b], 1);
      mbar_init(&bars->o_full[b], 1); mbar_init(&bars->o_free[b], 4);
      mbar_init(&bars->item_full[b], 1); mbar_init(&bars->item_empty[b], kCodes ? 15 : 11);   // eight softmax warps, two issuers, the edge warp (or four converting ones and the scales')
      mbar_init(&bars->item_clean[b], kCodes ? 4 : 1);
      bars->notes[b] = 0;
    }
#pragma unroll 1
    for (int i = 0; i < 8; ++i) mbar_init(&bars->turn[i >> 2][i & 3], 1);
    mbar_init(&bars->v_ask, 2); mbar_init(&bars->v_clean, 1);
    bars->abort = 0;
    bars->dev_status = p.dev_status;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = bars->tmem_base;
  // everything above touched only this CTA's own resources; the plan, and what the caller's kernels before it wrote, is read from here on
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  const bool causal = p.groups == 0;
  const int half_rows = p.unit_rows >> 1;    // packed rows of a group: whole positions, at most 128
  // first tile of an entry in which some of its rows do not see every token
  auto edge_tile = [&](const PromptEntry &e) -> int {
    return causal ? max(e.tile_begin, min(e.tile_end, (e.vis0 + e.row0 / p.G + 1) / kTileTokens)) : e.tile_end;
  };
  // The entry of item n for the roles that follow the producer: false when there is none, or another role gave up.
  auto next_item = [&](uint32_t n, PromptEntry &e) -> bool {
    wait(&bars->item_full[n & 1], n >> 1, bars);
    e = bars->item[n & 1];
    return e.unit >= 0 && !bars->abort;
  };

  if (warp >= 8 && warp < 12) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Split::kOther));
  if (warp == 8) {
    // ------------------------------------------------------------------ producer
    const int n_units = p.hdr->n_units;
    const int pages_per_tile = kTileTokens >> p.log2P, tiles_per_group = 32 / pages_per_tile;
    uint32_t n_item = 0, n_kv = 0, n_q[2] = {0, 0};
    auto take = [&]() -> int {
      int u = 0;
      if (lane == 0) u = atomicAdd(&p.hdr->counter, 1);
      return u;
    };
    int unit_next = take();
    for (;;) {
      const int unit = __shfl_sync(0xffffffffu, unit_next, 0);
      if (unit >= n_units || bars->abort) break;
      unit_next = take();    // in flight until this one is done
      {
        PromptEntry e = p.entries[unit / p.Hkv];
        e.g = unit % p.Hkv;
        if (e.slot >= 0) e.slot += e.g;
        wait(&bars->item_empty[n_item & 1], (n_item >> 1) ^ 1, bars);
        if (lane == 0) { bars->item[n_item & 1] = e; bars->notes[n_item & 1] = 0; }
        warp_arrive(&bars->item_full[n_item & 1], lane);
        const int32_t *table = p.block_table + (int64_t)e.table_row * p.max_pages_per_req;
        const int t_end = min(e.t_end, e.tile_end * kTileTokens);
        // page ids of a group of tiles, a lane's (tile, page) each, one group ahead of the copies
        auto pages_of = [&](int tile0) -> int {
          const int tile = tile0 + lane / pages_per_tile, t = tile * kTileTokens + (lane % pages_per_tile) * p.P;
          return tile < e.tile_end && t < t_end ? table[t >> p.log2P] : 0;
        };
        int page_next = pages_of(e.tile_begin);
        for (int x = 0; x < 2; ++x) {
          if (x * half_rows >= e.rows) break;
          wait(&bars->q_empty[x], n_q[x] ^ 1, bars);
          if (elect_lane()) {
            const uint32_t bar = smem_u32(&bars->q_full[x]);
            expect_tx(bar, (uint32_t)p.box_rows * p.G * D * 2);
#pragma unroll
            for (int h = 0; h < Cfg::kHalves; ++h)
              tma_load_3d(smem_u32(sQ + x * Cfg::kTileBytes + h * Cfg::kHalfBytes), &qmap, &bars->q_full[x], h * 64, e.g * p.G,
                          e.q0 + (e.row0 + x * half_rows) / p.G);
          }
          __syncwarp();
          ++n_q[x];
        }
        int page = 0, tile0 = e.tile_begin;
#pragma unroll 1
        for (int tile = e.tile_begin; tile < e.tile_end; ++tile) {
          if (tile == tile0) {
            page = page_next;
            tile0 += tiles_per_group;
            page_next = pages_of(tile0);
            if (page < 0 || page >= p.num_pages) {
              page = 0;    // keep the copy in bounds; the request is flagged and its rows are voided
              atomicOr(p.dev_status, SPX_DEV_BAD_PAGE);
              p.unit_bad[e.unit] = 1;
              p.hdr->any_bad = 1;
            }
          }
          const int my_page = __shfl_sync(0xffffffffu, page, ((tile - tile0 + tiles_per_group) * pages_per_tile + lane) & 31);
          const int npages = (min(kTileTokens, t_end - tile * kTileTokens) + p.P - 1) >> p.log2P;
#pragma unroll
          for (int v = 0; v < 2; ++v, ++n_kv) {
            if constexpr (kCodes) {
              const uint32_t slot = n_kv % Cfg::kRawSlots;
              wait(&bars->raw_empty[slot], n_kv / Cfg::kRawSlots ^ 1, bars);
              if (lane == 0) expect_tx(smem_u32(&bars->raw_full[slot]), (uint32_t)npages * p.P * D);
              __syncwarp();
              if (lane < npages)
                e8::tma_page(smem_u32(smem + Cfg::kOffRaw + slot * Cfg::kRawBytes + lane * p.P * D), v ? &vmap : &kmap, smem_u32(&bars->raw_full[slot]),
                             p.head_inner ? e.g : 0, p.head_inner ? 0 : e.g, my_page);
              __syncwarp();
              continue;
            }
            const uint32_t slot = n_kv % Cfg::kSlots;
            wait(&bars->kv_empty[slot], n_kv / Cfg::kSlots ^ 1, bars);
            if (lane == 0) expect_tx(smem_u32(&bars->kv_full[slot]), (uint32_t)npages * p.P * D * 2);
            __syncwarp();
            if (lane < npages) {
#pragma unroll
              for (int h = 0; h < Cfg::kHalves; ++h)
                tma_load_4d(smem_u32(sKv + slot * Cfg::kTileBytes + h * Cfg::kHalfBytes + lane * p.P * 128), v ? &vmap : &kmap, &bars->kv_full[slot], h * 64,
                            p.head_inner ? e.g : 0, p.head_inner ? 0 : e.g, my_page);
            }
            __syncwarp();
          }
          if (bars->abort) break;
        }
        ++n_item;
      }
    }
    // no more: an entry of no unit
    wait(&bars->item_empty[n_item & 1], (n_item >> 1) ^ 1, bars);
    if (lane == 0) bars->item[n_item & 1].unit = -1;
    warp_arrive(&bars->item_full[n_item & 1], lane);
  } else if (warp <= 10) {
    // ------------------------------------------------------------------ issuer of a group
    constexpr uint32_t kIdescQK = idesc(64, false), kIdescPV = idesc(D, true);
    const int x = warp - 9;
    const uint32_t ts = tmem + Cfg::kColS + x * 128, to = tmem + Cfg::kColO + x * D;
    const uint64_t qd = smem_desc(smem_u32(sQ + x * Cfg::kTileBytes), 16, 1024);
    uint32_t n_kv = 0, n_p = 0, n_own = 0, n_clean = 0;   // tiles of the ring, the group's tiles and items, edge tiles
    PromptEntry e;
    for (uint32_t n = 0; next_item(n, e); ++n) {
      const bool active = x * half_rows < e.rows;           // (an idle group's issuer hands the tiles back)
      const int n_tiles = e.tile_end - e.tile_begin, edge = edge_tile(e) - e.tile_begin;
      // scores of half a tile, 64 tokens, over what the half's weights of the tile before leave
      auto scores = [&](uint32_t at, int h, bool last) {
        const uint32_t slot = at % Cfg::kSlots;
        if (h == 0) wait(&bars->kv_full[slot], at / Cfg::kSlots, bars);
        if (!active) {
          if (h == 1) warp_arrive(&bars->kv_empty[slot], lane);
          return;
        }
        fence_after();
        if (elect_lane()) {
          const uint64_t kd = smem_desc(smem_u32(sKv + slot * Cfg::kTileBytes), 16, 1024) + h * 512;
#pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint64_t off = ((k / 4) * Cfg::kHalfBytes + (k % 4) * 32) >> 4;   // (descriptors count 16 bytes)
            mma_ss(ts + h * 64, qd + off, kd + off, kIdescQK, k > 0);
          }
          commit(smem_u32(&bars->s_full[x][h]));
          if (h == 1) commit(smem_u32(&bars->kv_empty[slot]));
          if (h == 1 && last) commit(smem_u32(&bars->q_empty[x]));
        }
        __syncwarp();
      };
      if (active) wait(&bars->q_full[x], n_own, bars);
      scores(n_kv, 0, n_tiles == 1);
      scores(n_kv, 1, n_tiles == 1);
      if (!kCodes && edge <= 0) warp_arrive(&bars->v_ask, lane);
#pragma unroll 1
      for (int i = 0; i < n_tiles && !bars->abort; ++i, n_kv += 2) {
        const uint32_t at = n_kv + 1, slot = at % Cfg::kSlots;
        const bool more = i + 1 < n_tiles;
        wait(&bars->kv_full[slot], at / Cfg::kSlots, bars);
        if (!kCodes && i >= edge) wait(&bars->v_clean, n_clean++, bars);
        if (!kCodes && more && i + 1 >= edge) warp_arrive(&bars->v_ask, lane);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          if (active) {
            wait(&bars->p_full[x][h], n_p, bars);
            if (h == 0 && i == 0 && n_own > 0) wait(&bars->o_free[x], n_own - 1, bars);
            fence_after();
            if (elect_lane()) {
              const uint64_t vd = smem_desc(smem_u32(sKv + slot * Cfg::kTileBytes), Cfg::kHalfBytes, 1024);
#pragma unroll
              for (int k = 0; k < 4; ++k) mma_ts(to, ts + h * 64 + k * 8, vd + (4 * h + k) * 128, kIdescPV, i > 0 || h > 0 || k > 0);
              if (h == 0 && !more) commit(smem_u32(&bars->h_done[x]));
              if (h == 1) commit(smem_u32(&bars->kv_empty[slot]));
              if (h == 1 && !more) commit(smem_u32(&bars->o_full[x]));
            }
            __syncwarp();
          } else if (h == 1) {
            warp_arrive(&bars->kv_empty[slot], lane);
          }
          if (more) scores(at + 1, h, i + 2 == n_tiles);
        }
        if (active) ++n_p;
      }
      if (active) ++n_own;
      warp_arrive(&bars->item_empty[n & 1], lane);
    }
  } else if (!kCodes) {
    // ------------------------------------------------------------------ V tiles at the edge
    // The issuers ask for a tile while they work on the one before (so that the slot's barrier is in the phase waited for, and
    // not one that the ring is yet to come to) and do not go past it without an answer.
    uint32_t n_kv = 0, n_ask = 0;
    PromptNote *notes = p.notes + (int64_t)blockIdx.x * 2 * kPtNotes;
    PromptEntry e;
    for (uint32_t n = 0; next_item(n, e); ++n) {
      const int edge = edge_tile(e);
      const int whole = e.vis0 + e.row0 / p.G;             // every row sees the tokens up to here
#pragma unroll 1
      for (int tile = edge; tile < e.tile_end; ++tile) {
        const uint32_t at = n_kv + 2 * (uint32_t)(tile - e.tile_begin) + 1, slot = at % Cfg::kSlots;
        wait(&bars->v_ask, n_ask++, bars);
        wait(&bars->kv_full[slot], at / Cfg::kSlots, bars);
        unsigned char *vt = sKv + slot * Cfg::kTileBytes;
        const int t0 = tile * kTileTokens, n_tok = min(kTileTokens, e.t_end - t0);
#pragma unroll 1
        for (int tok = lane; tok < kTileTokens; tok += 32) {
          if (t0 + tok <= whole) continue;
          unsigned char *row = vt + (tok >> 3) * 1024 + (tok & 7) * 128;
          if (tok < n_tok) {
            look_through<D>(row, tok, t0 + tok, notes + (n & 1) * kPtNotes, &bars->notes[n & 1]);
          } else {
#pragma unroll
            for (int i = 0; i < D / 8; ++i) *reinterpret_cast<uint4 *>(row + (i >> 3) * Cfg::kHalfBytes + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
          }
        }
        fence_async_smem();
        warp_arrive(&bars->v_clean, lane);
        if (bars->abort) break;
      }
      n_kv += 2 * (uint32_t)(e.tile_end - e.tile_begin);
      warp_arrive(&bars->item_clean[n & 1], lane);
      warp_arrive(&bars->item_empty[n & 1], lane);
    }
  } else {
    // ------------------------------------------------------------------ scales of 8-bit pools: four tokens of a tile a lane
    float *sScale = reinterpret_cast<float *>(smem + Cfg::kOffScale);
    uint32_t n_tile = 0;
    PromptEntry e;
    for (uint32_t n = 0; next_item(n, e); ++n) {
      const int32_t *table = p.block_table + (int64_t)e.table_row * p.max_pages_per_req;
      const int t_end = min(e.t_end, e.tile_end * kTileTokens);
      int page[4];
      auto pages_of = [&](int tile) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = tile * kTileTokens + lane + 32 * i;
          page[i] = t < t_end ? table[t >> p.log2P] : -1;
        }
      };
      pages_of(e.tile_begin);
#pragma unroll 1
      for (int tile = e.tile_begin; tile < e.tile_end; ++tile, ++n_tile) {
        float ks[4], vs[4];
        bool general = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int t = tile * kTileTokens + lane + 32 * i;
          ks[i] = vs[i] = 1.f;
          if (page[i] >= 0 && page[i] < p.num_pages) {
            const int64_t at = (((int64_t)page[i] * p.Hkv + e.g) << (p.log2P - p.log2SB)) + ((t & (p.P - 1)) >> p.log2SB);
            ks[i] = p.k_scales[at];
            vs[i] = p.v_scales[at];
          }
        }
        pages_of(tile + 1);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t a = __float_as_uint(ks[i]), b = __float_as_uint(vs[i]);
          general |= ((a & 0x7fffffu) && (a & 0x7f800000u)) || ((b & 0x7fffffu) && (b & 0x7f800000u));
        }
        const uint32_t slot = n_tile % kPtScaleSlots;
        wait(&bars->sc_empty[slot], n_tile / kPtScaleSlots ^ 1, bars);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sScale[slot * 256 + lane + 32 * i] = ks[i];
          sScale[slot * 256 + 128 + lane + 32 * i] = vs[i];
        }
        general = __any_sync(0xffffffffu, general);
        if (lane == 0) bars->general[slot] = general;
        warp_arrive(&bars->sc_full[slot], lane);
        if (bars->abort) break;
      }
      warp_arrive(&bars->item_empty[n & 1], lane);
    }
  }
  } else if (kCodes && warp >= 12) {
    // ------------------------------------------------------------------ 8-bit tiles to bf16 ones: a thread a token
    // A code times the power of two in its scale is exact in bf16; what is left of a scale, 1 <= f < 2, multiplies the score,
    // or the weight, of its token.
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Split::kConvert));
    const int tok = tid - 384;
    const float *sScale = reinterpret_cast<const float *>(smem + Cfg::kOffScale);
    PromptNote *notes = p.notes + (int64_t)blockIdx.x * 2 * kPtNotes;
    uint32_t n_tile = 0;
    PromptEntry e;
    for (uint32_t n = 0; next_item(n, e); ++n) {
      const int edge = edge_tile(e), whole = e.vis0 + e.row0 / p.G;
#pragma unroll 1
      for (int tile = e.tile_begin; tile < e.tile_end; ++tile, ++n_tile) {
        const uint32_t sc = n_tile % kPtScaleSlots;
        wait(&bars->sc_full[sc], n_tile / kPtScaleSlots, bars);
        const float ks = sScale[sc * 256 + tok], vs = sScale[sc * 256 + 128 + tok];
        warp_arrive(&bars->sc_empty[sc], lane);
#pragma unroll 1
        for (int v = 0; v < 2; ++v) {
          const uint32_t at = 2 * n_tile + v, rs = at % Cfg::kRawSlots, slot = at % Cfg::kSlots;
          const uint32_t bits = __float_as_uint(v ? vs : ks);
          const uint32_t exponent = bits & 0x7f800000u;    // (a scale below the smallest normal, or not finite, is taken as it is)
          const float mul = __uint_as_float(exponent != 0 && exponent != 0x7f800000u ? bits & 0xff800000u : bits);
          const uint64_t mul2_ = pair(mul, mul);
          wait(&bars->raw_full[rs], at / Cfg::kRawSlots, bars);
          wait(&bars->kv_empty[slot], at / Cfg::kSlots ^ 1, bars);
          const unsigned char *src = smem + Cfg::kOffRaw + rs * Cfg::kRawBytes + tok * D;
          unsigned char *row = sKv + slot * Cfg::kTileBytes + (tok >> 3) * 1024 + (tok & 7) * 128;
#pragma unroll
          for (int c = 0; c < D / 16; ++c) {
            const uint4 w = *reinterpret_cast<const uint4 *>(src + ((D == 128 ? c ^ (tok & 7) : c ^ ((tok >> 1) & 3)) << 4));
            const uint32_t in[4] = {w.x, w.y, w.z, w.w};
            uint32_t o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(in[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
              const float2 f = __half22float2(__half2(h));
              float a, b;
              unpair(e8::mul2(pair(f.x, f.y), mul2_), a, b);
              o[i] = pack_bf16(a, b);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int oc = 2 * c + i;
              *reinterpret_cast<uint4 *>(row + (oc >> 3) * Cfg::kHalfBytes + (((oc & 7) ^ (tok & 7)) << 4)) = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
          }
          if (v && tile >= edge && tile * kTileTokens + tok > whole) {
            if (tile * kTileTokens + tok < e.t_end) {
              look_through<D>(row, tok, tile * kTileTokens + tok, notes + (n & 1) * kPtNotes, &bars->notes[n & 1]);
            } else {
#pragma unroll 1
              for (int i = 0; i < D / 8; ++i) *reinterpret_cast<uint4 *>(row + (i >> 3) * Cfg::kHalfBytes + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
          }
          fence_async_smem();
          warp_arrive(&bars->kv_full[slot], lane);
          warp_arrive(&bars->raw_empty[rs], lane);
        }
        if (bars->abort) break;
      }
      warp_arrive(&bars->item_clean[n & 1], lane);
      warp_arrive(&bars->item_empty[n & 1], lane);
    }
  } else {
    // ------------------------------------------------------------------ softmax and output
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Split::kSoftmax));
    const int x = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const uint32_t ts = tmem + Cfg::kColS + x * 128 + lane_addr, to = tmem + Cfg::kColO + x * D + lane_addr;
    const PromptNote *notes = p.notes + (int64_t)blockIdx.x * 2 * kPtNotes;
    __nv_bfloat16 *out = reinterpret_cast<__nv_bfloat16 *>(p.out);
    const bool sectors = (reinterpret_cast<uintptr_t>(out) & 31) == 0;
    const uint64_t scale2 = pair(p.scale_log2, p.scale_log2);
    const float *sScale = reinterpret_cast<const float *>(smem + Cfg::kOffScale);
    uint32_t n_s = 0, n_own = 0, n_tile = 0, n_turn = 0;
    PromptEntry e;
    for (uint32_t n = 0; next_item(n, e); ++n) {
      const int rows = min(e.rows - x * half_rows, half_rows);
      if (rows <= 0) {
        if constexpr (kCodes) {
#pragma unroll 1
          for (int tile = e.tile_begin; tile < e.tile_end && !bars->abort; ++tile, ++n_tile) {
            wait(&bars->sc_full[n_tile % kPtScaleSlots], n_tile / kPtScaleSlots, bars);
            warp_arrive(&bars->sc_empty[n_tile % kPtScaleSlots], lane);
          }
        }
        warp_arrive(&bars->item_empty[n & 1], lane);
        continue;
      }
      const int pr = e.row0 + x * half_rows + row;                       // packed row of the unit
      const bool active = quad * 32 < rows, valid = row < rows;
      const int limit = valid ? (causal ? e.vis0 + pr / p.G : e.vis0) : e.vis0 + (causal ? e.row0 / p.G : 0);   // last token the row sees
      const int whole = causal ? e.vis0 + (e.row0 + x * half_rows) / p.G : e.vis0;                               // ... and every row of the group
      // The warp of the other group on the same scheduler takes turns with this one at the exponentials: left alone the two fall into step, at the
      // exponential unit together and away from it together (the chunk of 500 rows behind 30,000 tokens 264 us, 249 with turns; a ragged
      // batch 302, 283).  Where codes are converted beside them turns only wait (six prompts over 8-bit pools: 477 without, 533 with).
      const bool turns = !kCodes && e.rows > half_rows + quad * 32;
      float m_ref = -INFINITY;
      bool fresh = true;          // some row of the warp has no reference yet
      uint64_t sum_a = pair(0.f, 0.f), sum_b = sum_a;
#pragma unroll 1
      for (int tile = e.tile_begin; tile < e.tile_end; ++tile, ++n_s, ++n_tile) {
        const float4 *factors = reinterpret_cast<const float4 *>(sScale + (n_tile % kPtScaleSlots) * 256);
        bool general = false;
        if constexpr (kCodes) {
          wait(&bars->sc_full[n_tile % kPtScaleSlots], n_tile / kPtScaleSlots, bars);
          general = bars->general[n_tile % kPtScaleSlots];
        }
        // what the power of two leaves of a scale
        auto factor = [](float scale) -> float {
          const uint32_t b = __float_as_uint(scale);
          return (b & 0x7f800000u) ? __uint_as_float((b & 0x7fffffu) | 0x3f800000u) : 1.f;
        };
        const int t0 = tile * kTileTokens;
        const bool edge = t0 + kTileTokens - 1 > whole;
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          wait(&bars->s_full[x][h], n_s, bars);
          fence_after();
          if (active) {
            const float4 *fk = factors + h * 16;
            const float2 *fv = reinterpret_cast<const float2 *>(factors + 32 + h * 16);
            uint32_t pk[32];
            uint64_t half_a, half_b;     // sums of the half's weights
            // The weights are made under the reference as it is; only if their sum is past 64 * 2^8 (or a row has no reference yet) is
            // the maximum taken, the reference moved and the weights made once more from the scores, which are still there.  (bf16
            // has fp32's exponents: large weights lose nothing; looking for the largest weight instead took 5% more time.)
            bool look = fresh, held = false;
#pragma unroll 1
            for (;;) {
              float s[64];
              uint32_t(&su)[2][32] = reinterpret_cast<uint32_t(&)[2][32]>(s);
              tmem_ld32(ts + h * 64, su[0]);
              tmem_ld32(ts + h * 64 + 32, su[1]);
              wait_ld();
              if (kCodes && general) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                  const float4 f = fk[i];
                  s[4 * i] *= factor(f.x); s[4 * i + 1] *= factor(f.y); s[4 * i + 2] *= factor(f.z); s[4 * i + 3] *= factor(f.w);
                }
              }
              if (edge) {
                const int last = limit - t0 - h * 64;
#pragma unroll
                for (int i = 0; i < 64; ++i) s[i] = i <= last ? s[i] : -INFINITY;
              }
              if (look) {
                float mx[2] = {s[0], s[1]};
#pragma unroll
                for (int i = 2; i < 64; i += 2) { mx[0] = fmaxf(mx[0], s[i]); mx[1] = fmaxf(mx[1], s[i + 1]); }
                const float top = fmaxf(mx[0], mx[1]) * p.scale_log2;
                float alpha = 1.f;
                bool rescale = false;
                if (m_ref == -INFINITY) {
                  m_ref = top;                        // (what is there so far is zero, or about to be overwritten)
                } else if (top > m_ref + kRescaleThreshold) {
                  alpha = fast_exp2(m_ref - top);
                  m_ref = top;
                  rescale = true;
                }
                if (__any_sync(0xffffffffu, rescale)) {
                  sum_a = e8::mul2(sum_a, pair(alpha, alpha));
                  sum_b = e8::mul2(sum_b, pair(alpha, alpha));
                  // The output has to be at rest: the half before this one is in it.  The scores that take its weights' place are
                  // made behind it; behind an entry's last tile there are none.
                  if (h == 0) wait(&bars->s_full[x][1], n_s, bars);
                  else if (tile + 1 < e.tile_end) wait(&bars->s_full[x][0], n_s + 1, bars);
                  else wait(&bars->h_done[x], n_own, bars);
                  fence_after();
#pragma unroll 1
                  for (int c = 0; c < D / 16; ++c) {
                    uint32_t r[16];
                    tmem_ld16(to + c * 16, r);
                    wait_ld();
#pragma unroll
                    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * alpha);
                    tmem_st16(to + c * 16, r);
                  }
                }
              }
              const float ref = m_ref == -INFINITY ? 0.f : -m_ref;
              const uint64_t ref2 = pair(ref, ref);
              if (look) fresh = __any_sync(0xffffffffu, m_ref == -INFINITY);
              half_a = half_b = pair(0.f, 0.f);
              if (turns && !held) wait(&bars->turn[x][quad], x == 0 ? n_turn ^ 1 : n_turn, bars);
              auto weights = [&](auto scaled) {
                constexpr int kBatch = 16, kHandOn = 48;
                auto consume = [&](int at) {
#pragma unroll
                  for (int i = 0; i < kBatch / 2; ++i) {
                    float a = s[at + 2 * i], b = s[at + 2 * i + 1];
                    if (i & 1) half_b = add2(half_b, pair(a, b));
                    else half_a = add2(half_a, pair(a, b));
                    if constexpr (decltype(scaled)::value) {
                      const float2 f = fv[at / 2 + i];
                      a *= factor(f.x);
                      b *= factor(f.y);
                    }
                    pk[at / 2 + i] = pack_bf16(a, b);
                  }
                };
#pragma unroll
                for (int at = 0; at < 64; at += kBatch) {
                  // (handed on a batch early: the other warp is a hundred cycles in coming)
                  if (at == kHandOn && turns && !held) { warp_arrive(&bars->turn[x ^ 1][quad], lane); ++n_turn; held = true; }
#pragma unroll
                  for (int i = 0; i < kBatch; i += 2) unpair(fma2(pair(s[at + i], s[at + i + 1]), scale2, ref2), s[at + i], s[at + i + 1]);
#pragma unroll
                  for (int i = 0; i < kBatch; ++i) s[at + i] = exp2_in_turn(s[at + i]);
                  if (at > 0) consume(at - kBatch);
                }
                consume(64 - kBatch);
              };
              if (kCodes && general) weights(std::true_type());
              else weights(std::false_type());
              float a, b;
              unpair(add2(half_a, half_b), a, b);
              if (look || !__any_sync(0xffffffffu, valid && !(a + b <= 16384.f))) break;   // (NaN too; rows that are none may hold anything)
              look = true;
            }
            sum_a = add2(sum_a, half_a);
            sum_b = add2(sum_b, half_b);
            tmem_st32(ts + h * 64, pk);
            wait_st();
          }
          fence_before();
          warp_arrive(&bars->p_full[x][h], lane);
        }
        if constexpr (kCodes) warp_arrive(&bars->sc_empty[n_tile % kPtScaleSlots], lane);
        if (bars->abort) break;
      }
      // ---- output
      wait(&bars->item_clean[n & 1], n >> 1, bars);
      const int n_notes = min(bars->notes[n & 1], kPtNotes);
      wait(&bars->o_full[x], n_own, bars);
      ++n_own;
      fence_after();
      if (active) {
        float l0, l1, l2, l3;
        unpair(sum_a, l0, l1);
        unpair(sum_b, l2, l3);
        const float l = (l0 + l1) + (l2 + l3);
        const int64_t qh = (int64_t)(e.q0 + pr / p.G) * p.Hq + e.g * p.G + pr % p.G;
        const int64_t part = (int64_t)e.slot * p.unit_rows + x * half_rows + row;
        const float inv = e.slot < 0 ? 1.f / l : 1.f;
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t r[32];
          tmem_ld32(to + c * 32, r);
          wait_ld();
          if (n_notes > 0) {
            uint32_t plus = 0, minus = 0;
#pragma unroll 1
            for (int i = 0; i < n_notes; ++i)
              if (notes[(n & 1) * kPtNotes + i].token <= limit) { plus |= notes[(n & 1) * kPtNotes + i].plus[c]; minus |= notes[(n & 1) * kPtNotes + i].minus[c]; }
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              float v = __uint_as_float(r[i]);
              if (plus >> i & 1) v += INFINITY;
              if (minus >> i & 1) v -= INFINITY;
              r[i] = __float_as_uint(v);
            }
          }
          if (valid && e.slot < 0) {
#pragma unroll
            for (int v = 0; v < 2; ++v) {
              uint32_t o[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) o[i] = pack_bf16(__uint_as_float(r[16 * v + 2 * i]) * inv, __uint_as_float(r[16 * v + 2 * i + 1]) * inv);
              store_sector(out + qh * D + c * 32 + v * 16, o, sectors);
            }
          } else if (valid) {
#pragma unroll
            for (int v = 0; v < 4; ++v) store_sector(p.part_o + part * D + c * 32 + v * 8, reinterpret_cast<const uint32_t(&)[8]>(r[8 * v]), true);
          }
          __syncwarp();
        }
        if (valid) {
          if (e.slot >= 0) p.part_ml[part] = make_float2(m_ref, l);
          else if (p.lse) p.lse[qh] = (m_ref + log2f(l)) * kLn2;
        }
      }
      fence_before();
      warp_arrive(&bars->o_free[x], lane);
      warp_arrive(&bars->item_empty[n & 1], lane);
    }
  }

  // ---------------------------------------------------------------------- teardown
  __syncwarp();
  if (bars->abort) {
    // give copies that are still in flight time to land before shared memory is released
    for (int i = 0; i < 1000; ++i) __nanosleep(1000);
  }
  fence_before();
  __syncthreads();
  if (warp == 9) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
  }
}

}  // namespace spx
