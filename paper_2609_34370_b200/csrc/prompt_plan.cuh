// Work plan and join for the attention of many query rows: whole prompts (causal, any number of new
// rows a request), and the shared prefix of a group of requests (every row sees all of it).
//
// A unit is a request, or a group of requests with the block-table row of its first and the query
// rows of all.  Its packed rows (position * G + head of the group) are cut into items of unit_rows rows;
// an item of a kv head is an entry, whose tiles of kTileTokens tokens are those its last row sees.
//
// Entries are independent, so the persistent kernel's CTAs take them through a counter, the longest first:
// the shorter ones then fill what the longer ones leave uneven.  Where there are too few of them for that (a chunk of a
// prompt behind a long history: 64 entries of 238 tiles for 148 CTAs), long entries are cut into equal pieces along the tokens,
// whose partial results a second kernel joins.  All items of a request are cut at the same tokens and are neighbours in the list,
// so that the CTAs that read the same tokens do so together (a range of the tiles for each CTA, cut where it fell, balanced
// better on paper and read the cache from HBM several times over: 250 to 420 us for that chunk, from board to board).  A latency chain: 7 to 11 us a plan,
// joins 1 us (24 prompts) to 23 (128 requests behind shared prefixes, 64 heads).
#pragma once
#include "common.cuh"
#include "plan.cuh"

namespace spx {

constexpr int kPromptBuckets = 1024;       // lengths the entries are sorted by (longer ones share the last)

struct PromptHeader {
  int32_t n_units;       // units of work: entries times kv heads
  int32_t counter;       // next unit of work
  int32_t n_join;        // items in pieces (prompts)
  int32_t any_bad;       // some request's rows are to be voided
};

// A piece of an item, or a whole one, for every kv head.
struct __align__(16) PromptEntry {
  int32_t unit;                  // request, or group
  int32_t table_row;             // block-table row
  int32_t q0;                    // first query row of the unit
  int32_t row0, rows;            // packed rows of the item
  int32_t vis0;                  // position j of the unit sees tokens 0 .. vis0 + j (causal), 0 .. vis0 (prefix)
  int32_t tile_begin, tile_end;
  int32_t t_end;                 // tokens the item's last row sees
  int32_t slot;                  // partial result of kv head 0 (the others' follow), -1: the entry is whole and goes to the output
  int32_t g;                     // kv head (filled in by the kernel that takes it)
  int32_t pad;
};
static_assert(sizeof(PromptEntry) == 48, "read as three 16-byte vectors");

// An item in pieces: piece c of kv head g is in slot first + c * Hkv + g.
struct __align__(16) PromptJoin {
  int32_t unit, q0, row0, rows;
  int32_t first, pieces, pad[2];
};

// Elements of a V row that are not finite, by column: infinities of either sign, NaN in both (prompt_tc.cuh).
struct __align__(16) PromptNote { uint32_t plus[4], minus[4]; int32_t token, pad[3]; };
constexpr int kPtNotes = 256;      // noted tokens of an item: those its rows do not all see, one per position at most

struct PromptParams {
  int32_t batch, total_q, Hq, Hkv, G, D, P, log2P, num_pages, max_pages_per_req;
  float scale_log2;
  const void *q, *k_cache, *v_cache;
  int64_t stride_page, stride_head, stride_token;
  const int32_t *block_table, *seq_lens, *q_indptr;
  void *out;
  float *lse;
  const float *k_scales, *v_scales;   // 8-bit pools
  int32_t log2SB;
  int32_t head_inner;                 // tensor-map dimension order
  int32_t box_rows;                   // query positions of one Q box
  int32_t *dev_status;
  // shared prefixes (groups = 0: prompts, causal)
  int32_t groups;
  const int32_t *group_indptr, *prefix_lens;
  int32_t *req_group;                 // [batch] group of a request, -1: none
  int32_t *group_tiles;               // [groups] tiles of the prefix that are read once, 0: none
  int32_t *req_flag;                  // [batch] 1: the block-table row differs from its group's
  // plan
  int32_t units;                      // batch or groups
  int32_t unit_rows;                  // packed rows of an item (whole positions in the tensor-core kernel)
  int32_t workers;                    // CTAs of the persistent kernel
  int32_t entry_cost, join_cost;      // of an entry's ends, of the join, in eighths of a tile
  int32_t min_piece;                  // tiles
  PromptHeader *hdr;
  int32_t *unit_item0;                // [units + 1]
  int32_t *unit_bad;                  // [units]
  int32_t *item_tiles;                // [max_items]
  PromptEntry *entries;               // [max_items + max_pieces]
  PromptJoin *join;                   // prompts: [max_pieces]
  int2 *item_part;                    // prefixes: [max_items] (first slot, pieces)
  int32_t max_items;
  int32_t max_pieces;                 // pieces that items are cut into; times Hkv slots, in front of those of a prefix plan's whole items
  float *part_o;                      // [slot][unit_rows][D]
  float2 *part_ml;                    // [slot][unit_rows]  (m in log2 units, l)
  PromptNote *notes;                  // [workers][2][kPtNotes]  (tensor-core kernel)
};

// Exclusive scan over the 1024 threads of a block; total in every thread.  scratch: 33 values of shared memory.
__device__ __forceinline__ int64_t scan_1024(int64_t v, int64_t *scratch, int64_t &total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t n = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += n;
  }
  __syncthreads();
  if (lane == 31) scratch[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    const int64_t w = scratch[lane];
    int64_t wi = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t n = __shfl_up_sync(0xffffffffu, wi, o);
      if (lane >= o) wi += n;
    }
    scratch[lane] = wi - w;
    if (lane == 31) scratch[32] = wi;
  }
  __syncthreads();
  total = scratch[32];
  return scratch[warp] + incl - v;
}

// largest i in [0, n) with a[i] <= x (a ascending, a[0] <= x)
template <typename T, typename X>
__device__ __forceinline__ int last_at_most(const T *a, int n, X x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// What a unit is: first query row, positions, tokens, block-table row, whether it is to be voided.
struct PromptUnit { int q0, m, L, row; bool bad; };
__device__ __forceinline__ PromptUnit prompt_unit(const PromptParams &p, int u) {
  PromptUnit x{0, 0, 0, 0, false};
  if (p.groups == 0) {
    const int q0 = p.q_indptr[u], q1 = p.q_indptr[u + 1], L = p.seq_lens[u];
    x.q0 = q0; x.m = q1 - q0; x.L = L; x.row = u;
    x.bad = q0 < 0 || q1 < q0 || q1 > p.total_q || L < x.m || (((int64_t)L + p.P - 1) >> p.log2P) > (int64_t)p.max_pages_per_req;
    if (x.bad) x.m = 0;
    return x;
  }
  const int r0 = max(p.group_indptr[u], 0), r1 = min(p.group_indptr[u + 1], p.batch), len = p.prefix_lens[u];
  if (r1 - r0 < 2 || len < kTileTokens) return x;             // nobody to share with, nothing to share
  const int q0 = p.q_indptr[r0], q1 = p.q_indptr[r1];
  if (q0 < 0 || q1 <= q0 || q1 > p.total_q) return x;         // (the requests' own check voids them)
  const int tokens = len / kTileTokens * kTileTokens;
  if ((tokens >> p.log2P) > p.max_pages_per_req) return x;
  x.q0 = q0; x.m = q1 - q0; x.L = tokens; x.row = r0;
  return x;
}
// The group of a request, -1: none.
__device__ __forceinline__ int prompt_group_of(const PromptParams &p, int r) {
  if (p.group_indptr[0] > r) return -1;
  const int u = last_at_most(p.group_indptr, p.groups, r);
  return r < p.group_indptr[u + 1] ? u : -1;
}

// One block of 1024 threads.
__device__ __forceinline__ void prompt_plan_block(const PromptParams &p) {
  const int tid = threadIdx.x;
  __shared__ int64_t s_scratch[33];
  __shared__ int s_hist[kPromptBuckets];
  __shared__ int s_longest, s_bad;
  __shared__ long long s_best;
  using Unit = PromptUnit;
  auto unit_of = [&](int u) -> Unit { return prompt_unit(p, u); };
  for (int i = tid; i < kPromptBuckets; i += 1024) s_hist[i] = 0;
  if (tid == 0) { s_longest = 0; s_bad = 0; s_best = 0x7fffffffffffffffll; }
  __syncthreads();

  // items of the units
  int64_t n_items = 0, total;
  for (int base = 0; base < p.units; base += 1024) {
    const int u = base + tid;
    int64_t n = 0;
    if (u < p.units) {
      const Unit x = unit_of(u);
      n = ((int64_t)x.m * p.G + p.unit_rows - 1) / p.unit_rows;
      p.unit_bad[u] = x.bad;
      if (x.bad) s_bad = 1;
      if (p.groups) p.group_tiles[u] = x.m > 0 ? x.L / kTileTokens : 0;
    }
    const int64_t off = scan_1024(n, s_scratch, total) + n_items;
    n_items += total;
    if (u < p.units) p.unit_item0[u] = (int)min(off, (int64_t)p.max_items);
  }
  if (n_items > p.max_items) n_items = p.max_items;   // (only where q_indptr, or the bounds of groups, descend somewhere)
  if (tid == 0) p.unit_item0[p.units] = (int)n_items;
  __syncthreads();
  const int NI = (int)n_items;

  // tiles of the items, and how many there are of each length
  for (int i = tid; i < NI; i += 1024) {
    const int u = last_at_most(p.unit_item0, p.units, i);   // (units without items start where the next one does)
    const Unit x = unit_of(u);
    const int64_t row0 = (int64_t)(i - p.unit_item0[u]) * p.unit_rows;
    const int64_t last = (min(row0 + p.unit_rows, (int64_t)x.m * p.G) - 1) / p.G;
    const int64_t seen = p.groups ? (int64_t)x.L : (int64_t)x.L - x.m + last + 1;
    const int tiles = (int)((seen + kTileTokens - 1) / kTileTokens);
    p.item_tiles[i] = tiles;
    atomicAdd(&s_hist[min(tiles, kPromptBuckets) - 1], 1);
    atomicMax(&s_longest, tiles);
  }
  __syncthreads();

  // Pieces of at most `piece` tiles: each warp works out what cutting the longest item into n would take (in eighths of a tile): the
  // work for each CTA, the longest piece, and the rounds that the pieces of the longer half need.  (Items past the last
  // bucket count as long as the longest.)
  const int longest = s_longest;
  auto pieces_of = [](int tiles, int piece) -> int { return (tiles + piece - 1) / piece; };
  {
    const int warp = tid >> 5, lane = tid & 31;
    const int n = warp < 16 ? warp + 1 : warp < 24 ? 16 + 4 * (warp - 15) : 48 + 16 * (warp - 23);   // 1 .. 16, 20 .. 48, 64 .. 176
    const int piece = max(max(1, p.min_piece), pieces_of(longest, n));
    int64_t work = 0, cut = 0, most = 0, big = 0, big_len = 0;
    if (n == 1 || pieces_of(longest, n) >= p.min_piece) {
      for (int b = lane; b < min(longest, kPromptBuckets); b += 32) {
        const int64_t count = (int64_t)s_hist[b] * p.Hkv;
        if (count == 0) continue;
        const int tiles = b == kPromptBuckets - 1 ? longest : b + 1, k = pieces_of(tiles, piece), len = pieces_of(tiles, k);
        work += count * (8 * (int64_t)tiles + (int64_t)k * p.entry_cost);
        if (k > 1) cut += count * k;
        most = max(most, (int64_t)len);
        if (2 * len > piece) { big += count * k; big_len += count * k * len; }
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      work += __shfl_xor_sync(0xffffffffu, work, o); cut += __shfl_xor_sync(0xffffffffu, cut, o);
      big += __shfl_xor_sync(0xffffffffu, big, o); big_len += __shfl_xor_sync(0xffffffffu, big_len, o);
      most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    }
    if (lane == 0 && work > 0 && cut <= (int64_t)p.max_pieces * p.Hkv) {
      int64_t time = max(work / p.workers, 8 * most + p.entry_cost);
      if (big > 0) time = max(time, (big + p.workers - 1) / p.workers * (8 * big_len / big + p.entry_cost));
      if (cut > 0) time += p.join_cost;
      atomicMin(&s_best, (long long)(time << 8 | n));
    }
  }
  __syncthreads();
  const int best = NI > 0 ? (int)(s_best & 255) : 1, piece = max(max(1, p.min_piece), pieces_of(max(longest, 1), best));
  const int piece_of_all = best == 1 ? 1 << 30 : piece;   // (tiles are below 2^24)

  // places of the pieces: sorted by length, the longest first; their slots
  __syncthreads();
  if (best > 1) {   // lengths of pieces now, not of items
    for (int i = tid; i < kPromptBuckets; i += 1024) s_hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < NI; i += 1024) {
      const int tiles = p.item_tiles[i], k = pieces_of(tiles, piece_of_all);
      atomicAdd(&s_hist[min(pieces_of(tiles, k), kPromptBuckets) - 1], k);
    }
    __syncthreads();
  }
  const int place = (int)scan_1024(s_hist[kPromptBuckets - 1 - tid], s_scratch, total);
  const int n_entries = (int)total;
  __syncthreads();
  s_hist[kPromptBuckets - 1 - tid] = place;
  __syncthreads();
  int64_t slots = 0, joins = 0;
  for (int base = 0; base < NI; base += 1024) {
    const int i = base + tid;
    const int tiles = i < NI ? p.item_tiles[i] : 0, k = i < NI ? pieces_of(tiles, piece_of_all) : 0;
    const int64_t slot = scan_1024(k > 1 ? k : 0, s_scratch, total) + slots;
    slots += total;
    int64_t at_join = 0;
    if (!p.groups) {   // (those of a prefix are joined with the requests' own tokens, item by item)
      at_join = scan_1024(k > 1 ? 1 : 0, s_scratch, total) + joins;
      joins += total;
    }
    if (i >= NI) continue;
    PromptEntry e;
    const int u = last_at_most(p.unit_item0, p.units, i);
    const Unit x = unit_of(u);
    const int64_t row0 = (int64_t)(i - p.unit_item0[u]) * p.unit_rows, all = (int64_t)x.m * p.G;
    e.unit = u; e.table_row = x.row; e.q0 = x.q0;
    e.row0 = (int)row0; e.rows = (int)min((int64_t)p.unit_rows, all - row0);
    e.vis0 = p.groups ? x.L - 1 : x.L - x.m;
    e.t_end = p.groups ? x.L : x.L - x.m + (e.row0 + e.rows - 1) / p.G + 1;
    e.g = 0; e.pad = 0;
    const int first = k > 1 ? (int)slot * p.Hkv : (p.max_pieces + i) * p.Hkv;   // (behind the pieces' slots: whole items of a prefix plan)
    const int len = pieces_of(tiles, k);
    int at = atomicAdd(&s_hist[min(len, kPromptBuckets) - 1], k);
    for (int c = 0; c < k; ++c, ++at) {
      e.tile_begin = min(c * len, tiles); e.tile_end = min(e.tile_begin + len, tiles);
      e.slot = k > 1 || p.groups ? first + c * p.Hkv : -1;
      p.entries[at] = e;
    }
    if (p.groups) {
      p.item_part[i] = make_int2(first, k);
    } else if (k > 1) {
      PromptJoin j;
      j.unit = u; j.q0 = e.q0; j.row0 = e.row0; j.rows = e.rows; j.first = first; j.pieces = k; j.pad[0] = j.pad[1] = 0;
      p.join[at_join] = j;
    }
  }
  if (tid == 0) {
    p.hdr->n_units = n_entries * p.Hkv;
    p.hdr->counter = 0;
    p.hdr->n_join = (int)joins;
    p.hdr->any_bad = s_bad;
    if (s_bad) atomicOr(p.dev_status, SPX_DEV_BAD_LEN);
  }
}

__global__ void __launch_bounds__(1024) prompt_plan_kernel(PromptParams p) {
  SPX_TL_SCOPE(kTlPlan);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  prompt_plan_block(p);
}

// Block 0 plans the prefixes of the groups, block 1 the requests' own tokens behind them.  The blocks behind compare the block-table
// rows of the requests with their groups' first, so that a request that does not share what its group reads once is found,
// not answered wrongly.
__global__ void __launch_bounds__(1024) prefix_plan_kernel(AttnParams a, PromptParams p, int n_cta) {
  SPX_TL_SCOPE(kTlPlan);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (blockIdx.x == 0) {
    prompt_plan_block(p);
  } else if (blockIdx.x == 1) {
    plan_block<true>(a, n_cta, [&](int r) -> int {
      const int u = prompt_group_of(p, r);
      return u < 0 ? 0 : prompt_unit(p, u).L / kTileTokens;
    });
  } else {
    // a warp a request (few blocks: in the whole step they share the one SM that the logits pass leaves)
    const int lane = threadIdx.x & 31;
    for (int r = (blockIdx.x - 2) * 32 + (threadIdx.x >> 5); r < p.batch; r += (gridDim.x - 2) * 32) {
      const int u = prompt_group_of(p, r);
      int differs = 0;
      PromptUnit x{0, 0, 0, 0, false};
      if (u >= 0) x = prompt_unit(p, u);
      if (x.m > 0) {
        const int32_t *mine = p.block_table + (int64_t)r * p.max_pages_per_req, *first = p.block_table + (int64_t)x.row * p.max_pages_per_req;
#pragma unroll 8
        for (int i = lane; i < x.L >> p.log2P; i += 32) differs |= mine[i] ^ first[i];
      }
      differs = __any_sync(0xffffffffu, differs != 0);
      if (lane == 0) {
        p.req_group[r] = u;
        p.req_flag[r] = differs;
        if (differs) atomicOr(p.dev_status, SPX_DEV_BAD_PAGE);
      }
    }
  }
}

__device__ __forceinline__ void store4(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

// Joins the pieces of items (see combine_kernel) and voids the rows of requests with a bad length or page id.
// Blocks (b, y): kv head b mod Hkv of item b / Hkv of the list, (row, four columns) y * 256 + t of it.
template <typename T>
__global__ void __launch_bounds__(256) prompt_join_kernel(PromptParams p) {
  SPX_TL_SCOPE(kTlCombine);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  T *out = reinterpret_cast<T *>(p.out);
  const int vecs = p.D / 4;
  const int n_join = p.hdr->n_join, any_bad = p.hdr->any_bad;
  for (int li = blockIdx.x; li < n_join * p.Hkv; li += gridDim.x) {
    const PromptJoin e = p.join[li / p.Hkv];
    const int g = li % p.Hkv;
    if (p.unit_bad[e.unit]) continue;
    for (int item = blockIdx.y * blockDim.x + threadIdx.x; item < e.rows * vecs; item += gridDim.y * blockDim.x) {
      const int row = item / vecs, dv = item % vecs;
      float mstar = -INFINITY, lstar = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      auto slot_row = [&](int c) -> int64_t { return (int64_t)(e.first + c * p.Hkv + g) * p.unit_rows + row; };
      for (int c0 = 0; c0 < e.pieces; c0 += 4) {
        // four chunks' loads in flight at a time, their maximum taken first
        float2 ml[4];
        float4 o[4];
        float top = mstar;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int64_t at = slot_row(min(c0 + u, e.pieces - 1));
          ml[u] = p.part_ml[at];
          o[u] = *reinterpret_cast<const float4 *>(p.part_o + at * p.D + dv * 4);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (c0 + u < e.pieces) top = fmaxf(top, ml[u].x);
        if (mstar != -INFINITY && top > mstar) {
          const float w = fast_exp2(mstar - top);
          lstar = rescaled_sum(lstar, mstar - top);
          acc.x *= w; acc.y *= w; acc.z *= w; acc.w *= w;
        }
        mstar = top;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (c0 + u >= e.pieces || (ml[u].x == -INFINITY && ml[u].y == 0.f)) continue;   // (saw nothing)
          const float d = ml[u].x == -INFINITY ? 0.f : ml[u].x - mstar, w = fast_exp2(d);
          lstar += rescaled_sum(ml[u].y, d);
          acc.x += w * o[u].x; acc.y += w * o[u].y; acc.z += w * o[u].z; acc.w += w * o[u].w;
        }
      }
      const int pr = e.row0 + row, h = g * p.G + pr % p.G;
      const int64_t qrow = e.q0 + pr / p.G, at = (qrow * p.Hq + h) * p.D + dv * 4;
      const float inv = 1.f / lstar;
      store4(out + at, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
      if (dv == 0 && p.lse) p.lse[qrow * p.Hq + h] = (mstar + log2f(lstar)) * kLn2;
    }
  }
  if (!any_bad) return;
  // zero rows, NaN lse, all blocks together (the rows of a request whose own bounds make no sense stay as they are)
  const int64_t first = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * gridDim.y * blockDim.x;
  for (int r = 0; r < p.batch; ++r) {
    if (!p.unit_bad[r]) continue;
    const int q0 = p.q_indptr[r], q1 = p.q_indptr[r + 1];
    if (q0 < 0 || q1 < q0 || q1 > p.total_q) continue;
    const int64_t rows = (int64_t)(q1 - q0) * p.Hq, base = (int64_t)q0 * p.Hq;
    for (int64_t i = first; i < rows * p.D; i += step) st_from_float(out, base * p.D + i, 0.f);
    if (p.lse)
      for (int64_t i = first; i < rows; i += step) p.lse[base + i] = __int_as_float(0x7fc00000);
  }
}

// Joins a request's partial results of its group's prefix with those of its own tokens.  Block (r, y): request r, items (position,
// head, four columns) y * 256 + t.  a: the plan of the requests' own tokens; p: that of the prefixes.
constexpr int kJoinHeads = 128;                              // kv heads whose chunks are kept in shared memory
constexpr int kJoinItems = SPX_MAX_PACKED_ROWS / 64 + 2;     // items (of 64 rows at least) that a request's rows can lie in
template <typename T>
__global__ void __launch_bounds__(256) prefix_join_kernel(AttnParams a, PromptParams p) {
  SPX_TL_SCOPE(kTlCombine);
  // The plans are read ahead of the wait for the attention kernel, which has read them itself when it lets this one up.
  const int r = blockIdx.x;
  T *out = reinterpret_cast<T *>(a.out);
  const int vecs = a.D / 4, G = a.G;
  const int q0 = a.q_indptr[r], u = p.req_group[r];
  int m = a.q_indptr[r + 1] - q0;
  if (m < 0) m = 0;
  if (m > a.max_q_len) m = a.max_q_len;
  const bool inside = q0 >= 0 && (int64_t)q0 + m <= a.total_q;
  const int tiles = u >= 0 ? p.group_tiles[u] : 0;
  int item0 = 0;
  int64_t row0 = 0;    // the request's first packed row among its group's
  bool bad = false;
  if (tiles > 0) {
    item0 = p.unit_item0[u];
    row0 = (int64_t)(q0 - p.q_indptr[max(p.group_indptr[u], 0)]) * G;
    bad = row0 < 0 || row0 + (int64_t)m * G > (int64_t)(p.unit_item0[u + 1] - item0) * p.unit_rows;
  }
  // chunks and first slots of the request's pairs, and of the few items that its rows lie in
  __shared__ int2 s_pair[kJoinHeads], s_part[kJoinItems];
  const int64_t first_item = row0 / p.unit_rows;
  const int row_in = (int)(row0 - first_item * p.unit_rows);   // of the request's first packed row
  for (int g = threadIdx.x; g < min(a.Hkv, kJoinHeads); g += blockDim.x) s_pair[g] = make_int2(a.pair_nchunks[r * a.Hkv + g], a.pair_part_base[r * a.Hkv + g]);
  if (tiles > 0 && !bad && threadIdx.x < kJoinItems && item0 + first_item + threadIdx.x < p.unit_item0[u + 1]) s_part[threadIdx.x] = p.item_part[item0 + first_item + threadIdx.x];
  __syncthreads();
  const int n_items = inside ? m * a.Hq * vecs : 0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  bad = bad || a.req_bad[r] || p.req_flag[r] || (u >= 0 && p.unit_bad[u]);
#pragma unroll 2
  for (int item = blockIdx.y * blockDim.x + threadIdx.x; item < n_items; item += gridDim.y * blockDim.x) {
    const int dv = item % vecs, jh = item / vecs, h = jh % a.Hq, j = jh / a.Hq, g = h / G, hg = h % G;
    const int2 own = g < kJoinHeads ? s_pair[g] : make_int2(a.pair_nchunks[r * a.Hkv + g], a.pair_part_base[r * a.Hkv + g]);
    const int nch = own.x, base = own.y;
    const int64_t qh = (int64_t)(q0 + j) * a.Hq + h, at = qh * a.D + dv * 4;
    if (bad || nch == 0) {
      store4(out + at, make_float4(0.f, 0.f, 0.f, 0.f));
      if (dv == 0 && a.lse) a.lse[qh] = __int_as_float(0x7fc00000);
      continue;
    }
    int2 part = make_int2(0, 0);     // first slot, pieces
    int64_t prow = 0;
    if (tiles > 0) {
      int row = row_in + j * G + hg, it = 0;
      while (row >= p.unit_rows) { row -= p.unit_rows; ++it; }
      part = s_part[it];
      prow = row;
    }
    float mstar = -INFINITY, lstar = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const int n = nch + part.y;
    for (int c0 = 0; c0 < n; c0 += 4) {
      float2 ml[4];
      float4 o[4];
      float top = mstar;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = min(c0 + i, n - 1) - nch;    // below zero: the request's own
        const float2 *ml_at;
        const float *o_at;
        if (c < 0) {
          const int64_t s = (int64_t)(base + c + nch) * a.rows_cap + j * G + hg;
          ml_at = a.part_ml + s; o_at = a.part_o + s * a.D;
        } else {
          const int64_t s = (int64_t)(part.x + c * p.Hkv + g) * p.unit_rows + prow;
          ml_at = p.part_ml + s; o_at = p.part_o + s * a.D;
        }
        ml[i] = *ml_at;
        o[i] = *reinterpret_cast<const float4 *>(o_at + dv * 4);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c0 + i < n) top = fmaxf(top, ml[i].x);
      if (mstar != -INFINITY && top > mstar) {
        const float w = fast_exp2(mstar - top);
        lstar = rescaled_sum(lstar, mstar - top);
        acc.x *= w; acc.y *= w; acc.z *= w; acc.w *= w;
      }
      mstar = top;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (c0 + i >= n || (ml[i].x == -INFINITY && ml[i].y == 0.f)) continue;
        const float d = ml[i].x == -INFINITY ? 0.f : ml[i].x - mstar, w = fast_exp2(d);
        lstar += rescaled_sum(ml[i].y, d);
        acc.x += w * o[i].x; acc.y += w * o[i].y; acc.z += w * o[i].z; acc.w += w * o[i].w;
      }
    }
    const float inv = 1.f / lstar;
    store4(out + at, make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
    if (dv == 0 && a.lse) a.lse[qh] = (mstar + log2f(lstar)) * kLn2;
  }
}

}  // namespace spx
