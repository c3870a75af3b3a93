// Work plan and join for the attention of many query rows: whole prompts (causal, any number of new
// rows a request), and the shared prefix of a group of requests (every row sees all of it).
//
// A unit is a request, or a group of requests with the block-table row of its first and the query
// rows of all.  Its packed rows (position * G + head of the group) are cut into items of unit_rows rows;
// an item of a kv head is an entry, whose tiles of kTileTokens tokens are those its last row sees.
//
// Entries are independent, so the persistent kernel's CTAs take them through a counter, the longest first:
// the shorter ones then fill what the longer ones leave uneven.  Where there are too few of them for that (a chunk of a
// prompt behind a long history: 64 entries of 238 tiles), the axis of all entries' tiles is cut into ranges of equal cost
// instead, one for each CTA; the parts of an entry that a cut crosses are joined by a second kernel.
#pragma once
#include "common.cuh"

namespace spx {

constexpr int kPromptMaxWorkers = 512;     // ranges
constexpr int kPromptMaxRanged = 8192;     // entries of a plan that is cut into ranges
constexpr int kPromptBuckets = 1024;       // lengths the entries are sorted by (longer ones share the last)

struct PromptHeader {
  int32_t n_units;       // units of work: entries (ranged = 0) or ranges (ranged = 1)
  int32_t ranged;
  int32_t counter;       // next unit of work
  int32_t n_items;       // items of all units
  int32_t n_join;        // entries to be joined (ranged plans of whole outputs)
  int32_t any_bad;       // some request's rows are to be voided
  int32_t pad[2];
};

struct __align__(16) PromptEntry {
  int32_t unit;                  // request, or group
  int32_t table_row;             // block-table row
  int32_t q0;                    // first query row of the unit
  int32_t row0, rows;            // packed rows of the item
  int32_t vis0;                  // position j of the unit sees tokens 0 .. vis0 + j (causal), 0 .. vis0 (prefix)
  int32_t tile_begin, tile_end;
  int32_t t_end;                 // tokens the item's last row sees
  int32_t slot;                  // partial result, -1: the entry is whole and goes to the output
  int32_t g;                     // kv head (ranged plans)
  int32_t pad;
};
static_assert(sizeof(PromptEntry) == 48, "read as three 16-byte vectors");

// An entry's partial results: chunk 0 in slot first, chunk j in slot next + 2 (j - 1).
struct __align__(16) PromptJoin {
  int32_t unit, q0, row0, rows;
  int32_t g, first, next, nch;
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
  int32_t min_range, overhead;        // tiles: the shortest range worth a CTA, what cuts cost
  int32_t entry_cost;                 // of an entry's ends, in eighths of a tile
  PromptHeader *hdr;
  int32_t *unit_item0;                // [units + 1]
  int32_t *unit_bad;                  // [units]
  int32_t *item_tiles;                // [max_items]
  int64_t *item_cost;                 // [max_items + 1]
  PromptEntry *entries;               // [max_entries]
  int32_t *range_off;                 // [workers + 1]
  PromptJoin *join;                   // [workers]
  int4 *entry_part;                   // prefixes: [max_items * Hkv] (first, next, chunks, 0)
  int32_t max_items, max_entries, whole_slot0;
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

// Block 0 plans.  Of a plan over groups the blocks behind it compare the block-table rows of the requests with
// their groups' first, so that a request that does not share what its group reads once is found, not answered wrongly.
__global__ void __launch_bounds__(1024) prompt_plan_kernel(PromptParams p) {
  SPX_TL_SCOPE(kTlPlan);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x;
  __shared__ int64_t s_scratch[33];
  __shared__ int s_off[kPromptMaxWorkers + 1], s_cut_e[kPromptMaxWorkers + 1], s_cut_t[kPromptMaxWorkers + 1];
  __shared__ int s_hist[kPromptBuckets];
  __shared__ int s_level, s_longest, s_bad;

  // what a unit is: first query row, positions, tokens, block-table row, whether it is to be voided
  struct Unit { int q0, m, L, row; bool bad; };
  auto unit_of = [&](int u) -> Unit {
    Unit x{0, 0, 0, 0, false};
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
  };

  if (blockIdx.x > 0) {
    // one block a request
    for (int r = blockIdx.x - 1; r < p.batch; r += gridDim.x - 1) {
      // its group (requests that no group holds share nothing)
      __syncthreads();
      if (tid == 0) s_level = -1;
      __syncthreads();
      for (int i = tid; i < p.groups; i += blockDim.x)
        if (p.group_indptr[i] <= r && r < p.group_indptr[i + 1]) atomicMax(&s_level, i);
      __syncthreads();
      const int u = s_level;
      if (tid == 0) p.req_group[r] = u;
      int differs = 0;
      if (u >= 0) {
        const Unit x = unit_of(u);
        if (x.m > 0) {
          const int32_t *mine = p.block_table + (int64_t)r * p.max_pages_per_req, *first = p.block_table + (int64_t)x.row * p.max_pages_per_req;
          for (int i = tid; i < x.L >> p.log2P; i += blockDim.x) differs |= mine[i] != first[i];
        }
      }
      differs = __syncthreads_or(differs);
      if (tid == 0) {
        p.req_flag[r] = differs != 0;
        if (differs) atomicOr(p.dev_status, SPX_DEV_BAD_PAGE);
      }
    }
    return;
  }

  for (int i = tid; i < kPromptBuckets; i += 1024) s_hist[i] = 0;
  if (tid == 0) { s_level = kPromptBuckets; s_longest = 0; s_bad = 0; }
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
  if (n_items > p.max_items) n_items = p.max_items;   // (cannot be: the units' rows do not overlap)
  if (tid == 0) p.unit_item0[p.units] = (int)n_items;
  __syncthreads();
  const int NI = (int)n_items;

  // tiles of the items, their sum and how many there are of each length
  const int entry_cost = p.entry_cost;   // an entry's ends, in eighths of a tile
  int64_t cost_sum = 0, tile_sum = 0;
  for (int base = 0; base < NI; base += 1024) {
    const int i = base + tid;
    int tiles = 0;
    if (i < NI) {
      const int u = last_at_most(p.unit_item0, p.units, i);   // (units without items start where the next one does)
      const Unit x = unit_of(u);
      const int64_t row0 = (int64_t)(i - p.unit_item0[u]) * p.unit_rows;
      const int64_t last = (min(row0 + p.unit_rows, (int64_t)x.m * p.G) - 1) / p.G;
      const int64_t seen = p.groups ? (int64_t)x.L : (int64_t)x.L - x.m + last + 1;
      tiles = (int)((seen + kTileTokens - 1) / kTileTokens);
      p.item_tiles[i] = tiles;
      atomicAdd(&s_hist[min(tiles, kPromptBuckets) - 1], 1);
      atomicMax(&s_longest, tiles);
    }
    const int64_t off = scan_1024(i < NI ? 8 * (int64_t)tiles + entry_cost : 0, s_scratch, total) + cost_sum;
    cost_sum += total;
    if (i < NI) p.item_cost[i] = off;
    scan_1024(tiles, s_scratch, total);
    tile_sum += total;
  }
  if (tid == 0) p.item_cost[NI] = cost_sum;
  __syncthreads();

  // How long does taking whole entries, the longest first, take?  Entries up to the level x fill what those above it leave
  // uneven if there are x tiles of them for each worker; past that the last entries are x long.
  const int64_t N = (int64_t)NI * p.Hkv, T = tile_sum * p.Hkv;
  {
    int64_t work = tid < kPromptBuckets ? (int64_t)s_hist[tid] * (tid + 1) * p.Hkv : 0;
    const int64_t below = scan_1024(work, s_scratch, total) + work;
    if (below >= (int64_t)p.workers * (tid + 1)) atomicMin(&s_level, tid + 1);
    __syncthreads();
  }
  const int64_t even = (T + p.workers - 1) / p.workers;
  const int64_t whole = N <= p.workers ? s_longest : min(even + s_level, (N + p.workers - 1) / p.workers * (int64_t)s_longest);
  const int n_ranges = (int)max((int64_t)1, min((int64_t)p.workers, T / p.min_range));
  const int64_t cut = (T + n_ranges - 1) / n_ranges + p.overhead;
  const bool ranged = N <= kPromptMaxRanged && N > 0 && cut < whole;

  auto entry_of = [&](int i) -> PromptEntry {
    PromptEntry e;
    const int u = last_at_most(p.unit_item0, p.units, i);
    const Unit x = unit_of(u);
    const int64_t row0 = (int64_t)(i - p.unit_item0[u]) * p.unit_rows, all = (int64_t)x.m * p.G;
    e.unit = u; e.table_row = x.row; e.q0 = x.q0;
    e.row0 = (int)row0; e.rows = (int)min((int64_t)p.unit_rows, all - row0);
    e.vis0 = p.groups ? x.L - 1 : x.L - x.m;
    e.tile_begin = 0; e.tile_end = p.item_tiles[i];
    e.t_end = p.groups ? x.L : x.L - x.m + (e.row0 + e.rows - 1) / p.G + 1;
    e.slot = -1; e.g = 0; e.pad = 0;
    return e;
  };

  if (!ranged) {
    // sorted by length, the longest first: a bucket's first place, then a place for each of its entries
    const int mine = tid < kPromptBuckets ? s_hist[kPromptBuckets - 1 - tid] : 0;
    const int place = (int)scan_1024(mine, s_scratch, total);
    __syncthreads();
    if (tid < kPromptBuckets) s_hist[kPromptBuckets - 1 - tid] = place;
    __syncthreads();
    for (int i = tid; i < NI; i += 1024) {
      PromptEntry e = entry_of(i);
      const int at = atomicAdd(&s_hist[min(e.tile_end, kPromptBuckets) - 1], 1);
      if (p.groups) {
        e.slot = p.whole_slot0 + i * p.Hkv;   // plus the kv head, which the kernel knows
        for (int g = 0; g < p.Hkv; ++g) p.entry_part[(int64_t)i * p.Hkv + g] = make_int4(e.slot + g, 0, 1, 0);
      }
      p.entries[at] = e;
    }
  } else {
    // cuts at equal steps of the cost axis of all entries (item, kv head), moved onto an entry's end if close to one
    const int snap = max(1, min(p.min_range / 2, 3));
    if (tid <= n_ranges) {
      int e = 0, t = 0;
      if (tid == n_ranges) {
        e = (int)N;
      } else if (tid > 0) {
        const int64_t x = (int64_t)((double)cost_sum * p.Hkv * tid / n_ranges);
        const int i = last_at_most(p.item_cost, NI, x / p.Hkv);
        const int tiles = p.item_tiles[i], c = 8 * tiles + entry_cost;
        const int64_t rel = x - p.item_cost[i] * p.Hkv;
        int g = (int)min(rel / c, (int64_t)p.Hkv - 1);
        t = (int)max((int64_t)0, (rel - (int64_t)g * c - entry_cost) / 8);
        if (t < snap) t = 0;
        else if (tiles - t < snap) { t = 0; ++g; }
        e = i * p.Hkv + g;
      }
      s_cut_e[tid] = e; s_cut_t[tid] = t;
    }
    __syncthreads();
    int n = 0;
    if (tid < n_ranges) n = max(0, s_cut_e[tid + 1] - s_cut_e[tid] + (s_cut_t[tid + 1] > 0 ? 1 : 0));
    if (tid < n_ranges && s_cut_e[tid + 1] == s_cut_e[tid] && s_cut_t[tid + 1] <= s_cut_t[tid]) n = 0;   // two cuts in one place
    const int off = (int)scan_1024(n, s_scratch, total);
    if (tid <= n_ranges) { s_off[tid] = tid < n_ranges ? off : (int)total; p.range_off[tid] = s_off[tid]; }
    __syncthreads();
    // (an entry that a cut opens: its first part belongs to the range before the cut, whose last entry it is)
    for (int k = tid; k < s_off[n_ranges]; k += 1024) {
      const int c = last_at_most(s_off, n_ranges, k);   // (empty ranges start where the next one does)
      const int e = s_cut_e[c] + k - s_off[c];
      PromptEntry x = entry_of(e / p.Hkv);
      x.g = e % p.Hkv;
      const int tiles = x.tile_end;
      if (e == s_cut_e[c]) x.tile_begin = s_cut_t[c];
      if (e == s_cut_e[c + 1]) x.tile_end = s_cut_t[c + 1];
      if (x.tile_begin > 0) x.slot = 2 * c;
      else if (x.tile_end < tiles) x.slot = 2 * c + 1;
      else if (p.groups) {
        x.slot = p.whole_slot0 + e;
        p.entry_part[e] = make_int4(x.slot, 0, 1, 0);
      }
      p.entries[k] = x;
    }
  }
  // the entries that cuts open: the first cut inside one tells how many there are
  int joins = 0;
  if (ranged && tid >= 1 && tid < n_ranges && s_cut_t[tid] > 0) {
    // the first cut in the entry, and the one whose range is not empty among equal ones
    const bool first = s_cut_e[tid - 1] != s_cut_e[tid] || s_cut_t[tid - 1] == 0;
    if (first) joins = 1;
  }
  const int at = (int)scan_1024(joins, s_scratch, total);
  const int n_join = ranged ? (int)total : 0;
  if (joins) {
    const int e = s_cut_e[tid];
    int nch = 1;
    for (int c = tid; c < n_ranges && s_cut_e[c] == e && s_cut_t[c] > 0; ++c) ++nch;
    const PromptEntry x = entry_of(e / p.Hkv);
    PromptJoin j;
    j.unit = x.unit; j.q0 = x.q0; j.row0 = x.row0; j.rows = x.rows; j.g = e % p.Hkv;
    j.first = 2 * (tid - 1) + 1; j.next = 2 * tid; j.nch = nch;
    if (p.groups) p.entry_part[e] = make_int4(j.first, j.next, nch, 0);
    p.join[at] = j;
  }
  if (tid == 0) {
    p.hdr->n_units = ranged ? n_ranges : (int)N;
    p.hdr->ranged = ranged;
    p.hdr->counter = 0;
    p.hdr->n_items = NI;
    p.hdr->n_join = n_join;
    p.hdr->any_bad = s_bad;
    if (s_bad) atomicOr(p.dev_status, SPX_DEV_BAD_LEN);
  }
}

// Joins the parts of the entries that cuts opened (see combine_kernel) and voids the rows of requests with a bad length or page id.
// Blocks (b, y): entry b of the list, items (row, four columns) y * 256 + t of it.
template <typename T>
__global__ void __launch_bounds__(256) prompt_join_kernel(PromptParams p) {
  SPX_TL_SCOPE(kTlCombine);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  T *out = reinterpret_cast<T *>(p.out);
  const int vecs = p.D / 4;
  const int n_join = p.hdr->n_join, any_bad = p.hdr->any_bad;
  for (int li = blockIdx.x; li < n_join; li += gridDim.x) {
    const PromptJoin e = p.join[li];
    if (p.unit_bad[e.unit]) continue;
    for (int item = blockIdx.y * blockDim.x + threadIdx.x; item < e.rows * vecs; item += gridDim.y * blockDim.x) {
      const int row = item / vecs, dv = item % vecs;
      float mstar = -INFINITY, lstar = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      auto slot_row = [&](int c) -> int64_t { return (int64_t)(c == 0 ? e.first : e.next + 2 * (c - 1)) * p.unit_rows + row; };
      for (int c0 = 0; c0 < e.nch; c0 += 4) {
        // four chunks' loads in flight at a time, their maximum taken first
        float2 ml[4];
        float4 o[4];
        float top = mstar;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int64_t at = slot_row(min(c0 + u, e.nch - 1));
          ml[u] = p.part_ml[at];
          o[u] = *reinterpret_cast<const float4 *>(p.part_o + at * p.D + dv * 4);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (c0 + u < e.nch) top = fmaxf(top, ml[u].x);
        if (mstar != -INFINITY && top > mstar) {
          const float w = fast_exp2(mstar - top);
          lstar = rescaled_sum(lstar, mstar - top);
          acc.x *= w; acc.y *= w; acc.z *= w; acc.w *= w;
        }
        mstar = top;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (c0 + u >= e.nch || (ml[u].x == -INFINITY && ml[u].y == 0.f)) continue;   // (saw nothing)
          const float d = ml[u].x == -INFINITY ? 0.f : ml[u].x - mstar, w = fast_exp2(d);
          lstar += rescaled_sum(ml[u].y, d);
          acc.x += w * o[u].x; acc.y += w * o[u].y; acc.z += w * o[u].z; acc.w += w * o[u].w;
        }
      }
      const int pr = e.row0 + row, h = e.g * p.G + pr % p.G;
      const int64_t qrow = e.q0 + pr / p.G, at = (qrow * p.Hq + h) * p.D + dv * 4;
      const float inv = 1.f / lstar;
      st_from_float(out, at + 0, acc.x * inv);
      st_from_float(out, at + 1, acc.y * inv);
      st_from_float(out, at + 2, acc.z * inv);
      st_from_float(out, at + 3, acc.w * inv);
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
template <typename T>
__global__ void __launch_bounds__(256) prefix_join_kernel(AttnParams a, PromptParams p) {
  SPX_TL_SCOPE(kTlCombine);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int r = blockIdx.x;
  T *out = reinterpret_cast<T *>(a.out);
  const int vecs = a.D / 4, G = a.G;
  const int q0 = a.q_indptr[r];
  int m = a.q_indptr[r + 1] - q0;
  if (m < 0) m = 0;
  if (m > a.max_q_len) m = a.max_q_len;
  if (q0 < 0 || (int64_t)q0 + m > a.total_q) return;
  const int u = p.req_group[r];
  const int tiles = u >= 0 ? p.group_tiles[u] : 0;
  bool bad = a.req_bad[r] || p.req_flag[r] || (u >= 0 && p.unit_bad[u]);
  int64_t row0 = 0;    // the request's first packed row among its group's
  if (tiles > 0) {
    row0 = (int64_t)(q0 - p.q_indptr[max(p.group_indptr[u], 0)]) * G;
    const int64_t rows = (int64_t)(p.unit_item0[u + 1] - p.unit_item0[u]) * p.unit_rows;
    bad = bad || row0 < 0 || row0 + (int64_t)m * G > rows;
  }
  for (int item = blockIdx.y * blockDim.x + threadIdx.x; item < m * a.Hq * vecs; item += gridDim.y * blockDim.x) {
    const int dv = item % vecs, jh = item / vecs, h = jh % a.Hq, j = jh / a.Hq, g = h / G, hg = h % G;
    const int64_t qh = (int64_t)(q0 + j) * a.Hq + h, at = qh * a.D + dv * 4;
    const int nch = a.pair_nchunks[r * a.Hkv + g], base = a.pair_part_base[r * a.Hkv + g];
    if (bad || nch == 0) {
      for (int i = 0; i < 4; ++i) st_from_float(out, at + i, 0.f);
      if (dv == 0 && a.lse) a.lse[qh] = __int_as_float(0x7fc00000);
      continue;
    }
    int4 part = make_int4(0, 0, 0, 0);
    int64_t prow = 0;
    if (tiles > 0) {
      const int64_t row = row0 + (int64_t)j * G + hg;
      part = p.entry_part[(p.unit_item0[u] + row / p.unit_rows) * p.Hkv + g];
      prow = row % p.unit_rows;
    }
    float mstar = -INFINITY, lstar = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const int n = nch + part.z;
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
          const int64_t s = (int64_t)(c == 0 ? part.x : part.y + 2 * (c - 1)) * p.unit_rows + prow;
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
    st_from_float(out, at + 0, acc.x * inv);
    st_from_float(out, at + 1, acc.y * inv);
    st_from_float(out, at + 2, acc.z * inv);
    st_from_float(out, at + 3, acc.w * inv);
    if (dv == 0 && a.lse) a.lse[qh] = (mstar + log2f(lstar)) * kLn2;
  }
}

}  // namespace spx
