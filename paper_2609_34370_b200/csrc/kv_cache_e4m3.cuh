// Append to a paged cache of 8-bit floats with one scale per block of tokens and kv head, with the
// position rotation applied on the way.
//
// The scale blocks that receive a new row are quantised anew, the older tokens of the request in
// them included: amax over the block's values, scale = 2^e with the smallest e for which
// amax <= 448 * 2^e, code = round(value / scale).  A power of two divides exactly, so an older
// token's change of scale rounds only where its last bits fall below the smallest subnormal, and
// appending the same rows again changes nothing.
//
// A prompt has to read its rows and write half as many bytes and the rotated queries: 14.6k rows of the Llama-3-8B layer
// shape are 329 MB, 51 us at HBM's rate.  They take 104, bound by latency: the 16 warps
// of an SM (two blocks, for their registers and the angles in shared memory) alternate between a task's rows and the
// dependent arithmetic on them, the compensated rotation above all (float64 angles t f, off by 2^-53 of themselves, that is
// 2^-40 at position 8191; products kept to 2^-46: a stored code is that of float64 arithmetic); 44% of the issue slots and
// 33% of DRAM's peak are used.  Rows fetched a task ahead, whole (157 us) or item by item into the registers just read
// (119), were slower.  Every block of a tile looks at all page ids of its request's new positions; that does not show up to
// 131,072 rows (6.2 to 6.5 ns a row with pages of 16 and 32 tokens, like a prompt of 2048).
#pragma once
#include <type_traits>

#include "attn_e4m3.cuh"   // e8::pair and the packed fp32 arithmetic
#include "common.cuh"
#include "rotate.cuh"

namespace spx {

constexpr int kQuantThreads = 256;
constexpr int kQuantWarps = kQuantThreads / 32;
constexpr int kQuantItems = 4;   // 16-element items a lane holds: a warp covers 4 * 32 * 16 elements of one head

// A warp covers kWarpTokens consecutive tokens of one head (16 of 128 columns, 32 of 64); a tile is
// the tokens a task's warps cover, at least one scale block, aligned to its own size.
template <int D>
struct QuantShape {
  static constexpr int kVecs = D / 16;                          // items of a token: 8 columns of each half
  static constexpr int kWarpTokens = kQuantItems * 32 / kVecs;
  __host__ __device__ static int task_warps(int scale_block) { return scale_block > kWarpTokens ? scale_block / kWarpTokens : 1; }
};

struct KvQuantParams {
  int32_t batch, total_q, Hkv, Hq, log2P, log2SB, num_pages, max_pages_per_req;
  int32_t task_warps;      // warps of a task: tile = task_warps * kWarpTokens tokens
  int32_t log2_tile;
  const void *new_k, *new_v, *q_in;   // q_in NULL: no query rows
  void *q_out;
  unsigned char *k_cache, *v_cache;
  int64_t stride_page, stride_head, stride_token;   // bytes
  float *k_scales, *v_scales;
  const int32_t *block_table, *seq_lens, *q_indptr;
  int32_t *dev_status;
  int32_t rope;
  double inv_freq[64];     // base^(-2i/D)
  // positions of several axes (axes = 0: a row's position is its place in the request)
  int32_t axes;
  const int32_t *positions;
  int64_t position_stride;
  unsigned char axis_of[64];
};

// Eight elements of a row as they are stored, and as floats.  (Plain loads: query rows may be rotated in place, so they are
// not read-only for the kernel's life, which the non-coherent load promises.)
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
  uint4 a;
  __device__ void set_codes(uint2 lo, uint2 hi) { a = make_uint4(lo.x, lo.y, hi.x, hi.y); }
  __device__ void codes(uint2 &lo, uint2 &hi) const { lo = make_uint2(a.x, a.y); hi = make_uint2(a.z, a.w); }
  __device__ void load(const __nv_bfloat16 *p) { a = *reinterpret_cast<const uint4 *>(p); }
  __device__ void values(float (&x)[8]) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ void set_codes(uint2 lo, uint2 hi) { a = make_float4(__uint_as_float(lo.x), __uint_as_float(lo.y), __uint_as_float(hi.x), __uint_as_float(hi.y)); }
  __device__ void codes(uint2 &lo, uint2 &hi) const {
    lo = make_uint2(__float_as_uint(a.x), __float_as_uint(a.y));
    hi = make_uint2(__float_as_uint(a.z), __float_as_uint(a.w));
  }
  __device__ void load(const float *p) { a = *reinterpret_cast<const float4 *>(p); b = *(reinterpret_cast<const float4 *>(p) + 1); }
  __device__ void values(float (&x)[8]) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
};
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t *>(&b);
  }
  *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
  *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void decode8(uint2 c, float (&x)[8]) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    x[2 * i] = f.x; x[2 * i + 1] = f.y;
  }
}
// (the conversion saturates: no value passes 448 but an infinity, which the caller has made a NaN)
__device__ __forceinline__ uint2 encode8(const float (&x)[8]) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    uint16_t a, b;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(a) : "f"(x[4 * i + 1]), "f"(x[4 * i]));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(b) : "f"(x[4 * i + 3]), "f"(x[4 * i + 2]));
    w[i] = (uint32_t)a | ((uint32_t)b << 16);
  }
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ float amax8(const float (&x)[8], float m) {   // NaNs do not count
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
  return m;
}

// The exponent field of 2^e with the smallest e for which amax <= 448 * 2^e = 1.75 * 2^(e+8); amax as
// its bit pattern.  Subnormal values count as the smallest exponent: their scale is 2^-126 anyway.
__device__ __forceinline__ uint32_t scale_exponent(uint32_t amax_bits) {
  if (amax_bits == 0) return 127;
  const int e = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 1);
}

// grid = (tiles, splits of the tasks), block = 256.  A task is one kv head's K or V rows of a tile,
// or one query head's rows; a block's warps take its tasks in turn.  Tile u belongs to the request r
// with base(r) <= u < base(r + 1), base(r) = q_indptr[r] / tile + 2 r: m rows overlap at most
// m / tile + 2 aligned tiles, so no prefix sums over the lengths are needed; tiles past a request's
// last one leave at once.
template <typename T, int D>
__global__ void __launch_bounds__(kQuantThreads, 2) kv_append_e4m3_kernel(const __grid_constant__ KvQuantParams p) {
  using S = QuantShape<D>;
  constexpr int kVecs = S::kVecs, kStep = 32 / kVecs;   // tokens between a lane's items
  extern __shared__ __align__(16) unsigned char quant_smem[];
  // (ch, ch', cl, cl'), (sh, sh', sl, sl') of two neighbouring pairs: [tile tokens][4][2][kVecs] of 16 bytes
  float *s_cs = reinterpret_cast<float *>(quant_smem);
  __shared__ uint32_t s_amax[2][kQuantWarps];
  __shared__ int s_req;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int tile_tokens = 1 << p.log2_tile;

  // the request of this tile: 32 probes at a time
  if (warp == 0) {
    int lo = 0, hi = p.batch;   // base(lo) <= u, hi past the last candidate
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32;
      const int c = lo + lane * step;
      const bool below = c < hi && (int64_t)(p.q_indptr[c] >> p.log2_tile) + 2 * (int64_t)c <= (int64_t)blockIdx.x;
      const int n = __popc(__ballot_sync(0xffffffffu, below || lane == 0));   // the probes ascend
      const int nlo = lo + (n - 1) * step;
      hi = min(hi, nlo + step);
      lo = nlo;
    }
    if (lane == 0) s_req = lo;
  }
  __syncthreads();
  const int r = s_req;
  const int q0 = p.q_indptr[r];
  const int m = p.q_indptr[r + 1] - q0;
  const int L = p.seq_lens[r];
  const int64_t i_tile = (int64_t)blockIdx.x - ((q0 >> p.log2_tile) + 2 * (int64_t)r);
  const bool ok_len = m >= 1 && L >= m && q0 >= 0 && m <= p.total_q - q0 &&
                      (((int64_t)L + (1 << p.log2P) - 1) >> p.log2P) <= (int64_t)p.max_pages_per_req;
  if (!ok_len) {
    if (tid == 0) atomicOr(p.dev_status, SPX_DEV_BAD_LEN);
    return;
  }
  const int t_new = L - m;                                      // first new position
  const int64_t tile64 = (int64_t)(t_new >> p.log2_tile) + i_tile;
  if (i_tile < 0 || tile64 > ((L - 1) >> p.log2_tile)) return;
  const int t0 = (int)tile64 << p.log2_tile;
  const int32_t *table = p.block_table + (int64_t)r * p.max_pages_per_req;

  const int slots = kQuantWarps / p.task_warps;                  // tasks the block works on at a time
  const int wsub = warp & (p.task_warps - 1);
  const int first_task = blockIdx.y * slots + warp / p.task_warps, task_step = gridDim.y * slots;
  const int n_kv = 2 * p.Hkv, n_tasks = n_kv + (p.q_in ? p.Hq : 0);
  const int t_block = (t_new >> p.log2SB) << p.log2SB;            // first token of the first touched block
  const int tok0 = (wsub * kQuantItems * 32 + lane) / kVecs, vec = lane % kVecs;
  int page[kQuantItems];
#pragma unroll
  for (int k = 0; k < kQuantItems; ++k) {
    const int t = t0 + tok0 + k * kStep;
    page[k] = t >= t_block && t < L ? table[t >> p.log2P] : -1;
  }
  // a lane's new rows of a task, fetched before anything else is waited for
  struct Rows { Raw8<T> lo[kQuantItems], hi[kQuantItems]; } rows;
  auto fetch = [&](int task) {
    const bool is_q = task >= n_kv, is_v = !is_q && (task & 1);
    const int head = is_q ? task - n_kv : task >> 1, heads = is_q ? p.Hq : p.Hkv;
    const T *src = reinterpret_cast<const T *>(is_q ? p.q_in : is_v ? p.new_v : p.new_k) + head * D + vec * 8;
#pragma unroll
    for (int k = 0; k < kQuantItems; ++k) {
      const int t = t0 + tok0 + k * kStep;
      if (t >= t_new && t < L) {
        const T *row = src + (int64_t)(q0 + t - t_new) * heads * D;
        rows.lo[k].load(row);
        rows.hi[k].load(row + D / 2);
      }
    }
  };
  if (first_task < n_tasks) fetch(first_task);
  // a request with a bad page among its new positions is skipped as a whole: every one of its tiles
  // looks at all of these pages
  int bad = 0;
  for (int i = (t_new >> p.log2P) + tid; i <= (L - 1) >> p.log2P; i += kQuantThreads) {
    const int pg = table[i];
    bad |= pg < 0 || pg >= p.num_pages;
  }
  // (ch, cl) and (sh, sl) of a token's pair
  auto angle_at = [&](int tok, int pair) -> float * {
    return s_cs + ((((tok * 4 + ((pair & 7) >> 1)) * 2) * kVecs + (pair >> 3)) << 2) + (pair & 1);
  };
  auto keep = [&](float *at, double c, double sn) {
    const float ch = (float)c, sh = (float)sn;
    at[0] = ch; at[2] = (float)(c - (double)ch);
    at[4 * kVecs] = sh; at[4 * kVecs + 2] = (float)(sn - (double)sh);
  };
  if (p.rope && p.axes) {
    // positions of several axes: as below, where a token's position is that of the one before or the next (an axis of a grid
    // stands still or counts up for most tokens), by a sine and cosine of its own elsewhere
    const int t_lo = max(t0, t_new), n = min(t0 + tile_tokens, L) - t_lo;   // the tile's new tokens
    for (int i = tid; i < (n + 3) / 4 * (D / 2); i += kQuantThreads) {
      const int pair = i % (D / 2), tok = t_lo - t0 + i / (D / 2) * 4;
      const int32_t *at_pos = p.positions + (int64_t)p.axis_of[pair] * p.position_stride + q0 + (t0 + tok - t_new);
      const int left = t_lo - t0 + n - tok;
      int pos[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) pos[u] = u < left ? at_pos[u] : 0;
      const double f = p.inv_freq[pair];
      double c, sn, cf = 1.0, sf = 0.0;
      sincos((double)pos[0] * f, &sn, &c);
      bool turning = false;
#pragma unroll
      for (int u = 1; u < 4; ++u) turning |= u < left && pos[u] == pos[u - 1] + 1ll;
      if (turning) sincos(f, &sf, &cf);
      keep(angle_at(tok, pair), c, sn);
#pragma unroll
      for (int u = 1; u < 4; ++u) {
        if (u >= left) break;
        if (pos[u] == pos[u - 1] + 1ll) {
          const double c2 = c * cf - sn * sf;
          sn = sn * cf + c * sf;
          c = c2;
        } else if (pos[u] != pos[u - 1]) {
          sincos((double)pos[u] * f, &sn, &c);
        }
        keep(angle_at(tok + u, pair), c, sn);
      }
    }
  } else if (p.rope) {
    // angles in float64; a thread takes four tokens of a pair: one sine and cosine, and three turns by the pair's
    // frequency (each adds 2^-52)
    const int t_lo = max(t0, t_new), n = min(t0 + tile_tokens, L) - t_lo;   // the tile's new tokens
    for (int i = tid; i < (n + 3) / 4 * (D / 2); i += kQuantThreads) {
      const int pair = i % (D / 2), tok = t_lo - t0 + i / (D / 2) * 4;
      const double f = p.inv_freq[pair];
      double c, sn, cf, sf;
      sincos((double)(t0 + tok) * f, &sn, &c);
      sincos(f, &sf, &cf);
      float *at = angle_at(tok, pair);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (tok + u < t_lo - t0 + n) keep(at, c, sn);
        at += 4 * 2 * kVecs * 4;
        const double c2 = c * cf - sn * sf;
        sn = sn * cf + c * sf;
        c = c2;
      }
    }
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) atomicOr(p.dev_status, SPX_DEV_BAD_PAGE);
    return;
  }

  auto turn = [&](int tok, float (&lo)[8], float (&hi)[8], auto exact) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const ulonglong2 *at = reinterpret_cast<const ulonglong2 *>(s_cs) + (tok * 4 + u) * 2 * kVecs + vec;
      const ulonglong2 a = at[0], b = at[kVecs];
      const CosSin cs{a.x, a.y, b.x, b.y};
      uint64_t y0, y1;
      rotate2<decltype(exact)::value>(e8::pair(lo[2 * u], lo[2 * u + 1]), e8::pair(hi[2 * u], hi[2 * u + 1]), cs, y0, y1);
      e8::unpair(y0, lo[2 * u], lo[2 * u + 1]);
      e8::unpair(y1, hi[2 * u], hi[2 * u + 1]);
    }
  };
  int parity = 0;
  for (int task = first_task; task < n_tasks; task += task_step, parity ^= 1) {
    if (task != first_task) fetch(task);
    if (task >= n_kv) {
      // ---- query rows
      const int head = task - n_kv;
#pragma unroll
      for (int k = 0; k < kQuantItems; ++k) {
        const int tok = tok0 + k * kStep, t = t0 + tok;
        if (t < t_new || t >= L) continue;
        float lo[8], hi[8];
        rows.lo[k].values(lo);
        rows.hi[k].values(hi);
        turn(tok, lo, hi, std::integral_constant<bool, sizeof(T) == 4>());
        T *dst = reinterpret_cast<T *>(p.q_out) + ((int64_t)(q0 + t - t_new) * p.Hq + head) * D + vec * 8;
        store8(dst, lo);
        store8(dst + D / 2, hi);
      }
      continue;
    }
    // ---- K or V rows
    const bool is_v = task & 1;
    const int head = task >> 1;
    unsigned char *cache = (is_v ? p.v_cache : p.k_cache) + head * p.stride_head + vec * 8;
    float *scales = is_v ? p.v_scales : p.k_scales;
    auto scale_at = [&](int k, int t) -> float * {
      return scales + ((((int64_t)page[k] * p.Hkv + head) << (p.log2P - p.log2SB)) + ((t & ((1 << p.log2P) - 1)) >> p.log2SB));
    };
    auto cache_at = [&](int k, int t) -> unsigned char * {
      return cache + (int64_t)page[k] * p.stride_page + (int64_t)(t & ((1 << p.log2P) - 1)) * p.stride_token;
    };
    // Two passes over the rows as they were fetched, 16 elements at a time: the maxima, then the codes.  (Keeping the
    // rotated values of the first pass takes 64 registers more and spills; three blocks per SM, 80 registers, do too:
    // 142 us for 14.6k rows.)
    uint32_t amax[kQuantItems];
    float old_scale[kQuantItems];
    auto values = [&](int k, float (&lo)[8], float (&hi)[8]) {
      const int tok = tok0 + k * kStep, t = t0 + tok;
      if (t >= t_new) {
        rows.lo[k].values(lo);
        rows.hi[k].values(hi);
        if (p.rope && !is_v) turn(tok, lo, hi, std::true_type());
      } else {
        uint2 c_lo, c_hi;
        rows.lo[k].codes(c_lo, c_hi);
        decode8(c_lo, lo);
        decode8(c_hi, hi);
#pragma unroll
        for (int u = 0; u < 8; ++u) { lo[u] *= old_scale[k]; hi[u] *= old_scale[k]; }
      }
    };
#pragma unroll
    for (int k = 0; k < kQuantItems; ++k) {
      const int t = t0 + tok0 + k * kStep;
      old_scale[k] = 0.f;
      if (t < t_new && t >= t_block) {
        const unsigned char *at = cache_at(k, t);
        rows.lo[k].set_codes(*reinterpret_cast<const uint2 *>(at), *reinterpret_cast<const uint2 *>(at + D / 2));
        old_scale[k] = *scale_at(k, t);
      }
    }
    bool infinite = false;
#pragma unroll
    for (int k = 0; k < kQuantItems; ++k) {
      const int t = t0 + tok0 + k * kStep;
      amax[k] = 0;
      if (t >= L || t < t_block) continue;
      float lo[8], hi[8];
      values(k, lo, hi);
      float a = amax8(hi, amax8(lo, 0.f));
      if (a == INFINITY) {   // infinities do not count
        infinite = true;
        a = 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          if (fabsf(lo[u]) < INFINITY) a = fmaxf(a, fabsf(lo[u]));
          if (fabsf(hi[u]) < INFINITY) a = fmaxf(a, fabsf(hi[u]));
        }
      }
      amax[k] = __float_as_uint(a);
    }
    // amax of the scale block of each item: over the lanes, the items and the warps that share it
    const int share = kVecs << p.log2SB;   // items of a block
    for (int o = 1; o < min(32, share); o <<= 1)
#pragma unroll
      for (int k = 0; k < kQuantItems; ++k) amax[k] = max(amax[k], __shfl_xor_sync(0xffffffffu, amax[k], o));
    if (share >= 64) {
      amax[0] = amax[1] = max(amax[0], amax[1]);
      amax[2] = amax[3] = max(amax[2], amax[3]);
    }
    if (share >= 128) amax[0] = amax[1] = amax[2] = amax[3] = max(amax[0], amax[2]);
    if (p.task_warps > 1) {
      // the block is the tile: the task's warps exchange their maxima (two buffers in turn)
      if (lane == 0) s_amax[parity][warp] = amax[0];
      asm volatile("bar.sync %0, %1;" ::"r"(1 + warp / p.task_warps), "r"(p.task_warps * 32) : "memory");
      uint32_t a = 0;
      for (int w = 0; w < p.task_warps; ++w) a = max(a, s_amax[parity][warp / p.task_warps * p.task_warps + w]);
#pragma unroll
      for (int k = 0; k < kQuantItems; ++k) amax[k] = a;
    }
#pragma unroll
    for (int k = 0; k < kQuantItems; ++k) {
      const int t = t0 + tok0 + k * kStep;
      if (t >= L || t < t_block) continue;
      const uint32_t e = scale_exponent(amax[k]);
      const float scale = __uint_as_float(e << 23), inv = __uint_as_float((254 - e) << 23);   // 2^127 / 2^-126 at most: both normal
      if (vec == 0 && (t & ((1 << p.log2SB) - 1)) == 0) *scale_at(k, t) = scale;
      if (t < t_new && scale == old_scale[k]) continue;
      float lo[8], hi[8];
      values(k, lo, hi);
#pragma unroll
      for (int u = 0; u < 8; ++u) { lo[u] *= inv; hi[u] *= inv; }
      if (infinite) {   // and become NaN
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          if (fabsf(lo[u]) == INFINITY) lo[u] = __int_as_float(0x7fc00000);
          if (fabsf(hi[u]) == INFINITY) hi[u] = __int_as_float(0x7fc00000);
        }
      }
      unsigned char *at = cache_at(k, t);
      *reinterpret_cast<uint2 *>(at) = encode8(lo);
      *reinterpret_cast<uint2 *>(at + D / 2) = encode8(hi);
    }
  }
}

}  // namespace spx
