// Append to a paged cache of 8-bit floats with one scale per block of tokens and kv head, with the
// position rotation applied on the way.
//
// The scale blocks that receive a new row are quantised anew, the older tokens of the request in
// them included: amax over the block's values, scale = 2^e with the smallest e for which
// amax <= 448 * 2^e, code = round(value / scale).  A power of two divides exactly, so an older
// token's change of scale rounds only where its last bits fall below the smallest subnormal, and
// appending the same rows again changes nothing.
#pragma once
#include "common.cuh"

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
};

// 8 elements of a row as floats
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float (&x)[8]) {
  const uint4 v = *reinterpret_cast<const uint4 *>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
  const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
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
// 8 codes as floats, and back (values within the format's range, or not finite: NaN)
__device__ __forceinline__ void decode8(uint2 c, float (&x)[8]) {
  const uint32_t w[2] = {c.x, c.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    x[2 * i] = f.x; x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint2 encode8(const float (&x)[8]) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(x[2 * i], x[2 * i + 1]), __NV_NOSAT, __NV_E4M3) << (16 * (i & 1));
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint32_t finite_amax8(const float (&x)[8], uint32_t m) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
    m = b < 0x7f800000u && b > m ? b : m;
  }
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
__global__ void __launch_bounds__(kQuantThreads) kv_append_e4m3_kernel(const __grid_constant__ KvQuantParams p) {
  using S = QuantShape<D>;
  constexpr int kVecs = S::kVecs;
  extern __shared__ __align__(16) unsigned char quant_smem[];
  double2 *s_cs = reinterpret_cast<double2 *>(quant_smem);   // [tile tokens][8][kVecs] (cos, sin) of the new tokens
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
  // a request with a bad page among its new positions is skipped as a whole: every one of its tiles
  // looks at all of these pages
  int bad = 0;
  for (int i = (t_new >> p.log2P) + tid; i <= (L - 1) >> p.log2P; i += kQuantThreads) {
    const int page = table[i];
    bad |= page < 0 || page >= p.num_pages;
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) atomicOr(p.dev_status, SPX_DEV_BAD_PAGE);
    return;
  }

  const int slots = kQuantWarps / p.task_warps;                  // tasks the block works on at a time
  const int wsub = warp & (p.task_warps - 1);
  const int first_task = blockIdx.y * slots + warp / p.task_warps, task_step = gridDim.y * slots;
  const int n_kv = 2 * p.Hkv, n_tasks = n_kv + (p.q_in ? p.Hq : 0);
  if (p.rope) {
    const int n = min(tile_tokens, L - t0);
    for (int i = tid; i < n * (D / 2); i += kQuantThreads) {
      const int tok = i / (D / 2), pair = i % (D / 2);
      const int t = t0 + tok;
      if (t < t_new) continue;
      double2 cs;
      sincos((double)t * p.inv_freq[pair], &cs.y, &cs.x);
      s_cs[(tok * 8 + (pair & 7)) * kVecs + (pair >> 3)] = cs;
    }
    __syncthreads();
  }

  const int t_block = (t_new >> p.log2SB) << p.log2SB;            // first token of the first touched block
  const int tok0 = (wsub * kQuantItems * 32 + lane) / kVecs, vec = lane % kVecs;
  int page[kQuantItems];
#pragma unroll
  for (int k = 0; k < kQuantItems; ++k) {
    const int t = t0 + tok0 + k * (32 / kVecs);
    page[k] = t >= t_block && t < L ? table[t >> p.log2P] : -1;
  }
  int parity = 0;
  for (int task = first_task; task < n_tasks; task += task_step, parity ^= 1) {
    const bool is_q = task >= n_kv, is_v = !is_q && (task & 1);
    const int head = is_q ? task - n_kv : task >> 1;
    const int heads = is_q ? p.Hq : p.Hkv;
    const T *src = reinterpret_cast<const T *>(is_q ? p.q_in : is_v ? p.new_v : p.new_k) + head * D + vec * 8;
    unsigned char *cache = (is_v ? p.v_cache : p.k_cache) + head * p.stride_head + vec * 8;
    float *scales = is_v ? p.v_scales : p.k_scales;
    float lo[kQuantItems][8], hi[kQuantItems][8];
    uint32_t amax[kQuantItems];
    float old_scale[kQuantItems];
#pragma unroll
    for (int k = 0; k < kQuantItems; ++k) {
      const int tok = tok0 + k * (32 / kVecs), t = t0 + tok;
      amax[k] = 0;
      old_scale[k] = 0.f;
      if (t >= L || t < t_block) continue;
      if (t >= t_new) {
        const T *row = src + (int64_t)(q0 + t - t_new) * heads * D;
        load8(row, lo[k]);
        load8(row + D / 2, hi[k]);
        if (p.rope && !is_v) {
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const double2 cs = s_cs[(tok * 8 + u) * kVecs + vec];
            const double x0 = lo[k][u], x1 = hi[k][u];
            lo[k][u] = __double2float_rn(x0 * cs.x - x1 * cs.y);
            hi[k][u] = __double2float_rn(x1 * cs.x + x0 * cs.y);
          }
        }
        if (is_q) {
          T *dst = reinterpret_cast<T *>(p.q_out) + (int64_t)(q0 + t - t_new) * heads * D + head * D + vec * 8;
          store8(dst, lo[k]);
          store8(dst + D / 2, hi[k]);
        }
      } else if (!is_q) {
        const unsigned char *at = cache + (int64_t)page[k] * p.stride_page + (int64_t)(t & ((1 << p.log2P) - 1)) * p.stride_token;
        const float sc = scales[(((int64_t)page[k] * p.Hkv + head) << (p.log2P - p.log2SB)) + ((t & ((1 << p.log2P) - 1)) >> p.log2SB)];
        decode8(*reinterpret_cast<const uint2 *>(at), lo[k]);
        decode8(*reinterpret_cast<const uint2 *>(at + D / 2), hi[k]);
#pragma unroll
        for (int u = 0; u < 8; ++u) { lo[k][u] *= sc; hi[k][u] *= sc; }
        old_scale[k] = sc;
      }
      amax[k] = finite_amax8(hi[k], finite_amax8(lo[k], 0));
    }
    if (is_q) continue;   // no exchange between the warps of a query task
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
      const int t = t0 + tok0 + k * (32 / kVecs);
      if (t >= L || t < t_block) continue;
      const uint32_t e = scale_exponent(amax[k]);
      const float scale = __uint_as_float(e << 23), inv = __uint_as_float((254 - e) << 23);   // 2^127 / 2^-126 at most: both normal
      const int slot = t & ((1 << p.log2P) - 1);
      if (vec == 0 && (t & ((1 << p.log2SB) - 1)) == 0)
        scales[(((int64_t)page[k] * p.Hkv + head) << (p.log2P - p.log2SB)) + (slot >> p.log2SB)] = scale;
      if (t < t_new && scale == old_scale[k]) continue;
#pragma unroll
      for (int u = 0; u < 8; ++u) { lo[k][u] *= inv; hi[k][u] *= inv; }
      unsigned char *at = cache + (int64_t)page[k] * p.stride_page + (int64_t)slot * p.stride_token;
      *reinterpret_cast<uint2 *>(at) = encode8(lo[k]);
      *reinterpret_cast<uint2 *>(at + D / 2) = encode8(hi[k]);
    }
  }
}

}  // namespace spx
