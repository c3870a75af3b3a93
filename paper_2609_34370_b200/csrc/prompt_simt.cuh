// Attention of many query rows in fp32 FMA arithmetic: fp32 rows over any pool (tensor-core tf32 would round the operands to
// 10-bit mantissas), and 16-bit rows over pages of fewer than 8 tokens, which no swizzle atom of a TMA copy fits.
//
// An item is 64 packed rows of one kv head; a step takes 64 tokens.  Threads hold 8 rows x 4 tokens of the scores and 8 rows x
// D / 16 columns of the output, so that 24 shared-memory wavefronts feed 128 (256) FMAs of a warp.  The running maximum and
// sum of a row live in the 16 lanes that share it; weights go through shared memory once.  113 KB and 128 threads a block:
// two blocks per SM, one of which computes while the other loads (8-bit pools, heads of 128, six prompts up to 1200 tokens: 354 us,
// 474 with one).  Two prompts of 8192
// tokens in bf16 take 33.8 ms here (32 of the 74 TFLOP/s that FMAs alone would allow); a 128-token piece of fp32 rows is a latency chain of 27 us.
#pragma once
#include "common.cuh"
#include "prompt_plan.cuh"

namespace spx {

constexpr int kPsThreads = 128;
constexpr int kPsRows = 64, kPsTokens = 64;
template <int D> constexpr int kPsSmem = (kPsRows * D + 2 * kPsTokens * D + kPsRows * kPsTokens) * 4;
// What a block holds beside its tiles.  (The scales of 8-bit pools' tokens lie where the weights are to come: with 512 bytes more a second
// block would not fit.)
struct PsShared {
  int64_t at[kPsTokens];     // element offset of a token's row in the pool, -1: none
  int unit, infinite;
};
static_assert(2 * (kPsSmem<128> + sizeof(PsShared) + 1024) <= 228 * 1024, "two blocks per SM, and 1 KB of the system's for each");

// 16-byte vectors of a row of D floats, spread so that eight rows' vectors of one column lie in eight different banks
template <int D>
__device__ __forceinline__ float4 *ps_vec(float *tile, int row, int vec) { return reinterpret_cast<float4 *>(tile) + row * (D / 4) + (vec ^ (row & 7)); }

template <typename Q> struct PsLoad;   // four elements of a row of type Q
template <> struct PsLoad<float> { static __device__ float4 get(const float *p) { return *reinterpret_cast<const float4 *>(p); } };
template <> struct PsLoad<__nv_bfloat16> {
  static __device__ float4 get(const __nv_bfloat16 *p) {
    const uint2 a = *reinterpret_cast<const uint2 *>(p);
    return make_float4(__uint_as_float(a.x << 16), __uint_as_float(a.x & 0xffff0000u), __uint_as_float(a.y << 16), __uint_as_float(a.y & 0xffff0000u));
  }
};
template <> struct PsLoad<unsigned char> {   // e4m3 codes
  static __device__ float4 get(const unsigned char *p) {
    const uint32_t a = *reinterpret_cast<const uint32_t *>(p);
    const float2 lo = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)a, __NV_E4M3)));
    const float2 hi = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(a >> 16), __NV_E4M3)));
    return make_float4(lo.x, lo.y, hi.x, hi.y);
  }
};

// T: rows and output; KV: pool elements (T, or unsigned char for 8-bit floats).
template <typename T, typename KV, int D>
__global__ void __launch_bounds__(kPsThreads) prompt_simt_kernel(PromptParams p) {
  SPX_TL_SCOPE(kTlAttention);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // (the kernel behind this one reads the plan ahead of its own wait)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ __align__(16) unsigned char smem_raw[];
  float *sQ = reinterpret_cast<float *>(smem_raw), *sK = sQ + kPsRows * D, *sV = sK + kPsTokens * D, *sP = sV + kPsTokens * D;
  __shared__ PsShared s;
  float *sScale = sP;                     // [K, V][token], until the weights are written
  constexpr bool kCodes = sizeof(KV) == 1;
  constexpr int kVecs = D / 4;
  constexpr int kCols = D / 64;           // output columns of a thread, in vectors
  const T *Q = reinterpret_cast<const T *>(p.q);
  const KV *Kc = reinterpret_cast<const KV *>(p.k_cache), *Vc = reinterpret_cast<const KV *>(p.v_cache);
  T *out = reinterpret_cast<T *>(p.out);
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int n_units = p.hdr->n_units;
  // where there is an SM for each unit, the SMs' second blocks leave them to the first (four prompts up to 200 tokens over 8-bit pools, heads
  // of 128: 52 us, 61 with both)
  if (n_units <= (int)gridDim.x / 2 && blockIdx.x >= gridDim.x / 2) return;

  for (;;) {
    __syncthreads();
    if (tid == 0) s.unit = atomicAdd(&p.hdr->counter, 1);
    __syncthreads();
    const int unit = s.unit;
    if (unit >= n_units) break;
    {
      const PromptEntry e = p.entries[unit / p.Hkv];
      const int g = unit % p.Hkv;
      const int slot = e.slot < 0 ? -1 : e.slot + g;
      const int32_t *table = p.block_table + (int64_t)e.table_row * p.max_pages_per_req;
      const int t_begin = e.tile_begin * kTileTokens, t_end = min(e.t_end, e.tile_end * kTileTokens);
      const bool causal = p.groups == 0;
      // what the thread's rows see: tokens up to limit[i]
      int limit[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int row = e.row0 + ty * 8 + i;
        limit[i] = ty * 8 + i >= e.rows ? -1 : causal ? e.vis0 + row / p.G : e.vis0;
      }
      const int whole = causal ? e.vis0 + e.row0 / p.G : e.vis0;   // every row sees the tokens up to here
      __syncthreads();   // the previous entry's rows are read
#pragma unroll 8
      for (int i = tid; i < kPsRows * kVecs; i += kPsThreads) {
        const int row = i / kVecs, v = i % kVecs, pr = e.row0 + row;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < e.rows) x = PsLoad<T>::get(Q + ((int64_t)(e.q0 + pr / p.G) * p.Hq + g * p.G + pr % p.G) * D + v * 4);
        x.x *= p.scale_log2; x.y *= p.scale_log2; x.z *= p.scale_log2; x.w *= p.scale_log2;
        *ps_vec<D>(sQ, row, v) = x;
      }
      float m[8], l[8];
      float4 o[8][kCols];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        m[i] = -INFINITY; l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < kCols; ++c) o[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll 1
      for (int t0 = t_begin; t0 < t_end; t0 += kPsTokens) {
        __syncthreads();   // K, V and P of the previous step are read
        if (tid < kPsTokens) {
          const int t = t0 + tid;
          int64_t at = -1;
          if (t < t_end) {
            const int page = table[t >> p.log2P], in_page = t & (p.P - 1);
            if (page < 0 || page >= p.num_pages) {
              atomicOr(p.dev_status, SPX_DEV_BAD_PAGE);
              p.unit_bad[e.unit] = 1;
              p.hdr->any_bad = 1;
            } else {
              at = (int64_t)page * p.stride_page + (int64_t)g * p.stride_head + (int64_t)in_page * p.stride_token;
              if constexpr (kCodes) {
                const int64_t sc = (((int64_t)page * p.Hkv + g) << (p.log2P - p.log2SB)) + (in_page >> p.log2SB);
                sScale[tid] = p.k_scales[sc];
                sScale[kPsTokens + tid] = p.v_scales[sc];
              }
            }
          }
          s.at[tid] = at;
        }
        if (tid == 0) s.infinite = 0;
        __syncthreads();
        const bool edge = t0 + kPsTokens - 1 > whole;
        bool infinite = false;
        // (the loads of eight vectors of each are in flight together: four fp32 prompts up to 260 tokens 43 us, so 42)
#pragma unroll 8
        for (int i = tid; i < kPsTokens * kVecs; i += kPsThreads) {
          const int tok = i / kVecs, v = i % kVecs;
          const int64_t at = s.at[tok];
          float4 k = make_float4(0.f, 0.f, 0.f, 0.f), w = k;
          if (at >= 0) {
            k = PsLoad<KV>::get(Kc + at + v * 4);
            w = PsLoad<KV>::get(Vc + at + v * 4);
            if constexpr (kCodes) {
              const float a = sScale[tok], b = sScale[kPsTokens + tok];
              k.x *= a; k.y *= a; k.z *= a; k.w *= a;
              w.x *= b; w.y *= b; w.z *= b; w.w *= b;
            }
            if (edge) {   // 0 times it would be NaN in the rows that do not see the token
              const float z = fmaf(w.x, 0.f, fmaf(w.y, 0.f, fmaf(w.z, 0.f, w.w * 0.f)));
              infinite |= z != 0.f;
            }
          }
          *ps_vec<D>(sK, tok, v) = k;
          *ps_vec<D>(sV, tok, v) = w;
        }
        if (edge && infinite) s.infinite = 1;
        __syncthreads();
        // scores of rows ty * 8 + i, tokens tx + 16 j
        float x[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][j] = 0.f;
#pragma unroll 2
        for (int v = 0; v < kVecs; ++v) {
          float4 k[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) k[j] = *ps_vec<D>(sK, tx + 16 * j, v);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 a = *ps_vec<D>(sQ, ty * 8 + i, v);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              x[i][j] = fmaf(a.x, k[j].x, x[i][j]); x[i][j] = fmaf(a.y, k[j].y, x[i][j]);
              x[i][j] = fmaf(a.z, k[j].z, x[i][j]); x[i][j] = fmaf(a.w, k[j].w, x[i][j]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float top = -INFINITY;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int t = t0 + tx + 16 * j;
            if (edge && !(t < t_end && t <= limit[i])) x[i][j] = -INFINITY;
            top = fmaxf(top, x[i][j]);
          }
#pragma unroll
          for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
          const float m_new = fmaxf(m[i], top), ref = m_new == -INFINITY ? 0.f : m_new;
          const float alpha = m[i] == -INFINITY ? 1.f : fast_exp2(m[i] - m_new);   // (nothing summed yet: zeros)
          float sum = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float w = fast_exp2(x[i][j] - ref);
            sum += w;
            sP[(ty * 8 + i) * kPsTokens + tx + 16 * j] = w;
          }
          m[i] = m_new;
          l[i] = l[i] * alpha + sum;
#pragma unroll
          for (int c = 0; c < kCols; ++c) { o[i][c].x *= alpha; o[i][c].y *= alpha; o[i][c].z *= alpha; o[i][c].w *= alpha; }
        }
        __syncwarp();   // (a row's weights are written and read by one half warp)
        const bool guard = edge && s.infinite;
#pragma unroll 2
        for (int tv = 0; tv < kPsTokens / 4; ++tv) {
          float4 w[4][kCols];
#pragma unroll
          for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int c = 0; c < kCols; ++c) w[u][c] = *ps_vec<D>(sV, tv * 4 + u, tx + 16 * c);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 a = *(reinterpret_cast<const float4 *>(sP + (ty * 8 + i) * kPsTokens) + tv);
            const float b[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              if (guard && t0 + tv * 4 + u > limit[i]) continue;
#pragma unroll
              for (int c = 0; c < kCols; ++c) {
                o[i][c].x = fmaf(b[u], w[u][c].x, o[i][c].x); o[i][c].y = fmaf(b[u], w[u][c].y, o[i][c].y);
                o[i][c].z = fmaf(b[u], w[u][c].z, o[i][c].z); o[i][c].w = fmaf(b[u], w[u][c].w, o[i][c].w);
              }
            }
          }
        }
      }
      // the row's sum over its 16 lanes
#pragma unroll
      for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int d = 8; d > 0; d >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
        const int row = ty * 8 + i, pr = e.row0 + row;
        if (row >= e.rows) continue;
        if (slot < 0) {
          const float inv = 1.f / l[i];
          const int64_t qh = (int64_t)(e.q0 + pr / p.G) * p.Hq + g * p.G + pr % p.G;
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
            const int64_t at = qh * D + (tx + 16 * c) * 4;
            st_from_float(out, at + 0, o[i][c].x * inv); st_from_float(out, at + 1, o[i][c].y * inv);
            st_from_float(out, at + 2, o[i][c].z * inv); st_from_float(out, at + 3, o[i][c].w * inv);
          }
          if (tx == 0 && p.lse) p.lse[qh] = (m[i] + log2f(l[i])) * kLn2;
        } else {
          const int64_t at = (int64_t)slot * p.unit_rows + row;
#pragma unroll
          for (int c = 0; c < kCols; ++c) *reinterpret_cast<float4 *>(p.part_o + at * D + (tx + 16 * c) * 4) = o[i][c];
          if (tx == 0) p.part_ml[at] = make_float2(m[i], l[i]);
        }
      }
    }
  }
}

}  // namespace spx
