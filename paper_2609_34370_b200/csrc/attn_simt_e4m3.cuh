// Verify attention over 8-bit pools in fp32 arithmetic: fp32 queries, and pages of fewer than eight tokens.
//
// A block works on one entry of the plan in steps of 64 tokens.  K and V are dequantised (code * scale,
// one fp32 rounding) into shared memory, the codes of the next step on their way meanwhile.  Warp w owns the packed
// rows w, w + 8, ... through scores, softmax and values, so a step has two block barriers and none
// between those: scores with a lane per token (two), the row's maximum by shuffles, values with a lane per D/32
// columns and O in registers.  Bound by shared-memory reads: a K or V vector costs four cycles of it and
// feeds 4 kRows fused multiply-adds a lane.  The kernel for pools of the kv dtype, which takes its elements
// one by one and keeps O in shared memory, takes 75 us a call there where this one takes 37 (4 requests of up to 256 tokens; 30 of them in this kernel).
#pragma once
#include "attn_e4m3.cuh"   // e8: two fp32 operations in one instruction
#include "attn_simt.cuh"
#include "kv_cache_e4m3.cuh"   // decode8

namespace spx {

constexpr int kSfThreads = 256;
constexpr int kSfTokens = 64;   // tokens per step

struct SfSmem {
  int q, k, v, p, total;
  __host__ __device__ SfSmem(int R, int D) {
    int off = 0;
    q = off; off += R * D * 4;
    k = off; off += kSfTokens * (D + 4) * 4;   // rows padded: eight lanes read eight banks of 16 bytes
    v = off; off += kSfTokens * D * 4;
    p = off; off += R * kSfTokens * 4;
    total = off;
  }
};

// kRows: packed rows per warp, at least (G * m + 7) / 8.
template <typename T, int D, int kRows>
__global__ void __launch_bounds__(kSfThreads) attn_simt_e4m3_kernel(AttnParams p) {
  SPX_TL_SCOPE(kTlAttention);
  // the combine kernel may take its places now (see attn_simt_kernel)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ __align__(16) unsigned char smem_raw[];
  __shared__ int s_item, s_nan;
  const SfSmem lay(p.rows_cap, D);
  float *sQ = reinterpret_cast<float *>(smem_raw + lay.q), *sK = reinterpret_cast<float *>(smem_raw + lay.k);
  float *sV = reinterpret_cast<float *>(smem_raw + lay.v), *sP = reinterpret_cast<float *>(smem_raw + lay.p);
  const T *Q = reinterpret_cast<const T *>(p.q);
  const unsigned char *Kc = reinterpret_cast<const unsigned char *>(p.k_cache), *Vc = reinterpret_cast<const unsigned char *>(p.v_cache);
  T *out = reinterpret_cast<T *>(p.out);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kVecs = D / 16;                              // 16-code vectors of a token
  constexpr int kMine = kSfTokens * kVecs / kSfThreads;      // of them a thread's, in K and in V: 1 or 2
  constexpr int kCols = D / 32;                              // output columns of a lane: 2 or 4
  static_assert(kMine >= 1, "a vector for each thread");
  if (p.hdr->overflow) return;
  const int n_items = p.hdr->n_work;

  for (;;) {
    __syncthreads();
    if (tid == 0) { s_item = atomicAdd(&p.hdr->work_counter, 1); s_nan = 0; }
    __syncthreads();
    const int item = s_item;
    if (item >= n_items) break;
    const WorkEntry we = p.work[item];
    const int g = we.g, q0 = we.q0, m = we.m, L = we.L, G = p.G, R = m * G;
    const int t_begin = we.tile_begin * kTileTokens, t_end = min(we.tile_end * kTileTokens, L);
    const int32_t *bt = p.block_table + (int64_t)we.req * p.max_pages_per_req;

    // a thread's tokens of the step at t0 are t0 + tid / kVecs + i * (256 / kVecs), its columns (tid % kVecs) * 16 ..
    const int my_tok = tid / kVecs, my_col = (tid % kVecs) * 16;
    auto page_of = [&](int t0, int i) -> int {
      const int t = t0 + my_tok + i * (kSfThreads / kVecs);
      if (t >= t_end) return -1;
      const int page = bt[t >> p.log2P];
      if (page < 0 || page >= p.num_pages) {
        atomicOr(p.dev_status, SPX_DEV_BAD_PAGE);
        p.req_bad[we.req] = 1;   // the combine kernel writes the request's sentinel rows
        return -1;
      }
      return page;
    };
    uint4 k_codes[kMine], v_codes[kMine];
    float k_scale[kMine], v_scale[kMine];
    auto fetch = [&](int t0, const int (&page)[kMine]) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        k_codes[i] = v_codes[i] = make_uint4(0, 0, 0, 0);
        k_scale[i] = v_scale[i] = 0.f;
        if (page[i] < 0) continue;
        const int slot = (t0 + my_tok + i * (kSfThreads / kVecs)) & (p.P - 1);
        const int64_t at = (int64_t)page[i] * p.stride_page + (int64_t)g * p.stride_head + (int64_t)slot * p.stride_token + my_col;
        const int64_t si = (((int64_t)page[i] * p.Hkv + g) << (p.log2P - p.log2SB)) + (slot >> p.log2SB);
        k_codes[i] = __ldg(reinterpret_cast<const uint4 *>(Kc + at));
        v_codes[i] = __ldg(reinterpret_cast<const uint4 *>(Vc + at));
        k_scale[i] = __ldg(p.k_scales + si);
        v_scale[i] = __ldg(p.v_scales + si);
      }
    };
    int page[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) page[i] = page_of(t_begin, i);
    // queries, scaled into the log2 domain
    for (int i = tid; i < R * D; i += kSfThreads) {
      const int row = i / D, d = i % D, j = row / G, hg = row % G;
      sQ[i] = ld_as_float(Q, ((int64_t)(q0 + j) * p.Hq + g * G + hg) * D + d) * p.scale_log2;
    }
    fetch(t_begin, page);
#pragma unroll
    for (int i = 0; i < kMine; ++i) page[i] = page_of(t_begin + kSfTokens, i);

    float o[kRows][kCols], m_run[kRows], l_run[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      m_run[i] = -INFINITY;
      l_run[i] = 0.f;
#pragma unroll
      for (int c = 0; c < kCols; ++c) o[i][c] = 0.f;
    }
    // rows past the end are computed like the last one and not written
    int row_of[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) row_of[i] = min(warp + 8 * i, R - 1);

    for (int t0 = t_begin; t0 < t_end; t0 += kSfTokens) {
      __syncthreads();   // the last step's K and V have been read
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int tok = my_tok + i * (kSfThreads / kVecs);
        float x[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          decode8(h ? make_uint2(k_codes[i].z, k_codes[i].w) : make_uint2(k_codes[i].x, k_codes[i].y), x);
          float4 *dst = reinterpret_cast<float4 *>(sK + tok * (D + 4) + my_col + 8 * h);
          dst[0] = make_float4(x[0] * k_scale[i], x[1] * k_scale[i], x[2] * k_scale[i], x[3] * k_scale[i]);
          dst[1] = make_float4(x[4] * k_scale[i], x[5] * k_scale[i], x[6] * k_scale[i], x[7] * k_scale[i]);
        }
        bool nan = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          decode8(h ? make_uint2(v_codes[i].z, v_codes[i].w) : make_uint2(v_codes[i].x, v_codes[i].y), x);
          float4 *dst = reinterpret_cast<float4 *>(sV + tok * D + my_col + 8 * h);
#pragma unroll
          for (int u = 0; u < 8; ++u) { x[u] *= v_scale[i]; nan |= x[u] != x[u]; }
          dst[0] = make_float4(x[0], x[1], x[2], x[3]);
          dst[1] = make_float4(x[4], x[5], x[6], x[7]);
        }
        if (nan && t0 + tok > L - m) s_nan = 1;   // at a position that some rows do not see
      }
      __syncthreads();
      if (t0 + kSfTokens < t_end) {
        fetch(t0 + kSfTokens, page);
#pragma unroll
        for (int i = 0; i < kMine; ++i) page[i] = page_of(t0 + 2 * kSfTokens, i);
      }
      // ---- scores: two tokens a lane
      float s[kRows][2];
#pragma unroll
      for (int i = 0; i < kRows; ++i) s[i][0] = s[i][1] = 0.f;
      const float4 *k0 = reinterpret_cast<const float4 *>(sK + lane * (D + 4)), *k1 = reinterpret_cast<const float4 *>(sK + (lane + 32) * (D + 4));
#pragma unroll 4
      for (int d = 0; d < D / 4; ++d) {
        const float4 a = k0[d], b = k1[d];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const float4 q = *reinterpret_cast<const float4 *>(sQ + row_of[i] * D + 4 * d);
          s[i][0] = fmaf(q.w, a.w, fmaf(q.z, a.z, fmaf(q.y, a.y, fmaf(q.x, a.x, s[i][0]))));
          s[i][1] = fmaf(q.w, b.w, fmaf(q.z, b.z, fmaf(q.y, b.y, fmaf(q.x, b.x, s[i][1]))));
        }
      }
      // ---- softmax; a hidden position's weight is -1 in shared memory where a NaN makes the difference
      const bool apart = s_nan != 0;
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const int limit = min(L - m + row_of[i] / G, t_end - 1);
        const bool vis0 = t0 + lane <= limit, vis1 = t0 + lane + 32 <= limit;
        const float a = vis0 ? s[i][0] : -INFINITY, b = vis1 ? s[i][1] : -INFINITY;
        const float m_new = fmaxf(m_run[i], warp_max(fmaxf(a, b)));
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float p0 = vis0 ? fast_exp2(a - m_use) : 0.f, p1 = vis1 ? fast_exp2(b - m_use) : 0.f;
        const float alpha = m_new == -INFINITY ? 1.f : fast_exp2(m_run[i] - m_new);
        l_run[i] = fmaf(l_run[i], alpha, warp_sum(p0 + p1));
        m_run[i] = m_new;
#pragma unroll
        for (int c = 0; c < kCols; ++c) o[i][c] *= alpha;
        if (warp + 8 * i < R) {
          sP[row_of[i] * kSfTokens + lane] = apart && !vis0 ? -1.f : p0;
          sP[row_of[i] * kSfTokens + lane + 32] = apart && !vis1 ? -1.f : p1;
        }
      }
      __syncwarp();
      // ---- values: kCols columns a lane
#pragma unroll 2
      for (int t = 0; t < kSfTokens; t += 4) {
        float v[4][kCols];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if constexpr (kCols == 4) {
            const float4 x = *reinterpret_cast<const float4 *>(sV + (t + u) * D + lane * 4);
            v[u][0] = x.x; v[u][1] = x.y; v[u][2] = x.z; v[u][3] = x.w;
          } else {
            const float2 x = *reinterpret_cast<const float2 *>(sV + (t + u) * D + lane * 2);
            v[u][0] = x.x; v[u][1] = x.y;
          }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const float4 w4 = *reinterpret_cast<const float4 *>(sP + row_of[i] * kSfTokens + t);
          const float w[4] = {w4.x, w4.y, w4.z, w4.w};
          if (apart) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (!(w[u] < 0.f))
#pragma unroll
                for (int c = 0; c < kCols; ++c) o[i][c] = fmaf(w[u], v[u][c], o[i][c]);
          } else {
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
              for (int c = 0; c < kCols; ++c) o[i][c] = fmaf(w[u], v[u][c], o[i][c]);
          }
        }
      }
      __syncwarp();   // the weights are rewritten by the next step
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int row = warp + 8 * i;
      if (row >= R) continue;
      if (we.part_slot < 0) {
        const int64_t at = (int64_t)(q0 + row / G) * p.Hq + g * G + row % G;
#pragma unroll
        for (int c = 0; c < kCols; ++c) st_from_float(out, at * D + lane * kCols + c, o[i][c] / l_run[i]);
        if (lane == 0 && p.lse) p.lse[at] = (m_run[i] + log2f(l_run[i])) * kLn2;
      } else {
        const int64_t slot = (int64_t)we.part_slot * p.rows_cap + row;
        // (a NaN sum stays one where the chunks are merged)
        const float m_part = l_run[i] != l_run[i] ? 0.f : m_run[i];
#pragma unroll
        for (int c = 0; c < kCols; ++c) p.part_o[slot * D + lane * kCols + c] = o[i][c];
        if (lane == 0) p.part_ml[slot] = make_float2(m_part, l_run[i]);
      }
    }
  }
}

}  // namespace spx
