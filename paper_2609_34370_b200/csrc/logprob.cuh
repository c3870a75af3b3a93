// Log-probabilities of given tokens, row entropies and top alternatives.
//
// With m the row's largest logit, lse = m + log(1 + rest), rest = sum_v e^(x_v - m) without one of the
// largest, and the entropy is log(1 + rest) - E[x - m].  The alternatives are the top_n by (logit, -id).
//
// One pass over the logits: a bulk-copy ring feeds warps that each reduce 4 KB of a row (a sub-segment:
// 2048 bf16 or 1024 fp32 logits) to its maximum, sum e^(x - M), sum e^(x - M) (x - M), and to the maxima of
// its 32 lanes' shares (a group: 64 or 32 logits).  A block per row then merges the sub-segments in 64 bits
// and finds the alternatives from the group maxima: the n-th largest sub-segment maximum bounds the n-th
// largest logit from below, so only groups whose maximum reaches it are read again (some 30 of 2016
// for 20 of 128,256).  Bound by HBM, with the exponential unit close behind (16 a cycle and SM, 72% busy at HBM's full
// rate on bf16 rows): 384 rows of 128,256 bf16 logits take 34.8 us a call, 23.4 of them in the pass (98.5 MB: 4.2
// TB/s, its start and end included) and some 9 in the merge, which is a chain of barriers and dependent reads.
#pragma once
#include "attn_e4m3.cuh"   // e8::pair and the packed fp32 arithmetic
#include "common.cuh"
#include "sampler.cuh"     // ring_wait

namespace spx {

constexpr int kLpSubBytes = 4096;                   // a sub-segment: one warp, 8 16-byte vectors a lane
constexpr int kLpStageSubs = 8;                     // sub-segments of a full ring stage
constexpr int kLpStages = 6;
constexpr int kLpGroups = 3;                        // groups of 8 consumer warps, each takes every third chunk
constexpr int kLpThreads = (kLpGroups * kLpStageSubs + 1) * 32;
constexpr int kLpSmemBytes = kLpStages * kLpStageSubs * kLpSubBytes + 1024 + 256;
constexpr int kLpTailThreads = 128;
constexpr int kLpMaxCand = 128;                     // groups looked at again in the common case
constexpr int kLpMaxList = 2048;                    // candidates: at least 31 groups of 64 and 32 more

struct LogprobParams {
  int32_t rows, vocab, top_n;
  int32_t nsub;             // sub-segments of a row
  int32_t chunk_subs;       // sub-segments of a ring stage: fewer than 8 when there are few rows
  int32_t chunks_per_row, n_chunks;
  int64_t row_stride;
  const void *logits;
  const int32_t *token_ids;
  float *logprobs, *entropy, *top_logprobs;
  int32_t *top_ids;
  float4 *seg;              // [rows][nsub]: maximum, sum, sum of products (log2 units)
  void *group_max;          // [rows][nsub][32] of the logits' type
  int32_t *dev_status;
};

// Order of the alternatives, as an unsigned key: larger logits first, equal ones (-0 and +0 too) alike,
// NaN above +inf.  16 bits hold a bf16 logit's.
__device__ __forceinline__ uint32_t logit_key32(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __float_as_uint(x + 0.f);   // -0 becomes +0
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
template <typename T>
__device__ __forceinline__ uint32_t logit_key(float x) { return sizeof(T) == 2 ? logit_key32(x) >> 16 : logit_key32(x); }
// the logit of a key (of -0: +0)
template <typename T>
__device__ __forceinline__ float key_logit(uint32_t key) {
  const uint32_t u = sizeof(T) == 2 ? key << 16 : key;
  return __uint_as_float((u & 0x80000000u) ? u ^ 0x80000000u : sizeof(T) == 2 ? ~u & 0xffff0000u : ~u);
}

template <typename T> struct LpVec;
template <> struct LpVec<__nv_bfloat16> {
  static constexpr int N = 8;                     // logits of a vector
  static constexpr int kSub = kLpSubBytes / 2;
  // the vector with the logits from `valid` on as -inf
  __device__ static uint4 cut(uint4 v, int valid) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (2 * j >= valid) w[j] = (w[j] & 0xffff0000u) | 0xff80u;
      if (2 * j + 1 >= valid) w[j] = (w[j] & 0x0000ffffu) | 0xff800000u;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ static uint32_t max_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  __device__ static float lane_max(const uint4 (&v)[8]) {
    uint32_t m = v[0].x;
#pragma unroll
    for (int c = 0; c < 8; ++c) m = max_nan(m, max_nan(max_nan(v[c].x, v[c].y), max_nan(v[c].z, v[c].w)));
    m = max_nan(m, m >> 16 | m << 16);
    return __uint_as_float(m << 16);
  }
  // pair i of the vector's logits, those below `floor` raised to it
  __device__ static uint64_t pair_of(const uint4 &v, int i, uint32_t floor2) {
    const uint32_t w = max_nan(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w, floor2);
    return e8::pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  __device__ static uint32_t floor_bits(float f) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(f, f);
    return *reinterpret_cast<const uint32_t *>(&b);
  }
  __device__ static float at(const uint4 &v, int i) {
    const uint32_t w = (i >> 1) == 0 ? v.x : (i >> 1) == 1 ? v.y : (i >> 1) == 2 ? v.z : v.w;
    return __uint_as_float((i & 1) ? w & 0xffff0000u : w << 16);
  }
};
template <> struct LpVec<float> {
  static constexpr int N = 4;
  static constexpr int kSub = kLpSubBytes / 4;
  __device__ static uint4 cut(uint4 v, int valid) {
    return make_uint4(valid > 0 ? v.x : 0xff800000u, valid > 1 ? v.y : 0xff800000u, valid > 2 ? v.z : 0xff800000u, valid > 3 ? v.w : 0xff800000u);
  }
  __device__ static float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
  }
  __device__ static float lane_max(const uint4 (&v)[8]) {
    float m = __uint_as_float(v[0].x);
#pragma unroll
    for (int c = 0; c < 8; ++c)
      m = max_nan(m, max_nan(max_nan(__uint_as_float(v[c].x), __uint_as_float(v[c].y)), max_nan(__uint_as_float(v[c].z), __uint_as_float(v[c].w))));
    return m;
  }
  __device__ static uint64_t pair_of(const uint4 &v, int i, uint32_t floor2) {
    const float f = __uint_as_float(floor2);
    return i == 0 ? e8::pair(max_nan(__uint_as_float(v.x), f), max_nan(__uint_as_float(v.y), f))
                  : e8::pair(max_nan(__uint_as_float(v.z), f), max_nan(__uint_as_float(v.w), f));
  }
  __device__ static uint32_t floor_bits(float f) { return __float_as_uint(f); }
  __device__ static float at(const uint4 &v, int i) { return __uint_as_float(i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w); }
};

// grid: one CTA per SM at most; chunk g of the list (row, share of the row) goes to CTA g % gridDim.x.
template <typename T>
__global__ void __launch_bounds__(kLpThreads, 1) logprob_stats_kernel(LogprobParams p) {
  using V = LpVec<T>;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the merge kernel's blocks may take their places
  extern __shared__ __align__(1024) unsigned char lp_smem[];
  unsigned char *stages = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(lp_smem) + 1023) & ~uintptr_t(1023));
  uint64_t *full = reinterpret_cast<uint64_t *>(stages + kLpStages * kLpStageSubs * kLpSubBytes);
  uint64_t *empty = full + kLpStages;
  volatile int *abort = reinterpret_cast<volatile int *>(empty + kLpStages);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kLpStages; ++s) {
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(&full[s])), "r"(1));
      asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(&empty[s])), "r"(kLpStageSubs));
    }
    *abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  const T *logits = reinterpret_cast<const T *>(p.logits);
  const int chunk_elems = p.chunk_subs * V::kSub;
  // rows without a token are not read
  auto token_of = [&](int g) -> int { return p.token_ids ? p.token_ids[g / p.chunks_per_row] : 0; };
  auto counts = [&](int tok) -> bool { return tok >= 0 && tok < p.vocab; };
  if (warp == kLpGroups * kLpStageSubs) {
    // ---- producer (one thread)
    if (lane == 0) {
      int i = 0;
      int tok_next = (int)blockIdx.x < p.n_chunks ? token_of(blockIdx.x) : 0;
      for (int g = blockIdx.x; g < p.n_chunks; g += gridDim.x, ++i) {
        const int tok = tok_next;
        if (g + (int)gridDim.x < p.n_chunks) tok_next = token_of(g + gridDim.x);   // off the issue path
        const int s = i % kLpStages;
        if (i >= kLpStages && !ring_wait(&empty[s], ((i / kLpStages) - 1) & 1, abort, p.dev_status)) break;
        const int row = g / p.chunks_per_row, e0 = (g % p.chunks_per_row) * chunk_elems;
        const uint32_t bar = (uint32_t)__cvta_generic_to_shared(&full[s]);
        if (!counts(tok)) {
          // handed over empty, the consumers release it at once
          asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
          continue;
        }
        const int elems = min(chunk_elems, p.vocab - e0);
        const uint32_t bytes = (uint32_t)((elems * (int)sizeof(T) + 15) & ~15);  // stays inside the row: its stride is a multiple of 16 bytes
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                     ::"r"((uint32_t)__cvta_generic_to_shared(stages + (size_t)s * kLpStageSubs * kLpSubBytes)),
                       "l"(logits + (int64_t)row * p.row_stride + e0), "r"(bytes), "r"(bar) : "memory");
      }
    }
  } else {
    // ---- consumers: group `grp` takes chunks grp, grp + kLpGroups, ...; its warp w reduces sub-segment w
    const int grp = warp / kLpStageSubs, wsub = warp % kLpStageSubs;
    int i = grp;
    for (int g = blockIdx.x + grp * gridDim.x; g < p.n_chunks; g += kLpGroups * gridDim.x, i += kLpGroups) {
      const int s = i % kLpStages;
      const int row = g / p.chunks_per_row, sub = (g % p.chunks_per_row) * p.chunk_subs + wsub;
      const int tok = token_of(g);   // in flight while the stage fills
      const bool ok = __all_sync(0xffffffffu, ring_wait(&full[s], (i / kLpStages) & 1, abort, p.dev_status));
      if (!ok) break;
      const bool mine = wsub < p.chunk_subs && sub < p.nsub && counts(tok);
      uint4 v[8];
      if (mine) {
        const uint4 *src = reinterpret_cast<const uint4 *>(stages + (size_t)(s * kLpStageSubs + wsub) * kLpSubBytes);
        const int left = p.vocab - sub * V::kSub;   // logits of the row from this sub-segment on
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          v[c] = src[c * 32 + lane];
          const int at = (c * 32 + lane) * V::N;
          if (at + V::N > left) v[c] = V::cut(v[c], left - at);   // past the vocabulary: never copied, or the row's padding
        }
      }
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"((uint32_t)__cvta_generic_to_shared(&empty[s])) : "memory");
      if (!mine) continue;
      const float lm = V::lane_max(v);
      const int64_t at = (int64_t)row * p.nsub + sub;
      st_from_float(reinterpret_cast<T *>(p.group_max), at * 32 + lane, lm);
      const bool nan = __any_sync(0xffffffffu, lm != lm);
      const float M = warp_max(lm);
      float S, P;
      if (nan || M == INFINITY) {
        S = P = __int_as_float(0x7fc00000);   // the row has no finite sum
      } else if (M == -INFINITY) {
        S = P = 0.f;
      } else if (M < -1e37f) {
        // a row of the types' lowest values: the floor below has no room under them
        S = P = 0.f;
#pragma unroll 1
        for (int c = 0; c < 8; ++c)
          for (int k = 0; k < V::N; ++k) {
            uint4 w = v[0];
#pragma unroll
            for (int u = 1; u < 8; ++u) w = c == u ? v[u] : w;
            const float t = fmaxf((V::at(w, k) - M) * kLog2e, -400.f), e = fast_exp2(t);
            S += e;
            P = fmaf(e, t, P);
          }
        S = warp_sum(S);
        P = warp_sum(P);
      } else {
        // logits more than 256 below the maximum (-inf among them) add nothing: they are raised to that, so that no
        // product is 0 * inf
        const uint32_t floor2 = V::floor_bits(M - fmaxf(256.f, fabsf(M) * 0.015625f));
        const uint64_t minus_m = e8::pair(-M, -M), log2e = e8::pair(kLog2e, kLog2e);
        uint64_t sum = 0, prod = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
          for (int k = 0; k < V::N / 2; ++k) {
            const uint64_t t = e8::mul2(e8::add2(V::pair_of(v[c], k, floor2), minus_m), log2e);
            float a, b;
            e8::unpair(t, a, b);
            const uint64_t e = e8::pair(fast_exp2(a), fast_exp2(b));
            sum = e8::add2(sum, e);
            prod = e8::fma2(e, t, prod);
          }
        float a, b;
        e8::unpair(sum, a, b);
        S = warp_sum(a + b);
        e8::unpair(prod, a, b);
        P = warp_sum(a + b);
      }
      if (lane == 0) p.seg[at] = make_float4(nan ? __int_as_float(0x7fc00000) : M, S, P, 0.f);
    }
  }
}

// One block per row: merge, then the alternatives.  A chain of dependent reads (statistics -> candidate groups ->
// their logits) with little between them: what the next step reads is asked for as early as it is known,
// and the 64-bit sums are done while the candidates' logits are on their way.
template <typename T>
__global__ void __launch_bounds__(kLpTailThreads) logprob_merge_kernel(LogprobParams p) {
  using V = LpVec<T>;
  constexpr int kThreads = kLpTailThreads, kWarps = kThreads / 32, kKeyBits = sizeof(T) * 8;
  constexpr int kMaxVecs = 2;            // 16-byte vectors of group maxima a thread holds in the common case
  __shared__ float s_f[kWarps];
  __shared__ double s_d[3][kWarps];
  __shared__ int s_i[kWarps];
  __shared__ uint32_t s_floor;
  __shared__ int s_cand_n, s_list_n;
  __shared__ __align__(16) uint32_t s_key[kThreads];
  __shared__ int s_cand[kLpMaxCand];
  __shared__ uint2 s_list[kLpMaxList];   // (key, ~id)
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int tok = p.token_ids ? p.token_ids[row] : 0;
  const float nan = __int_as_float(0x7fc00000);
  const T *x = reinterpret_cast<const T *>(p.logits) + (int64_t)row * p.row_stride;
  const bool counted = tok >= 0 && tok < p.vocab;
  const float x_tok = counted ? ld_as_float(x, tok) : 0.f;
  const int n = p.top_n;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // the statistics are read from here on
  if (!counted) {
    if (tid == 0) {
      if (p.logprobs) p.logprobs[row] = nan;
      if (p.entropy) p.entropy[row] = nan;
      if (tok != -1) atomicOr(p.dev_status, SPX_DEV_BAD_TOKEN);
    }
    if (tid < n) {
      if (p.top_ids) p.top_ids[(int64_t)row * n + tid] = -1;
      if (p.top_logprobs) p.top_logprobs[(int64_t)row * n + tid] = nan;
    }
    return;
  }
  const float4 *seg = p.seg + (int64_t)row * p.nsub;
  const T *gmax = reinterpret_cast<const T *>(p.group_max) + (int64_t)row * p.nsub * 32;
  const int n_groups = p.nsub * 32, n_vecs = n_groups / V::N;
  const float4 seg0 = tid < p.nsub ? seg[tid] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  const uint4 *gvec = reinterpret_cast<const uint4 *>(gmax);
  uint4 gv[kMaxVecs];
  if (n > 0) {
#pragma unroll
    for (int u = 0; u < kMaxVecs; ++u)
      if (tid + u * kThreads < n_vecs) gv[u] = gvec[tid + u * kThreads];
  }

  // ---- the row's maximum, and whether it has finite sums
  float m = seg0.x;
  bool bad = seg0.x != seg0.x || seg0.x == INFINITY;
  for (int i = tid + kThreads; i < p.nsub; i += kThreads) {
    const float f = seg[i].x;
    bad |= f != f || f == INFINITY;
    m = fmaxf(m, f);
  }
  m = warp_max(m);
  if (lane == 0) s_f[warp] = m;
  // Keys whose n-th largest bounds the n-th largest logit from below: the sub-segments' maxima, or, of a row
  // with fewer than n, the maxima of their q equal shares, the least power of two that makes n of them
  int q = 1;
  while (p.nsub * q < n) q *= 2;
  const int n_keys = p.nsub * q;
  uint32_t my_key = 0;
  if (n > 0) {
    if (q == 1) {
      my_key = logit_key<T>(seg0.x);
    } else if (tid < n_keys) {
      for (int i = 0; i < 32 / q; ++i) my_key = max(my_key, logit_key<T>(ld_as_float(gmax, tid * (32 / q) + i)));
    }
    s_key[tid] = tid < n_keys ? my_key : 0;
  }
  if (tid == 0) { s_cand_n = 0; s_list_n = 0; s_floor = 0xffffffffu; }
  bad = __syncthreads_or(bad);
#pragma unroll
  for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s_f[w]);
  bad |= m == -INFINITY;

  // the k-th largest of key_of(i), i < total (or a key that exactly k reach): bit by bit from the top
  auto kth_largest = [&](int total, int k, auto key_of) -> uint32_t {
    uint32_t thr = 0;
#pragma unroll 1
    for (int bit = kKeyBits - 1; bit >= 0; --bit) {
      const uint32_t cand = thr | (1u << bit);
      int count = 0;
      for (int i0 = 0; i0 < total; i0 += kThreads) count += __syncthreads_count(i0 + tid < total && key_of(i0 + tid) >= cand);
      if (count >= k) {
        thr = cand;
        if (count == k) break;
      }
    }
    return thr;
  };
  auto group_key = [&](int i) -> uint32_t { return logit_key<T>(ld_as_float(gmax, i)); };
  // the logits of the listed groups, one vector of a group per thread and round
  auto vec_at = [&](int i) -> int {
    const int g = s_cand[i >> 3], c = i & 7;
    return (g >> 5) * V::kSub + (c * 32 + (g & 31)) * V::N;
  };
  uint32_t floor_key = 0;
  int n_cand = 0;
  uint4 held[kMaxVecs];
  if (n > 0) {
    if (n_keys <= kThreads) {
      // the smallest of the keys that fewer than n others exceed, every thread counting for its own (they lie behind one
      // another in shared memory, zeros behind the last)
      uint32_t mine = 0xffffffffu;
      if (tid < n_keys) {
        int above = 0;
#pragma unroll 4
        for (int j = 0; j < n_keys; j += 4) {
          const uint4 k = *reinterpret_cast<const uint4 *>(s_key + j);
          above += (k.x > my_key) + (k.y > my_key) + (k.z > my_key) + (k.w > my_key);
        }
        if (above < n) mine = my_key;
      }
      mine = __reduce_min_sync(0xffffffffu, mine);
      if (lane == 0 && mine != 0xffffffffu) atomicMin(&s_floor, mine);
      __syncthreads();
      floor_key = s_floor;
    } else {
      floor_key = kth_largest(n_keys, n, [&](int i) -> uint32_t { return i == tid ? my_key : logit_key<T>(seg[i].x); });
    }
    auto list_vec = [&](const uint4 &v, int base) {
      uint32_t hits = 0;
#pragma unroll
      for (int k = 0; k < V::N; ++k) hits |= (uint32_t)(logit_key<T>(V::at(v, k)) >= floor_key) << k;
      if (hits == 0) return;
      for (int at = atomicAdd(&s_cand_n, __popc(hits)); hits != 0; ++at, hits &= hits - 1)
        if (at < kLpMaxCand) s_cand[at] = base + __ffs(hits) - 1;
    };
#pragma unroll
    for (int u = 0; u < kMaxVecs; ++u)
      if (tid + u * kThreads < n_vecs) list_vec(gv[u], (tid + u * kThreads) * V::N);
    for (int i = tid + kMaxVecs * kThreads; i < n_vecs; i += kThreads) list_vec(gvec[i], i * V::N);
    __syncthreads();
    n_cand = s_cand_n;
    if (n_cand <= kLpMaxCand) {
#pragma unroll
      for (int u = 0; u < kMaxVecs; ++u)
        if (tid + u * kThreads < n_cand * 8) {
          const int e0 = vec_at(tid + u * kThreads);
          if (e0 < p.vocab) held[u] = *reinterpret_cast<const uint4 *>(x + e0);
        }
    }
  }

  // ---- rest = sum e^(x - m) without one of the largest, and sum e^(x - m) (x - m), in 64 bits.  top: the first
  // sub-segment that holds the maximum
  double rest = 0.0, prod = 0.0, log_z = 0.0;
  if (!bad) {
    double top_sum = 0.0;
    int top = 0x7fffffff;
    for (int i = tid; i < p.nsub; i += kThreads) {
      const float4 f = i == tid ? seg0 : seg[i];
      if (f.x == -INFINITY) continue;
      const float d = f.x - m;   // (a rounded difference is a factor off by 2^-24 |d|)
      const float w = expf(d);
      if (w == 0.f) continue;    // its tokens have p = 0 (and d may be past the largest float: no product is 0 * inf)
      prod += (double)w * fma((double)f.z, 0.6931471805599453, (double)f.y * (double)d);
      if (d == 0.f && top == 0x7fffffff) { top = i; top_sum = f.y; }   // (a thread's first)
      else rest += (double)w * (double)f.y;
    }
    const int top_mine = top;
    top = __reduce_min_sync(0xffffffffu, top);
    if (lane == 0) s_i[warp] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = min(top, s_i[w]);
    if (top_mine != top) { rest += top_sum; top_sum = 0.0; }   // holds the maximum too, but not first
    auto block_sum3 = [&](double &a, double &b, double &c) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, o);
        b += __shfl_xor_sync(0xffffffffu, b, o);
        c += __shfl_xor_sync(0xffffffffu, c, o);
      }
      if (lane == 0) { s_d[0][warp] = a; s_d[1][warp] = b; s_d[2][warp] = c; }
      __syncthreads();
      a = b = c = 0.0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) { a += s_d[0][w]; b += s_d[1][w]; c += s_d[2][w]; }
    };
    double others = rest;
    block_sum3(others, prod, top_sum);
    rest = others + (top_sum - 1.0);
    if (rest < 0.125) {
      // near-certain row: the sub-segment's fp32 sum has rounded its share of the rest against the maximum's 1;
      // add it up again without that
      double a = 0.0, n_max = 0.0, none = 0.0;
      const int e0 = top * V::kSub;
      for (int i = tid; i < V::kSub && e0 + i < p.vocab; i += kThreads) {
        const float d = ld_as_float(x, e0 + i) - m;
        if (d == 0.f) n_max += 1.0;
        else a += (double)expf(d);
      }
      __syncthreads();
      block_sum3(a, n_max, none);
      rest = others + a + (n_max - 1.0);
    }
    log_z = log1p(rest);
  }
  if (tid == 0) {
    if (p.logprobs) p.logprobs[row] = bad ? nan : (float)((double)x_tok - m - log_z);
    if (p.entropy) p.entropy[row] = bad ? nan : (float)(log_z - prod / (1.0 + rest));
  }
  if (n == 0) return;

  // ---- the alternatives: every logit of the listed groups for which take(key) holds, behind the list's end
  // (which of a vector's logits first, without a branch each: eight of them a vector were 3,500 cycles a row)
  auto take_vec = [&](const uint4 &v, int e0, auto take) {
    uint32_t hits = 0, key[V::N];
#pragma unroll
    for (int k = 0; k < V::N; ++k) {
      key[k] = logit_key<T>(V::at(v, k));
      hits |= (uint32_t)(take(key[k]) && e0 + k < p.vocab) << k;
    }
    if (hits == 0) return;
    int at = atomicAdd(&s_list_n, __popc(hits));
#pragma unroll
    for (int k = 0; k < V::N; ++k)
      if (hits >> k & 1) {
        if (at < kLpMaxList) s_list[at] = make_uint2(key[k], ~(uint32_t)(e0 + k));
        ++at;
      }
  };
  auto gather = [&](int i0, int cands, auto take) {
    for (int i = i0 + tid; i < cands * 8; i += kThreads) {
      const int e0 = vec_at(i);
      if (e0 < p.vocab) take_vec(*reinterpret_cast<const uint4 *>(x + e0), e0, take);
    }
    __syncthreads();
  };
  bool listed = n_cand <= kLpMaxCand;
  if (listed) {
    auto take = [&](uint32_t key) { return key >= floor_key; };
#pragma unroll
    for (int u = 0; u < kMaxVecs; ++u)
      if (tid + u * kThreads < n_cand * 8) {
        const int e0 = vec_at(tid + u * kThreads);
        if (e0 < p.vocab) take_vec(held[u], e0, take);
      }
    gather(kMaxVecs * kThreads, n_cand, take);
    listed = s_list_n <= kLpMaxList;
  }
  if (!listed) {
    // ties by the hundred (a masked or constant row): with thr the n-th largest group maximum at most n groups lie
    // above it, and all their logits above thr fit the list; the ones equal to it are taken by ascending id
    const uint32_t thr = kth_largest(n_groups, n, group_key);
    __syncthreads();
    if (tid == 0) { s_cand_n = 0; s_list_n = 0; }
    __syncthreads();
    for (int i = tid; i < n_groups; i += kThreads)
      if (group_key(i) > thr) {
        const int at = atomicAdd(&s_cand_n, 1);
        if (at < kLpMaxCand) s_cand[at] = i;
      }
    __syncthreads();
    gather(0, min(s_cand_n, kLpMaxCand), [&](uint32_t key) { return key > thr; });
    const int above = s_list_n;
    int have = above;
    for (int e0 = 0; have < n && e0 < p.vocab; e0 += kThreads) {
      const int e = e0 + tid;
      const bool tie = e < p.vocab && logit_key<T>(ld_as_float(x, e)) == thr;
      const uint32_t ballot = __ballot_sync(0xffffffffu, tie);
      __syncthreads();
      if (lane == 0) s_i[warp] = __popc(ballot);
      __syncthreads();
      int before = have, all = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) { before += w < warp ? s_i[w] : 0; all += s_i[w]; }
      before += __popc(ballot & ((1u << lane) - 1));
      if (tie && before < n) s_list[before] = make_uint2(thr, ~(uint32_t)e);
      have += all;
    }
    __syncthreads();
    if (tid == 0) s_list_n = min(have, max(n, above));
    __syncthreads();
  }
  // ---- rank the candidates
  const int total = min(s_list_n, kLpMaxList);
  for (int i = tid; i < total; i += kThreads) {
    const uint2 me = s_list[i];
    int rank = 0;
    for (int j = 0; j < total; ++j) {
      const uint2 o = s_list[j];
      rank += o.x > me.x || (o.x == me.x && o.y > me.y);
    }
    if (rank < n) {
      const int id = (int)~me.y;
      if (p.top_ids) p.top_ids[(int64_t)row * n + rank] = id;
      if (p.top_logprobs) p.top_logprobs[(int64_t)row * n + rank] = bad ? nan : (float)((double)key_logit<T>(me.x) - m - log_z);
    }
  }
  if (tid >= total && tid < n) {   // fewer logits than alternatives
    if (p.top_ids) p.top_ids[(int64_t)row * n + tid] = -1;
    if (p.top_logprobs) p.top_logprobs[(int64_t)row * n + tid] = nan;
  }
}

}  // namespace spx
