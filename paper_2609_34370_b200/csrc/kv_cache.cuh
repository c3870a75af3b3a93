// Cache maintenance around the verify step: append the new positions' K/V into their pages,
// shrink the lengths by the rejected drafts afterwards.
#pragma once
#include <type_traits>

#include "common.cuh"
#include "rotate.cuh"

namespace spx {

constexpr int kRopeMaxHeadDim = 512;
constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 8;          // new rows of a block, at most
constexpr int kAppendAngles = 1024;     // (row, pair) angles a block keeps: 8 rows of 256 elements, 4 of 512

struct KvAppendParams {
  int32_t batch, total_q, Hkv, D, P, log2P, num_pages, max_pages_per_req, elem_size;
  int32_t log2_rows;       // new rows of a block
  const unsigned char *new_k, *new_v;
  unsigned char *k_cache, *v_cache;
  int64_t stride_page, stride_head, stride_token;  // elements
  const int32_t *block_table, *seq_lens, *q_indptr;
  int32_t *dev_status;
  double rope_base;        // 0: plain copy; > 0: K rows (and q_rows) are rotated to their positions
  unsigned char *q_rows;   // optional [TQ, Hq, D], rotated into q_out (in place when the two are one)
  unsigned char *q_out;
  int32_t Hq;
};
// Positions of several axes (axes = 0: a row's position is its place in the request).
struct KvAppendAxes {
  int32_t axes;
  const int32_t *positions;
  int64_t position_stride;
  unsigned char axis_of[kRopeMaxHeadDim / 2];
};
struct KvNoAxes {};

// Rotary embedding of the pairs (x[i], x[i + D/2]) of one head vector by angles whose cosine and sine are float64's; results
// rounded to binary32 and then to the element type (nearest even each).  lo / hi are the 16-byte vectors that hold the
// pairs' first and second elements.  cs: the angles of a row, 16 bytes a pair, laid out so that neighbouring vectors' lie side by
// side, vecs vectors to half a row.
//   float32 rows: products and sum in float64, (cos, sin) of vector v's pair u at [u * vecs + v].
//   16-bit rows: products and sum in pairs of binary32 to 2^-46 of |x| (float64's arithmetic but for one in some millions of last
//   bits of binary32, at a third of its time: conversions from and to float64 take 8 cycles each), (cos, cos', low parts) of pairs
//   2u, 2u + 1 at [2u * vecs + v], the sines at [(2u + 1) * vecs + v].
template <typename T>
__device__ __forceinline__ void rope_vectors(uint4 &lo, uint4 &hi, const double2 *cs, int vecs, int v) {
  if constexpr (sizeof(T) == 4) {
    union U { uint4 q; T e[4]; } a, b;
    a.q = lo; b.q = hi;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const double2 k = cs[u * vecs + v];
      const double x0 = (double)a.e[u], x1 = (double)b.e[u];
      a.e[u] = __double2float_rn(x0 * k.x - x1 * k.y);
      b.e[u] = __double2float_rn(x1 * k.x + x0 * k.y);
    }
    lo = a.q; hi = b.q;
  } else {
    const ulonglong2 *at = reinterpret_cast<const ulonglong2 *>(cs);
    uint32_t a[4] = {lo.x, lo.y, lo.z, lo.w}, b[4] = {hi.x, hi.y, hi.z, hi.w};
    uint64_t finite = e8::pair(0.f, 0.f);      // stays zero as long as results are finite
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const ulonglong2 c = at[2 * u * vecs + v], s = at[(2 * u + 1) * vecs + v];
      const CosSin k{c.x, c.y, s.x, s.y};
      uint64_t y0, y1;
      rotate2<true>(e8::pair(__uint_as_float(a[u] << 16), __uint_as_float(a[u] & 0xffff0000u)),
                    e8::pair(__uint_as_float(b[u] << 16), __uint_as_float(b[u] & 0xffff0000u)), k, y0, y1);
      finite = e8::fma2(y0, e8::pair(0.f, 0.f), e8::fma2(y1, e8::pair(0.f, 0.f), finite));
      float p, q;
      e8::unpair(y0, p, q);
      const __nv_bfloat162 r0 = __floats2bfloat162_rn(p, q);
      e8::unpair(y1, p, q);
      const __nv_bfloat162 r1 = __floats2bfloat162_rn(p, q);
      a[u] = *reinterpret_cast<const uint32_t *>(&r0); b[u] = *reinterpret_cast<const uint32_t *>(&r1);
    }
    float p, q;
    e8::unpair(finite, p, q);
    if (p != 0.f || q != 0.f) {
      // an infinity, a NaN or a result past binary32: the remainders above are none then, float64's arithmetic stands
      const float *cs32 = reinterpret_cast<const float *>(cs);
      const __nv_bfloat16 *x = reinterpret_cast<const __nv_bfloat16 *>(&lo), *y = reinterpret_cast<const __nv_bfloat16 *>(&hi);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float *k = cs32 + ((i & 6) * vecs + v) * 4 + (i & 1);
        const double c = (double)k[0] + (double)k[2], sn = (double)k[4 * vecs] + (double)k[4 * vecs + 2];
        const double x0 = (double)__bfloat162float(x[i]), x1 = (double)__bfloat162float(y[i]);
        const __nv_bfloat16 r0 = __float2bfloat16_rn(__double2float_rn(x0 * c - x1 * sn)), r1 = __float2bfloat16_rn(__double2float_rn(x1 * c + x0 * sn));
        const uint32_t w0 = *reinterpret_cast<const uint16_t *>(&r0), w1 = *reinterpret_cast<const uint16_t *>(&r1);
        a[i >> 1] = (i & 1) ? (a[i >> 1] & 0xffffu) | w0 << 16 : (a[i >> 1] & 0xffff0000u) | w0;
        b[i >> 1] = (i & 1) ? (b[i >> 1] & 0xffffu) | w1 << 16 : (b[i >> 1] & 0xffff0000u) | w1;
      }
    }
    lo = make_uint4(a[0], a[1], a[2], a[3]); hi = make_uint4(b[0], b[1], b[2], b[3]);
  }
}

// A block takes up to kAppendRows new rows of a request, all heads of K, V and the query rows, 16 bytes a thread and step.
// Block b belongs to the request r with base(r) <= b < base(r + 1), base(r) = q_indptr[r] / rows + r: m rows are at most
// m / rows + 1 blocks, so no prefix sums are needed; blocks past a request's last one, and past the last request's, leave at once.  The angles are
// worked out once a block and shared by its heads.
// Pure copy and rotation: bound by launch latency at verify-step sizes (a few MB), by HBM beyond that.
// kRope: with a rotary base (without, a kernel of fewer registers).  Eight rows a block, three blocks per SM: five prompts with images 40 us
// (16 rows 49, two vectors a thread in flight 44, four blocks 41).
template <bool kRope>
__global__ void __launch_bounds__(kAppendThreads, 3)
kv_append_kernel(const __grid_constant__ KvAppendParams p, const __grid_constant__ typename std::conditional<kRope, KvAppendAxes, KvNoAxes>::type ax) {
  __shared__ int s_page[kAppendRows], s_first;
  __shared__ uint32_t s_claims[kAppendThreads / 32];   // bit i of word w: request s_first + 32 w + i has rows of this block
  __shared__ double s_inv_freq[kRope ? kRopeMaxHeadDim / 2 : 1];
  __shared__ __align__(16) double2 s_cs[kRope ? kAppendAngles : 1];
  const int tid = threadIdx.x;
  auto valid = [&](int q0, int q1, int L) -> bool {
    return q0 >= 0 && q1 > q0 && q1 <= p.total_q && L >= q1 - q0 && (((int64_t)L + p.P - 1) >> p.log2P) <= (int64_t)p.max_pages_per_req;
  };
  if (p.batch <= kAppendThreads) {
    // the request of this block: each thread looks whether it is its own, in one memory round trip.  (Only where q_indptr descends
    // somewhere can it be more than one, or another than the one whose rows these are by their number.)
    const int c = tid;
    int q0 = 0, q1 = 0, L = 0;
    if (c < p.batch) { q0 = p.q_indptr[c]; q1 = p.q_indptr[c + 1]; L = p.seq_lens[c]; }
    if (kRope)
      for (int i = tid; i < (p.D >> 1); i += kAppendThreads) s_inv_freq[i] = pow(p.rope_base, -2.0 * (double)i / (double)p.D);
    const bool ok = c < p.batch && valid(q0, q1, L);
    const int64_t first = (int64_t)(q0 >> p.log2_rows) + c, next = (int64_t)(q1 >> p.log2_rows) + c + 1;
    const uint32_t claims = __ballot_sync(0xffffffffu, ok && first <= (int64_t)blockIdx.x && (int64_t)blockIdx.x < next);
    if ((tid & 31) == 0) s_claims[tid >> 5] = claims;
    if (tid == 0) s_first = 0;
    if (blockIdx.x == 0 && c < p.batch && !ok) atomicOr(p.dev_status, SPX_DEV_BAD_LEN);
  } else {
    if (kRope)
      for (int i = tid; i < (p.D >> 1); i += kAppendThreads) s_inv_freq[i] = pow(p.rope_base, -2.0 * (double)i / (double)p.D);
    if (tid < 32) {
      // 32 probes at a time
      int lo = 0, hi = p.batch;   // base(lo) <= block, hi past the last candidate
      while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, c = lo + tid * step;
        const bool below = c < hi && (int64_t)(p.q_indptr[c] >> p.log2_rows) + c <= (int64_t)blockIdx.x;
        const int n = __popc(__ballot_sync(0xffffffffu, below || tid == 0));   // the probes ascend
        const int at = lo + (n - 1) * step;
        hi = min(hi, at + step);
        lo = at;
      }
      if (tid < kAppendThreads / 32) s_claims[tid] = tid == 0;
      if (tid == 0) s_first = lo;
    }
    // lengths are looked at by the blocks together (a block of an invalid request may not come to it)
    for (int c = blockIdx.x * kAppendThreads + tid; c < p.batch; c += gridDim.x * kAppendThreads)
      if (!valid(p.q_indptr[c], p.q_indptr[c + 1], p.seq_lens[c])) atomicOr(p.dev_status, SPX_DEV_BAD_LEN);
  }
  __syncthreads();
  // the block's rows of request r, whose bounds are looked at here once more: no thread goes by another's
  auto append = [&](int r) {
    const int q0 = p.q_indptr[r], q1 = p.q_indptr[r + 1], L = p.seq_lens[r], m = q1 - q0;
    if (!valid(q0, q1, L)) return;
    const int64_t j0_64 = ((int64_t)blockIdx.x - ((q0 >> p.log2_rows) + (int64_t)r)) << p.log2_rows;
    if (j0_64 < 0 || j0_64 >= m) return;
    const int j0 = (int)j0_64, n = min(1 << p.log2_rows, m - j0), t0 = L - m + j0;
    const int32_t *table = p.block_table + (int64_t)r * p.max_pages_per_req;
    if (tid < n) s_page[tid] = table[(t0 + tid) >> p.log2P];
    // a request with a bad page among its new positions is skipped as a whole: every one of its blocks looks at all of them
    int bad = 0;
    for (int i = ((L - m) >> p.log2P) + tid; i <= (L - 1) >> p.log2P; i += kAppendThreads) {
      const int pg = table[i];
      bad |= pg < 0 || pg >= p.num_pages;
    }
    if constexpr (kRope) {
      const int half = p.D >> 1;
      for (int i = tid; i < n * half; i += kAppendThreads) {
        const int row = i / half, pair = i % half;
        const int t = ax.axes ? ax.positions[(int64_t)ax.axis_of[pair] * ax.position_stride + q0 + j0 + row] : t0 + row;
        double c, sn;
        sincos((double)t * s_inv_freq[pair], &sn, &c);
        if (p.elem_size == 4) {
          s_cs[row * half + (pair & 3) * (half >> 2) + (pair >> 2)] = make_double2(c, sn);
        } else {
          float *at = reinterpret_cast<float *>(s_cs + row * half + (pair & 6) * (half >> 3) + (pair >> 3)) + (pair & 1);
          const float ch = (float)c, sh = (float)sn;
          at[0] = ch; at[2] = (float)(c - (double)ch);
          at += (half >> 3) * 4;
          at[0] = sh; at[2] = (float)(sn - (double)sh);
        }
      }
    }
    if (__syncthreads_or(bad)) {
      if (tid == 0) atomicOr(p.dev_status, SPX_DEV_BAD_PAGE);
      return;
    }
    const int row_bytes = p.D * p.elem_size, vecs = row_bytes >> 4;
    auto cache_at = [&](int row, int g) -> int64_t {
      return ((int64_t)s_page[row] * p.stride_page + (int64_t)g * p.stride_head + (int64_t)((t0 + row) & (p.P - 1)) * p.stride_token) * p.elem_size;
    };
    if constexpr (kRope) {
      // a thread takes one vector of the first half of a head row and its partner in the second half: K's rows, then the
      // query rows (two at a time, in 114 registers: 44 us for prompts with images, against 40)
      const int half_vecs = vecs >> 1, half_bytes = row_bytes >> 1;
      const int n_k = n * p.Hkv * half_vecs, n_all = n_k + (p.q_rows ? n * p.Hq * half_vecs : 0);
      struct Task { const unsigned char *src; unsigned char *dst; int row, v; uint4 lo, hi; };
      auto open = [&](int i) -> Task {
        Task t;
        if (i < n_k) {
          t.v = i % half_vecs;
          const int jg = i / half_vecs, g = jg % p.Hkv;
          t.row = jg / p.Hkv;
          t.src = p.new_k + ((int64_t)(q0 + j0 + t.row) * p.Hkv + g) * row_bytes + t.v * 16;
          t.dst = p.k_cache + cache_at(t.row, g) + t.v * 16;
        } else {
          i -= n_k;
          t.v = i % half_vecs;
          const int jh = i / half_vecs, h = jh % p.Hq;
          t.row = jh / p.Hq;
          const int64_t at = ((int64_t)(q0 + j0 + t.row) * p.Hq + h) * row_bytes + t.v * 16;
          t.src = p.q_rows + at;
          t.dst = p.q_out + at;
        }
        t.lo = *reinterpret_cast<const uint4 *>(t.src);
        t.hi = *reinterpret_cast<const uint4 *>(t.src + half_bytes);
        return t;
      };
      auto close = [&](Task &t) {
        const double2 *cs = s_cs + t.row * (p.D >> 1);
        if (p.elem_size == 2) rope_vectors<__nv_bfloat16>(t.lo, t.hi, cs, half_vecs, t.v);
        else rope_vectors<float>(t.lo, t.hi, cs, half_vecs, t.v);
        *reinterpret_cast<uint4 *>(t.dst) = t.lo;
        *reinterpret_cast<uint4 *>(t.dst + half_bytes) = t.hi;
      };
      for (int i = tid; i < n_all; i += kAppendThreads) {
        Task t = open(i);
        close(t);
      }
    }
    for (int i = tid; i < n * p.Hkv * vecs; i += kAppendThreads) {
      const int v = i % vecs, jg = i / vecs, g = jg % p.Hkv, row = jg / p.Hkv;
      const int64_t src = ((int64_t)(q0 + j0 + row) * p.Hkv + g) * row_bytes + v * 16, dst = cache_at(row, g) + v * 16;
      if (!kRope) *reinterpret_cast<uint4 *>(p.k_cache + dst) = __ldg(reinterpret_cast<const uint4 *>(p.new_k + src));
      *reinterpret_cast<uint4 *>(p.v_cache + dst) = __ldg(reinterpret_cast<const uint4 *>(p.new_v + src));
    }
  };
  for (int w = 0; w < kAppendThreads / 32; ++w) {
    for (uint32_t claims = s_claims[w]; claims; claims &= claims - 1) {
      append(s_first + 32 * w + __ffs(claims) - 1);
      __syncthreads();   // page ids and angles are read
    }
  }
}

__global__ void kv_rollback_kernel(int32_t batch, const int32_t *seq_lens, const int32_t *q_indptr,
                                   const int32_t *accepted_len, int32_t *new_seq_lens, int32_t *dev_status) {
  const int r = blockIdx.x * blockDim.x + threadIdx.x;
  if (r >= batch) return;
  const int k = q_indptr[r + 1] - q_indptr[r] - 1;
  const int n = accepted_len[r];
  const int L = seq_lens[r];
  if (k < 0 || n < 0 || n > k || L < k + 1) {
    atomicOr(dev_status, SPX_DEV_BAD_LEN);
    new_seq_lens[r] = -1;
    return;
  }
  new_seq_lens[r] = L - (k - n);
}

}  // namespace spx
