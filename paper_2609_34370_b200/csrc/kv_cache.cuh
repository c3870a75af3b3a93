// Cache maintenance around the verify step: append the new positions' K/V into their pages,
// shrink the lengths by the rejected drafts afterwards.
#pragma once
#include <type_traits>

#include "common.cuh"
#include "rotate.cuh"

namespace spx {

constexpr int kRopeMaxHeadDim = 512;
constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 8;          // new rows of a step, at most
constexpr int kAppendVote = 1024;       // requests that the threads of a block look at in one go
constexpr int kAppendBlocks = 2048;     // blocks behind the requests' own that a call is cut into, at most
constexpr int kAppendAngles = 1024;     // (row, pair) angles a step keeps: 8 rows of 256 elements, 4 of 512

struct KvAppendParams {
  int32_t batch, total_q, Hkv, D, P, log2P, num_pages, max_pages_per_req, elem_size;
  int32_t log2_rows;       // new rows of a step
  int32_t log2_block;      // ... and of a block
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
// Positions of several axes; without, a row's position is its place in the request.
struct KvAppendAxes {
  const int32_t *positions;
  int64_t position_stride;
  unsigned char axis_of[kRopeMaxHeadDim / 2];
};
struct KvNoAxes {};

// A pair (x0, x1) turned by an angle in float64: y0 and y1 rounded to binary32 and to bfloat16, in the low and the high half.
// (Out of line: a few in a thousand vectors come here.)
static __device__ __noinline__ uint32_t rope_pair_exact(float x0, float x1, double angle) {
  double c, sn;
  sincos(angle, &sn, &c);
  const double a = (double)x0, b = (double)x1;
  const __nv_bfloat16 y0 = __float2bfloat16_rn(__double2float_rn(a * c - b * sn)), y1 = __float2bfloat16_rn(__double2float_rn(b * c + a * sn));
  return (uint32_t)*reinterpret_cast<const uint16_t *>(&y0) | (uint32_t)*reinterpret_cast<const uint16_t *>(&y1) << 16;
}

// Rotary embedding of the pairs (x[i], x[i + D/2]) of one head vector by angles whose cosine and sine are float64's; products and sum in
// float64, results rounded to binary32 and then to the element type (nearest even each).  lo / hi are the 16-byte vectors that
// hold the pairs' first and second elements.  cs: the angles of a row, 16 bytes a pair, laid out so that neighbouring vectors' lie side by
// side, vecs vectors to half a row.
//   float32 rows: (cos, sin) of vector v's pair u at [u * vecs + v].
//   16-bit rows: (cos, cos', low parts) of pairs 2u, 2u + 1 at [2u * vecs + v], the sines at [(2u + 1) * vecs + v].  Products and sum in
//   pairs of binary32 (conversions from and to float64 take 8 cycles each).  With X = max(|x0|, |x1|), y is off by the roundings of x0 cos - x1 sin
//   and of the last sum, half a last bit each, and by 2^-46 X beside them.  Where |y| > 2^-18 X that is 1.6 of y's last bits at most (a
//   last bit of the first may be two of y's), so that float64's result rounded to binary32 is at most two away, and rounds to another
//   bfloat16 only if y's lower half is within two of 0x8000.  Those pairs, the ones that cancel further, tiny ones and what is
//   not finite (6 in 100 warps' vectors) are made again in float64, angle(i) being that of the vector's pair i: results are
//   float64's, to the last bit and to the sign of a zero.
template <typename T, typename Angle>
__device__ __forceinline__ void rope_vectors(uint4 &lo, uint4 &hi, const double2 *cs, int vecs, int v, Angle angle) {
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
    const uint32_t x[4] = {lo.x, lo.y, lo.z, lo.w}, y[4] = {hi.x, hi.y, hi.z, hi.w};
    uint32_t a[4], b[4], again = 0;            // bit u: pairs 2u and 2u + 1
    uint64_t finite = e8::pair(0.f, 0.f);      // stays zero as long as results are finite
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const ulonglong2 c = at[2 * u * vecs + v], s = at[(2 * u + 1) * vecs + v];
      const CosSin k{c.x, c.y, s.x, s.y};
      const float x0 = __uint_as_float(x[u] << 16), x1 = __uint_as_float(x[u] & 0xffff0000u), y0 = __uint_as_float(y[u] << 16), y1 = __uint_as_float(y[u] & 0xffff0000u);
      uint64_t r0, r1;
      rotate2<false>(e8::pair(x0, x1), e8::pair(y0, y1), k, r0, r1);
      finite = e8::fma2(r0, e8::pair(0.f, 0.f), e8::fma2(r1, e8::pair(0.f, 0.f), finite));
      float p, q, r, t;
      e8::unpair(r0, p, q);
      e8::unpair(r1, r, t);
      // the lower halves plus 0x8004, two in a word (a carry moves the upper one by one): below 8 if they were 0x7ffe .. 0x8002
      const uint32_t half = __vminu2(__byte_perm(__float_as_uint(p), __float_as_uint(q), 0x5410) + 0x80048004u,
                                     __byte_perm(__float_as_uint(r), __float_as_uint(t), 0x5410) + 0x80048004u);
      const float least = fminf(fminf(fabsf(p), fabsf(q)), fminf(fabsf(r), fabsf(t)));
      const float most = fmaxf(fmaxf(fmaxf(fabsf(x0), fabsf(x1)), fmaxf(fabsf(y0), fabsf(y1))), 0x1p-82f);
      if ((half & 0xfff8u) == 0 || (half & 0xfff80000u) == 0 || !(least * 0x1p18f > most)) again |= 1u << u;
      const __nv_bfloat162 h0 = __floats2bfloat162_rn(p, q), h1 = __floats2bfloat162_rn(r, t);
      a[u] = *reinterpret_cast<const uint32_t *>(&h0); b[u] = *reinterpret_cast<const uint32_t *>(&h1);
    }
    float p, q;
    e8::unpair(finite, p, q);
    if (p != 0.f || q != 0.f) again = 15;
    if (again) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (!(again >> u & 1)) continue;
        const uint32_t even = rope_pair_exact(__uint_as_float(x[u] << 16), __uint_as_float(y[u] << 16), angle(2 * u));
        const uint32_t odd = rope_pair_exact(__uint_as_float(x[u] & 0xffff0000u), __uint_as_float(y[u] & 0xffff0000u), angle(2 * u + 1));
        a[u] = __byte_perm(even, odd, 0x5410);
        b[u] = __byte_perm(even, odd, 0x7632);
      }
    }
    lo = make_uint4(a[0], a[1], a[2], a[3]); hi = make_uint4(b[0], b[1], b[2], b[3]);
  }
}

// A block takes 1 << log2_block new rows of a request, up to kAppendRows a step, all heads of K, V and the query rows, 16 bytes a thread at a time.
// Block r < batch takes the first rows of request r: in a verify step nearly all there are, with no search for whose rows they are
// (64 requests of 6 rows, 8 heads of 128: 3.0 us with one, 2.6 without), and whatever the other requests' bounds are.  What a request has beyond is for the blocks behind:
// its rows from j << log2_block on, j > 0, are those of block batch + (q_indptr[r] >> log2_block) + j - 1, which is below
// batch + (q_indptr[r + 1] >> log2_block), so that no prefix sums are needed.  Blocks that are nobody's leave at once.  The angles are worked out once a
// step and shared by its heads.
// Pure copy and rotation: bound by launch latency at verify-step sizes (a few MB), by HBM beyond that.
// kRope: with a rotary base (without, a kernel of fewer registers).  Eight rows a step, three blocks per SM: five prompts with images 39 us
// (16 rows, two vectors a thread in flight, four blocks: slower each).
template <bool kRope, typename Axes>
__global__ void __launch_bounds__(kAppendThreads, kRope ? 3 : 4)
kv_append_kernel(const __grid_constant__ KvAppendParams p, const __grid_constant__ Axes ax) {
  __shared__ int s_page[kAppendRows];
  __shared__ int4 s_whose;                 // a request and its bounds
  __shared__ double s_inv_freq[kRope ? kRopeMaxHeadDim / 2 : 1];
  __shared__ __align__(16) double2 s_cs[kRope ? kAppendAngles : 1];
  const int tid = threadIdx.x, rows = 1 << p.log2_rows;
  const bool head = blockIdx.x < (unsigned)p.batch;
  const int chunk = (int)blockIdx.x - p.batch;
  auto valid = [&](int q0, int q1, int L) -> bool {
    return q0 >= 0 && q1 > q0 && q1 <= p.total_q && L >= q1 - q0 && (((int64_t)L + p.P - 1) >> p.log2P) <= (int64_t)p.max_pages_per_req;
  };
  // first of the block's rows of a request
  auto first_row = [&](int q0) -> int64_t { return head ? 0 : ((int64_t)chunk - (q0 >> p.log2_block) + 1) << p.log2_block; };
  auto takes_part = [&](int q0, int q1, int L) -> bool {
    const int64_t first = first_row(q0);
    return valid(q0, q1, L) && (head || first > 0) && first < q1 - q0;
  };
  int r = blockIdx.x, q0 = 0, q1 = 0, L = 0;
  if (head) { q0 = p.q_indptr[r]; q1 = p.q_indptr[r + 1]; L = p.seq_lens[r]; }
  uint32_t mine = 0;      // bit u: request tid + u * kAppendThreads has rows of this block
  if (!head) {
    if (p.batch <= kAppendVote) {
      // each thread looks whether the rows are its own requests', in one memory round trip
      int a[kAppendVote / kAppendThreads][3];
#pragma unroll
      for (int u = 0; u < kAppendVote / kAppendThreads; ++u) {
        const int c = tid + u * kAppendThreads;
        a[u][0] = -1; a[u][1] = a[u][2] = 0;
        if (c < p.batch) { a[u][0] = p.q_indptr[c]; a[u][1] = p.q_indptr[c + 1]; a[u][2] = p.seq_lens[c]; }
      }
#pragma unroll
      for (int u = 0; u < kAppendVote / kAppendThreads; ++u)
        if (takes_part(a[u][0], a[u][1], a[u][2])) {
          s_whose = make_int4(mine ? -1 : tid + u * kAppendThreads, a[u][0], a[u][1], a[u][2]);
          mine |= 1u << u;
        }
    } else if (tid < 32) {
      // the last request that starts at or before the block's rows, 32 probes at a time.  (Where q_indptr descends somewhere this may
      // miss a request, whose rows behind its first block's then stay out.)
      int lo = 0, hi = p.batch;
      while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, c = lo + tid * step;
        const bool below = c < hi && (p.q_indptr[c] >> p.log2_block) <= chunk;
        const int n = __popc(__ballot_sync(0xffffffffu, below || tid == 0));   // the probes ascend
        const int at = lo + (n - 1) * step;
        hi = min(hi, at + step);
        lo = at;
      }
      if (tid == 0) { s_whose = make_int4(lo, p.q_indptr[lo], p.q_indptr[lo + 1], p.seq_lens[lo]); mine = 1; }
    }
  }
  if (kRope)
    for (int i = tid; i < (p.D >> 1); i += kAppendThreads) s_inv_freq[i] = pow(p.rope_base, -2.0 * (double)i / (double)p.D);
  bool many = false;
  if (!head) {
    const int n = __syncthreads_count(mine != 0);
    if (n == 0) return;
    const int4 w = s_whose;     // (one thread's, unless n > 1)
    many = n > 1 || w.x < 0;
    r = w.x; q0 = w.y; q1 = w.z; L = w.w;
  } else if (kRope) {
    __syncthreads();
  }
  for (;;) {
    if (many) {
      // q_indptr descends somewhere, and the rows are several requests': one after the other
      __syncthreads();
      if (mine) s_whose.x = tid + (__ffs(mine) - 1) * kAppendThreads;
      __syncthreads();
      r = s_whose.x;
      q0 = p.q_indptr[r]; q1 = p.q_indptr[r + 1]; L = p.seq_lens[r];
    }
    if (!takes_part(q0, q1, L)) {
      if (head && tid == 0) atomicOr(p.dev_status, SPX_DEV_BAD_LEN);
      return;
    }
    const int m = q1 - q0, first = (int)first_row(q0), end = (int)min((int64_t)m, (int64_t)first + (1 << p.log2_block));
    const int32_t *table = p.block_table + (int64_t)r * p.max_pages_per_req;
    // a request with a bad page among its new positions is skipped as a whole: every one of its blocks looks at all of them
    int bad = 0;
    if (m > rows) {
      for (int i = ((L - m) >> p.log2P) + tid; i <= (L - 1) >> p.log2P; i += kAppendThreads) {
        const int pg = table[i];
        bad |= pg < 0 || pg >= p.num_pages;
      }
    }
    for (int j0 = first; j0 < end; j0 += rows) {
      if (j0 > first) __syncthreads();   // the step before has read its page ids and angles
      const int n = min(rows, end - j0), t0 = L - m + j0;
      if (tid < n) {
        const int pg = table[(t0 + tid) >> p.log2P];
        s_page[tid] = pg;
        bad |= pg < 0 || pg >= p.num_pages;
      }
      auto angle = [&](int row, int pair) -> double {
        int t = t0 + row;
        if constexpr (std::is_same<Axes, KvAppendAxes>::value) t = ax.positions[(int64_t)ax.axis_of[pair] * ax.position_stride + q0 + j0 + row];
        return (double)t * s_inv_freq[pair];
      };
      if constexpr (kRope) {
        const int half = p.D >> 1;
        for (int i = tid; i < n * half; i += kAppendThreads) {
          const int row = i / half, pair = i % half;
          double c, sn;
          sincos(angle(row, pair), &sn, &c);
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
      if (j0 == first ? __syncthreads_or(bad) : (__syncthreads(), 0)) {
        if (tid == 0) atomicOr(p.dev_status, SPX_DEV_BAD_PAGE);
        break;
      }
      const int row_bytes = p.D * p.elem_size, vecs = row_bytes >> 4;
      auto cache_at = [&](int row, int g) -> int64_t {
        return ((int64_t)s_page[row] * p.stride_page + (int64_t)g * p.stride_head + (int64_t)((t0 + row) & (p.P - 1)) * p.stride_token) * p.elem_size;
      };
      if constexpr (kRope) {
        // a thread takes one vector of the first half of a head row and its partner in the second half: K's rows, then the
        // query rows (two at a time, in 114 registers: 44 us for prompts with images, where this took 40)
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
          auto of_pair = [&](int i) -> double { return angle(t.row, t.v * 8 + i); };
          if (p.elem_size == 2) rope_vectors<__nv_bfloat16>(t.lo, t.hi, cs, half_vecs, t.v, of_pair);
          else rope_vectors<float>(t.lo, t.hi, cs, half_vecs, t.v, of_pair);
          *reinterpret_cast<uint4 *>(t.dst) = t.lo;
          *reinterpret_cast<uint4 *>(t.dst + half_bytes) = t.hi;
        };
        for (int i = tid; i < n_all; i += kAppendThreads) {
          Task t = open(i);
          close(t);
        }
      }
      // V, and K without a rotation: the step's rows lie one behind the other, so that loads need no division
      const int n_copy = n * p.Hkv * vecs;
      const uint4 *ks = reinterpret_cast<const uint4 *>(p.new_k + (int64_t)(q0 + j0) * p.Hkv * row_bytes);
      const uint4 *vs = reinterpret_cast<const uint4 *>(p.new_v + (int64_t)(q0 + j0) * p.Hkv * row_bytes);
      auto store = [&](int i, uint4 x, uint4 y) {
        const int v = i % vecs, jg = i / vecs, g = jg % p.Hkv, row = jg / p.Hkv;
        const int64_t dst = cache_at(row, g) + v * 16;
        if (!kRope) *reinterpret_cast<uint4 *>(p.k_cache + dst) = x;
        *reinterpret_cast<uint4 *>(p.v_cache + dst) = y;
      };
      constexpr int kAhead = 4;
      int i = tid;
      for (; i + (kAhead - 1) * kAppendThreads < n_copy; i += kAhead * kAppendThreads) {
        uint4 x[kAhead], y[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          if (!kRope) x[u] = __ldg(ks + i + u * kAppendThreads);
          y[u] = __ldg(vs + i + u * kAppendThreads);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) store(i + u * kAppendThreads, x[u], y[u]);
      }
#pragma unroll 1
      for (; i < n_copy; i += kAppendThreads) store(i, kRope ? uint4() : __ldg(ks + i), __ldg(vs + i));
    }
    if (!many) return;
    if (r % kAppendThreads == tid) mine &= mine - 1;
    if (!__syncthreads_or(mine)) return;
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
