// Cache maintenance around the verify step: append the new positions' K/V into their pages,
// shrink the lengths by the rejected drafts afterwards.
#pragma once
#include "common.cuh"

namespace spx {

constexpr int kRopeMaxHeadDim = 512;
constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 16;         // new rows of a block, at most
constexpr int kAppendAngles = 1024;     // (row, pair) angles a block keeps: 16 rows of 128 elements, 4 of 512

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
  // positions of several axes (axes = 0: a row's position is its place in the request)
  int32_t axes;
  const int32_t *positions;
  int64_t position_stride;
  unsigned char axis_of[kRopeMaxHeadDim / 2];
};

// Rotary embedding of the pairs (x[i], x[i + D/2]) of one head vector: x in double, cosine and sine of the pair's
// angle in double; results rounded double -> binary32 -> element type (round-to-nearest-even each).  lo / hi are the
// 16-byte vectors that hold the pairs' first and second elements, cs the (cos, sin) of the first.
template <typename T>
__device__ __forceinline__ void rope_vectors(uint4 &lo, uint4 &hi, const double2 *cs) {
  constexpr int N = 16 / sizeof(T);
  union U { uint4 q; T e[N]; } a, b;
  a.q = lo; b.q = hi;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const double2 k = cs[u];
    const double x0 = (double)ld_as_float(a.e, u), x1 = (double)ld_as_float(b.e, u);
    st_from_float(a.e, u, __double2float_rn(x0 * k.x - x1 * k.y));
    st_from_float(b.e, u, __double2float_rn(x1 * k.x + x0 * k.y));
  }
  lo = a.q; hi = b.q;
}

// A block takes up to kAppendRows new rows of a request, all heads of K, V and the query rows, 16 bytes a thread and step.
// Block b belongs to the request r with base(r) <= b < base(r + 1), base(r) = q_indptr[r] / rows + r: m rows are at most
// m / rows + 1 blocks, so no prefix sums are needed; blocks past a request's last one leave at once.  The angles are
// worked out once a block and shared by its heads.
// Pure copy and rotation: bound by launch latency at verify-step sizes (a few MB), by HBM beyond that.
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(const __grid_constant__ KvAppendParams p) {
  __shared__ int s_req, s_page[kAppendRows];
  __shared__ double s_inv_freq[kRopeMaxHeadDim / 2];
  __shared__ __align__(16) double2 s_cs[kAppendAngles];
  const int tid = threadIdx.x, lane = tid & 31;
  const bool rope = p.rope_base > 0.0;
  if (tid < 32) {
    // 32 probes at a time
    int lo = 0, hi = p.batch;   // base(lo) <= block, hi past the last candidate
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, c = lo + lane * step;
      const bool below = c < hi && (int64_t)(p.q_indptr[c] >> p.log2_rows) + c <= (int64_t)blockIdx.x;
      const int n = __popc(__ballot_sync(0xffffffffu, below || lane == 0));   // the probes ascend
      const int at = lo + (n - 1) * step;
      hi = min(hi, at + step);
      lo = at;
    }
    if (lane == 0) s_req = lo;
  } else if (rope) {
    for (int i = tid - 32; i < (p.D >> 1); i += kAppendThreads - 32) s_inv_freq[i] = pow(p.rope_base, -2.0 * (double)i / (double)p.D);
  }
  __syncthreads();
  const int r = s_req;
  const int q0 = p.q_indptr[r];
  const int m = p.q_indptr[r + 1] - q0;
  const int L = p.seq_lens[r];
  const bool ok_len = m >= 1 && L >= m && q0 >= 0 && m <= p.total_q - q0 &&
                      (((int64_t)L + p.P - 1) >> p.log2P) <= (int64_t)p.max_pages_per_req;
  if (!ok_len) {
    if (tid == 0) atomicOr(p.dev_status, SPX_DEV_BAD_LEN);
    return;
  }
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
  if (rope) {
    const int half = p.D >> 1;
    for (int i = tid; i < n * half; i += kAppendThreads) {
      const int row = i / half, pair = i % half;
      const int t = p.axes ? p.positions[(int64_t)p.axis_of[pair] * p.position_stride + q0 + j0 + row] : t0 + row;
      double2 cs;
      sincos((double)t * s_inv_freq[pair], &cs.y, &cs.x);
      s_cs[i] = cs;
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
  if (rope) {
    // a thread takes one vector of the first half of a head row and its partner in the second half
    const int half_vecs = vecs >> 1, per_vec = 16 / p.elem_size, half_bytes = row_bytes >> 1;
    auto turn = [&](const unsigned char *src, unsigned char *dst, int row, int v) {
      uint4 lo = *reinterpret_cast<const uint4 *>(src), hi = *reinterpret_cast<const uint4 *>(src + half_bytes);
      const double2 *cs = s_cs + row * (p.D >> 1) + v * per_vec;
      if (p.elem_size == 2) rope_vectors<__nv_bfloat16>(lo, hi, cs);
      else rope_vectors<float>(lo, hi, cs);
      *reinterpret_cast<uint4 *>(dst) = lo;
      *reinterpret_cast<uint4 *>(dst + half_bytes) = hi;
    };
    for (int i = tid; i < n * p.Hkv * half_vecs; i += kAppendThreads) {
      const int v = i % half_vecs, jg = i / half_vecs, g = jg % p.Hkv, row = jg / p.Hkv;
      turn(p.new_k + ((int64_t)(q0 + j0 + row) * p.Hkv + g) * row_bytes + v * 16, p.k_cache + cache_at(row, g) + v * 16, row, v);
    }
    if (p.q_rows)
      for (int i = tid; i < n * p.Hq * half_vecs; i += kAppendThreads) {
        const int v = i % half_vecs, jh = i / half_vecs, h = jh % p.Hq, row = jh / p.Hq;
        const int64_t at = ((int64_t)(q0 + j0 + row) * p.Hq + h) * row_bytes + v * 16;
        turn(p.q_rows + at, p.q_out + at, row, v);
      }
  }
  for (int i = tid; i < n * p.Hkv * vecs; i += kAppendThreads) {
    const int v = i % vecs, jg = i / vecs, g = jg % p.Hkv, row = jg / p.Hkv;
    const int64_t src = ((int64_t)(q0 + j0 + row) * p.Hkv + g) * row_bytes + v * 16, dst = cache_at(row, g) + v * 16;
    if (!rope) *reinterpret_cast<uint4 *>(p.k_cache + dst) = __ldg(reinterpret_cast<const uint4 *>(p.new_k + src));
    *reinterpret_cast<uint4 *>(p.v_cache + dst) = __ldg(reinterpret_cast<const uint4 *>(p.new_v + src));
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
