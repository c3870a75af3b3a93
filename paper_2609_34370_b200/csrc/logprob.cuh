// Log-probabilities of given tokens, row entropies and top alternatives.
#pragma once
#include "common.cuh"

namespace spx {

struct LogprobParams {
  int32_t rows, vocab, top_n;
  int64_t row_stride;
  const void *logits;
  const int32_t *token_ids;
  float *logprobs, *entropy, *top_logprobs;
  int32_t *top_ids;
  int32_t *dev_status;
};

constexpr int kLogprobThreads = 256;

// Order of the alternatives, as an unsigned key: larger logits first, equal ones (-0 and +0 too) alike,
// NaN above +inf.
__device__ __forceinline__ uint32_t logit_key(float x) {
  if (x != x) return 0xffffffffu;
  const uint32_t u = __float_as_uint(x + 0.f);   // -0 becomes +0
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// One block per row.
template <typename T>
__global__ void __launch_bounds__(kLogprobThreads) logprob_kernel(LogprobParams p) {
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  __shared__ float s_max[kLogprobThreads / 32];
  __shared__ double s_a[kLogprobThreads / 32], s_b[kLogprobThreads / 32];
  __shared__ int s_n[kLogprobThreads / 32];
  __shared__ unsigned long long s_k[kLogprobThreads / 32];
  const int tok = p.token_ids ? p.token_ids[row] : 0;
  const float nan = __int_as_float(0x7fc00000);
  if (tok < 0 || tok >= p.vocab) {
    if (tid == 0) {
      if (p.logprobs) p.logprobs[row] = nan;
      if (p.entropy) p.entropy[row] = nan;
      if (tok != -1) atomicOr(p.dev_status, SPX_DEV_BAD_TOKEN);
    }
    if (tid < p.top_n) {
      if (p.top_ids) p.top_ids[(int64_t)row * p.top_n + tid] = -1;
      if (p.top_logprobs) p.top_logprobs[(int64_t)row * p.top_n + tid] = nan;
    }
    return;
  }
  const T *x = reinterpret_cast<const T *>(p.logits) + row * p.row_stride;
  float m = -INFINITY;
  for (int v = tid; v < p.vocab; v += kLogprobThreads) m = fmaxf(m, ld_as_float(x, v));
  m = warp_max(m);
  if (lane == 0) s_max[warp] = m;
  __syncthreads();
  for (int w = 0; w < kLogprobThreads / 32; ++w) m = fmaxf(m, s_max[w]);
  double z = 0.0, s = 0.0;   // sum of e^(x - m) without the m's own ones, sum of e^(x - m) (x - m)
  int n_max = 0;
  for (int v = tid; v < p.vocab; v += kLogprobThreads) {
    const float d = ld_as_float(x, v) - m;
    if (d == 0.f) { ++n_max; continue; }
    const float e = expf(d);
    z += e;
    if (!(e == 0.f)) s += (double)e * d;
  }
  n_max = __reduce_add_sync(0xffffffffu, n_max);
  for (int o = 16; o > 0; o >>= 1) { z += __shfl_xor_sync(0xffffffffu, z, o); s += __shfl_xor_sync(0xffffffffu, s, o); }
  if (lane == 0) { s_a[warp] = z; s_b[warp] = s; s_n[warp] = n_max; }
  __syncthreads();
  z = 0.0; s = 0.0; n_max = -1;   // the largest logit's own 1 is left to log1p
  for (int w = 0; w < kLogprobThreads / 32; ++w) { z += s_a[w]; s += s_b[w]; n_max += s_n[w]; }
  z += n_max;
  const double log_z = log1p(z);
  if (tid == 0) {
    if (p.logprobs) p.logprobs[row] = (float)((double)ld_as_float(x, tok) - m - log_z);
    if (p.entropy) p.entropy[row] = (float)(log_z - s / (1.0 + z));
  }
  unsigned long long last = ~0ull;   // (key, ~id) of the alternative before
  for (int j = 0; j < p.top_n; ++j) {
    unsigned long long best = 0;
    for (int v = tid; v < p.vocab; v += kLogprobThreads) {
      const unsigned long long c = ((unsigned long long)logit_key(ld_as_float(x, v)) << 32) | (uint32_t)~v;
      if (c < last && c > best) best = c;
    }
    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    __syncthreads();
    if (lane == 0) s_k[warp] = best;
    __syncthreads();
    for (int w = 0; w < kLogprobThreads / 32; ++w) best = max(best, s_k[w]);
    last = best;
    const int id = best ? (int)~(uint32_t)best : -1;
    if (tid == 0) {
      if (p.top_ids) p.top_ids[(int64_t)row * p.top_n + j] = id;
      if (p.top_logprobs) p.top_logprobs[(int64_t)row * p.top_n + j] = id < 0 ? nan : (float)((double)ld_as_float(x, id) - m - log_z);
    }
  }
}

}  // namespace spx
