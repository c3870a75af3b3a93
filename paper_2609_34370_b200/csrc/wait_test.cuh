// Wait-test builds only (-DSPX_WAIT_TEST=1 with a small -DSPX_WAIT_LIMIT_CYCLES): one tiny kernel
// in which each bounded-wait helper of the library waits on a barrier that nothing ever arrives at.
// Nothing faults and nothing spins without a limit: every wait ends by its cycle limit or by the
// abort flag another role raised, the kernel returns, and the host reads what happened.
#pragma once
#include "attn_e4m3.cuh"
#include "attn_tc.cuh"
#include "lm_head.cuh"
#include "prompt_tc.cuh"
#include "sampler.cuh"

namespace spx {

// report[i]: 1 = the wait of role i returned true (must not happen), 2 = it gave up;
// report[4 + i]: clock cycles role i spent waiting.  Roles: 0 attention barrier wait (expires),
// 1 a second attention role on another barrier of the same CTA (leaves by the abort flag or its
// own limit), 2 the logits ring's wait, 3 the LM head's wait.
__global__ void __launch_bounds__(128) wait_expiry_kernel(int32_t *report, int32_t *dev_status) {
  __shared__ TcBarriers bars;
  __shared__ LmBarriers lbars;
  __shared__ uint64_t ring_bar;
  __shared__ int ring_abort;
  if (threadIdx.x == 0) {
    tc::mbar_init(&bars.k_full[0], 1);
    tc::mbar_init(&bars.v_full[0], 1);
    tc::mbar_init(&lbars.full[0], 1);
    tc::mbar_init(&ring_bar, 1);
    bars.abort = 0;
    lbars.abort = 0;
    ring_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  const int role = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0) {
    const long long t0 = clock64();
    bool got = false;
    if (role == 0) got = tc::mbar_wait(&bars.k_full[0], 0, &bars, dev_status);
    else if (role == 1) got = tc::mbar_wait(&bars.v_full[0], 0, &bars, dev_status);
    else if (role == 2) got = ring_wait(&ring_bar, 0, &ring_abort, dev_status);
    else got = lm_wait(&lbars.full[0], 0, &lbars, dev_status);
    report[role] = got ? 1 : 2;
    report[4 + role] = (int32_t)min(clock64() - t0, (long long)0x7fffffff);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    report[8] = bars.abort;
    report[9] = lbars.abort;
    report[10] = ring_abort;
  }
}

// The warp-wide waits that hand no outcome back: two warps wait on a barrier each, then each on another one.
// report[w], report[2 + w]: clock cycles warp w spent in its first and second wait; report[4]: the CTA's
// abort flag; report[5]: how many of the four waits were satisfied (must be none).
template <typename Bars, typename Wait>
__device__ __forceinline__ void two_warps_wait(Bars &bars, uint64_t *barriers, Wait wait, int32_t *report, int32_t *dev_status) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < 4; ++i) tc::mbar_init(&barriers[i], 1);
    bars.abort = 0;
    bars.dev_status = dev_status;
    report[5] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = 0; i < 2; ++i) {
    uint64_t *bar = &barriers[2 * i + warp];
    const long long t0 = clock64();
    wait(bar);
    if (lane == 0) {
      report[2 * i + warp] = (int32_t)min(clock64() - t0, (long long)0x7fffffff);
      if (e8::try_wait(tc::smem_u32(bar), 0)) atomicAdd(report + 5, 1);
    }
    __syncwarp();
  }
  __syncthreads();
  if (threadIdx.x == 0) report[4] = bars.abort;
}

// that of the attention over 8-bit pools
__global__ void __launch_bounds__(64) warp_wait_expiry_kernel(int32_t *report, int32_t *dev_status) {
  __shared__ E8Barriers bars;
  two_warps_wait(bars, bars.s_full, [&](uint64_t *bar) { e8::warp_wait(tc::smem_u32(bar), 0, &bars); }, report, dev_status);
}

// that of the attention of prompts and shared prefixes
__global__ void __launch_bounds__(64) prompt_wait_expiry_kernel(int32_t *report, int32_t *dev_status) {
  __shared__ PtBars bars;
  two_warps_wait(bars, &bars.s_full[0][0], [&](uint64_t *bar) { pt::wait(bar, 0, &bars); }, report, dev_status);
}

}  // namespace spx
