// Diagnostic kernel of the failure-reporting path (not on any product path).
#pragma once

#include "gemm_tc.cuh"

namespace sgc {

// Diagnostic kernel (one CTA): thread 0 waits, with the bounded wait that every role of the
// kernels above uses, on an mbarrier that nothing ever signals, so the wait runs into its clock
// limit, publishes kErrProbeWait in the error word and raises the CTA's abort flag; the second
// warp waits on the same barrier with the full limit and must leave as soon as the flag is up.
// Lets a test walk the path device wait -> error word -> host status without making any real
// pipeline fail.  `limit` is a few thousand clocks.
__global__ void wait_timeout_probe_kernel(unsigned int* err, long long limit) {
  __shared__ uint64_t bar;
  __shared__ uint32_t abort_flag;
  if (threadIdx.x == 0) {
    mbar_init(&bar, 1);
    abort_flag = 0u;
    fence_mbar_init();
  }
  __syncthreads();
  if (threadIdx.x == 0) mbar_wait_bounded(&bar, 0, &abort_flag, err, kErrProbeWait, 0u, limit);
  if (threadIdx.x == 32) mbar_wait_bounded(&bar, 0, &abort_flag, err, kErrProbeWait + 1, 0u, kWaitLimitClocks);
}

}  // namespace sgc
