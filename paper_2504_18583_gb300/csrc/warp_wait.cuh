// A warp's bounded wait on an mbarrier of its CTA.
#pragma once

#include "common.cuh"

namespace pard {

__device__ __forceinline__ bool mbar_try_wait_at(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}

// What a wait does once its first try has failed: tries until kWaitLimitNs have
// passed or *abort is raised.  One copy for all places that wait, since what a CTA
// runs once comes from L2 instruction by instruction: with the timed loop inlined
// into its twenty, the tree attention of 65000-token contexts took 60.2 us instead
// of 56.8.
static __device__ __noinline__ bool keep_waiting(uint32_t bar, uint32_t parity, volatile int* abort) {
  const unsigned long long t0 = globaltimer();
  bool done;
  do done = mbar_try_wait_at(bar, parity);
  while (!done && !*abort && globaltimer() - t0 <= kWaitLimitNs);
  return done;
}

// All lanes leave with the same answer: false if the wait ran out.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  bool done = mbar_try_wait(bar, parity);
  if (!done) done = keep_waiting(smem_u32(bar), parity, abort);
  return __all_sync(0xffffffffu, done);
}

}  // namespace pard
