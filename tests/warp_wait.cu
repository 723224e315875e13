// Cases of a warp's bounded wait, for the tests.
#include "warp_wait.cuh"

namespace {
using namespace pard;

// Warp 0 waits; what becomes of its barrier is the case's matter.
//   0: nothing ever arrives
//   1: nothing arrives, and warp 1 raises the abort flag some milliseconds later
//   2: warp 1 arrives some milliseconds later
__global__ void wait_kernel(int which, int* answers, unsigned long long* ns) {
  __shared__ __align__(8) uint64_t bar;
  __shared__ int abort_flag;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (threadIdx.x == 0) {
    mbar_init(&bar, 1);
    abort_flag = 0;
    fence_barrier_init();
  }
  __syncthreads();
  const unsigned long long t0 = globaltimer();
  if (warp == 0) {
    answers[lane] = warp_wait(&bar, 0, &abort_flag);
    if (lane == 0) *ns = globaltimer() - t0;
  } else if (lane == 0 && which) {
    for (int i = 0; i < 5000; ++i) __nanosleep(1000);
    if (which == 1) *(volatile int*)&abort_flag = 1; else mbar_arrive(&bar);
  }
}
}  // namespace

// answers: 32 ints, ns: one; device pointers
extern "C" int warp_wait_case(int which, int* answers, unsigned long long* ns) {
  wait_kernel<<<1, 64>>>(which, answers, ns);
  return (int)cudaDeviceSynchronize();
}
