// The tree operators' host side on a CUDA runtime that is made up here: two
// devices, on which nothing runs.  Linked with the library's own objects.  It
// checks that whatever a launch needs has been set and asked on its own device.
#include <cuda.h>
#include <cuda_runtime_api.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <string>
#include <utility>

#include "pard.h"

namespace {
int g_device = 0, g_asked = 0, g_fail_occupancy = 0;
std::map<std::pair<int, const void*>, int> g_allowed;  // dynamic shared memory of a kernel on a device
int g_launches = 0;
unsigned g_grid = 0;
std::string g_error;

CUresult encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
  return CUDA_SUCCESS;
}
void check(bool ok, const char* what) {
  if (ok) return;
  printf("wrong: %s (%s)\n", what, g_error.c_str());
  exit(1);
}
}  // namespace

extern "C" {
cudaError_t CUDARTAPI cudaGetDevice(int* d) { *d = g_device; return cudaSuccess; }
cudaError_t CUDARTAPI cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int dev) { *v = dev ? 20 : 100; return cudaSuccess; }
cudaError_t CUDARTAPI cudaFuncSetAttribute(const void* f, cudaFuncAttribute a, int v) {
  if (a == cudaFuncAttributeMaxDynamicSharedMemorySize) g_allowed[{g_device, f}] = v;
  return cudaSuccess;
}
cudaError_t CUDARTAPI cudaOccupancyMaxActiveClusters(int* n, const void* f, const cudaLaunchConfig_t* c) {
  ++g_asked;
  if (g_fail_occupancy && --g_fail_occupancy == 0) return cudaErrorUnknown;
  if (c->dynamicSmemBytes > 48 * 1024 && g_allowed[{g_device, f}] < (int)c->dynamicSmemBytes) return cudaErrorInvalidValue;
  // device 0 holds as many clusters of any size, device 1 many of one CTA only
  *n = g_device == 0 || c->gridDim.x == 1 ? 64 : 1;
  return cudaSuccess;
}
cudaError_t CUDARTAPI cudaLaunchKernelExC(const cudaLaunchConfig_t* c, const void* f, void**) {
  if (c->dynamicSmemBytes > 48 * 1024 && g_allowed[{g_device, f}] < (int)c->dynamicSmemBytes) return cudaErrorInvalidValue;
  ++g_launches;
  g_grid = c->gridDim.x;
  return cudaSuccess;
}
const char* CUDARTAPI cudaGetErrorString(cudaError_t) { return "refused by the made-up runtime"; }
cudaError_t CUDARTAPI cudaGetDriverEntryPointByVersion(const char*, void** p, unsigned, unsigned long long, cudaDriverEntryPointQueryResult* q) {
  *p = reinterpret_cast<void*>(&encode);
  *q = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}
void** __cudaRegisterFatBinary(void*) { static void* h; return &h; }
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
unsigned __cudaPopCallConfiguration(dim3*, dim3*, size_t*, void*) { return 1; }
cudaError_t __cudaGetKernel(cudaKernel_t*, const void*) { return cudaErrorUnknown; }
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void**, size_t, cudaStream_t) { return cudaErrorUnknown; }
}

namespace pard {
void set_error(const std::string& m) { g_error = m; }
}

int main() {
  alignas(16) static uint8_t any[64];
  auto* i32 = reinterpret_cast<int32_t*>(any);
  auto* f32 = reinterpret_cast<float*>(any);
  auto sample = [&](int vocab) {
    return pard_sample(any, vocab, PARD_F32, 464, vocab, f32, nullptr, nullptr, nullptr, nullptr, i32, f32, nullptr);
  };
  auto attend = [&] {
    return pard_tree_attention(any, 8 * 128, PARD_BF16, 2, 5, 8, 2, 128, any, any, 2 * 16 * 128, 4, i32, 4, i32, i32,
                               reinterpret_cast<uint64_t*>(any), 0.1f, any, any, size_t(1) << 30, nullptr);
  };
  unsigned attention_grid[2], sample_grid[2];
  for (int round = 0; round < 2; ++round)
    for (int dev = 0; dev < 2; ++dev) {
      g_device = dev;
      const int before = g_launches;
      check(attend() == PARD_OK, "an attention launch");
      attention_grid[dev] = g_grid;
      check(sample(40000) == PARD_OK, "a sampling launch");
      sample_grid[dev] = g_grid;
      check(g_launches == before + 2, "the launches' number");
    }
  check(attention_grid[0] == 100 && attention_grid[1] == 20, "one CTA a multiprocessor of the call's device");
  check(sample_grid[0] > 464 && sample_grid[1] == 464, "clusters by what the call's device holds");
  // what is known of the last vocabulary is not asked again; a question that fails spoils nothing
  check(sample(40000) == PARD_OK, "sampling");
  int asked = g_asked;
  check(sample(40000) == PARD_OK && g_asked == asked, "an answer kept");
  g_fail_occupancy = 3;
  check(sample(50000) == PARD_ERR_CUDA, "an error of the occupancy query");
  asked = g_asked;
  check(sample(40000) == PARD_OK && g_asked > asked && g_grid == 464, "a table taken again after an error");
  puts("right");
  return 0;
}
