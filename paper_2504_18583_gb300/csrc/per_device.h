// What a process works out once for each of its devices.
#pragma once

#include <cuda_runtime.h>

#include <atomic>

namespace pard {

constexpr int kMaxDevices = 64;

inline int current_device() {
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) throw e;
  if (dev < 0 || dev >= kMaxDevices) throw cudaErrorInvalidDevice;
  return dev;
}

// A whole number above 0 that f() gives on the current device; f is called once
// a device (twice if two threads come first at once) and throws what goes wrong.
// Function attributes belong to the current device too: f may set them.
class OncePerDevice {
  std::atomic<int> value_[kMaxDevices] = {};

 public:
  template <typename F>
  int get(int dev, F&& f) {
    int v = value_[dev].load(std::memory_order_acquire);
    if (v == 0) value_[dev].store(v = f(), std::memory_order_release);
    return v;
  }
};

// Allows `kernel` up to `bytes` of dynamic shared memory on the current device.
template <typename K>
int allow_shared(K* kernel, int bytes) {
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) throw e;
  return bytes;
}

}  // namespace pard
