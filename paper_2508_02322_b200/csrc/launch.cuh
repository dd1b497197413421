// What launches ask the device once: its SM count, and leave to use more than 48 KB of dynamic shared memory.
#pragma once

#include <cuda_runtime.h>

#include <atomic>

namespace camera {

constexpr int KNOWN_DEVICES = 64;      // devices whose answers are kept; later ones are asked on every call

inline int sm_count() {                // of the process's GPUs, which are all alike
  static std::atomic<int> known;
  int sms = known.load(std::memory_order_relaxed);
  if (sms == 0) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
      cudaGetLastError();
      return 148;
    }
    known.store(sms, std::memory_order_relaxed);
  }
  return sms;
}

// Lets a kernel use up to MOST bytes of dynamic shared memory: the most any of its launches takes, so that the attribute has
// one value whichever thread sets it.  Asks the driver once per kernel and device.
template <auto KERN, int MOST>
cudaError_t allow_smem() {
  static std::atomic<bool> allowed[KNOWN_DEVICES];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < KNOWN_DEVICES && allowed[dev].load(std::memory_order_relaxed)) return cudaSuccess;
  e = cudaFuncSetAttribute(KERN, cudaFuncAttributeMaxDynamicSharedMemorySize, MOST);
  if (e == cudaSuccess && dev < KNOWN_DEVICES) allowed[dev].store(true, std::memory_order_relaxed);
  return e;
}

}  // namespace camera
