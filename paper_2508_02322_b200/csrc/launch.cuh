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

// CTAs of `threads` threads and `smem` bytes of dynamic shared memory that an SM holds of a kernel: asked of the driver, the last
// answer kept per kernel and device.
template <auto KERN>
int ctas_per_sm(int threads, int smem) {
  static std::atomic<unsigned long long> known[KNOWN_DEVICES];          // smem << 32 | threads << 8 | CTAs
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 1; }
  const unsigned long long key = (unsigned long long)smem << 32 | (unsigned)threads << 8;
  const unsigned long long seen = dev < KNOWN_DEVICES ? known[dev].load(std::memory_order_relaxed) : 0;
  if ((seen & 0xff) != 0 && (seen & ~0xffull) == key) return (int)(seen & 0xff);
  if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, KERN, threads, (size_t)smem) != cudaSuccess || n < 1) { cudaGetLastError(); return 1; }
  if (dev < KNOWN_DEVICES) known[dev].store(key | (unsigned)n, std::memory_order_relaxed);
  return n;
}

// chained: the kernel may start while the one before it in the stream ends (it waits for that itself, griddepcontrol).
template <typename A>
inline cudaError_t launch_chained(void (*kern)(A), const A& args, int grid_x, int grid_y, int cluster_y, int threads, int smem, bool chained,
                           cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid_x, (unsigned)grid_y);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (cluster_y > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = 1; at[n].val.clusterDim.y = (unsigned)cluster_y; at[n].val.clusterDim.z = 1;
    ++n;
  }
  if (chained) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = at;
  cfg.numAttrs = (unsigned)n;
  return cudaLaunchKernelEx(&cfg, kern, args);
}

}  // namespace camera
