// Rows worked on by groups of warps: packs of elements, and sums over a group.
#pragma once

#include "common.cuh"

namespace camera {

template <typename T, int W> struct alignas(sizeof(T) * W) Pack { T v[W]; };

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Sums over the warps that share a row; every thread gets them.  The buffers alternate, so one barrier a call is enough:
// a buffer is written again only after the barrier of the call between.
template <int K>
__device__ __forceinline__ void group_sum(float (&v)[K], int warps, int group, int& buf) {
  __shared__ float red[2][32][K];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if (warps == 1) return;
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) red[buf][warp][k] = v[k];
  }
  asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * warps) : "memory");
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = 0.f;
  for (int i = 0; i < warps; ++i)
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] += red[buf][group * warps + i][k];
  buf ^= 1;
}

// Whether rows from p, ld elements of `size` bytes apart, all start on 16-byte boundaries.
inline bool vec_ok(const void* p, long long ld, int size) {
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld * size) % 16 == 0);
}

}  // namespace camera
