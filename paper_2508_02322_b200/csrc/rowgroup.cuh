// Rows worked on by groups of warps: packs of elements, and sums over a group.
#pragma once

#include "common.cuh"

namespace camera {

// W elements of a row as they lie in memory, loaded and stored at once.  bf16 pairs stay words: taken apart into 16-bit
// elements each would hold a register of its own.
template <typename T, int W> struct Pack;
template <int W> struct alignas(4 * W) Pack<float, W> {
  float v[W];
  __device__ __forceinline__ void get(float (&f)[W]) const {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = v[i];
  }
  __device__ __forceinline__ void set(const float (&f)[W]) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] = f[i];
  }
};
template <int W> struct alignas(2 * W) Pack<__nv_bfloat16, W> {
  static_assert(W % 2 == 0, "pairs");
  uint32_t v[W / 2];
  __device__ __forceinline__ void get(float (&f)[W]) const {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
      f[2 * i] = __uint_as_float(v[i] << 16);
      f[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[W]) {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
      const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      v[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
  }
};
template <> struct Pack<__nv_bfloat16, 1> {
  uint16_t v;
  __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = __uint_as_float((uint32_t)v << 16); }
  __device__ __forceinline__ void set(const float (&f)[1]) { v = __bfloat16_as_ushort(__float2bfloat16_rn(f[0])); }
};

// Two fp32 in a register pair, worked on by one instruction.
struct F2 { unsigned long long v; };
__device__ __forceinline__ F2 f2(float lo, float hi) {
  F2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void split(F2 a, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(a.v)); }
__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 mul2(F2 a, F2 b) {
  F2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) {
  F2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
  return r;
}
// N packs of W elements as pairs, and back.
template <typename P, int W, int N>
__device__ __forceinline__ void to_pairs(const P (&p)[N], F2 (&out)[N * W / 2]) {
  float f[N * W];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float g[W];
    p[j].get(g);
#pragma unroll
    for (int i = 0; i < W; ++i) f[j * W + i] = g[i];
  }
#pragma unroll
  for (int i = 0; i < N * W / 2; ++i) out[i] = f2(f[2 * i], f[2 * i + 1]);
}
template <typename P, int W, int N>
__device__ __forceinline__ void from_pairs(const F2 (&in)[N * W / 2], P (&p)[N]) {
  float f[N * W];
#pragma unroll
  for (int i = 0; i < N * W / 2; ++i) split(in[i], f[2 * i], f[2 * i + 1]);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    float g[W];
#pragma unroll
    for (int i = 0; i < W; ++i) g[i] = f[j * W + i];
    p[j].set(g);
  }
}

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

// Whether rows from p, ld elements of `size` bytes apart, all start on boundaries of `unit` bytes.
inline bool rows_on(const void* p, long long ld, int size, int unit) {
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) & (uintptr_t)(unit - 1)) == 0;
}
// How a call's rows can be accessed: 16 bytes at a time, two elements, or one.
enum { BY_16 = 0, BY_TWO = 1, BY_ONE = 2 };

}  // namespace camera
