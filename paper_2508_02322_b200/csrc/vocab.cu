// Operators over rows of vocabulary logits: the log-probability of a given token with the entropy and the top
// alternatives of its distribution, and the distillation loss against a teacher's top log-probabilities with its gradient.
//
// With z = x / temperature, c = log2(e) / temperature and m the largest logit met so far, a thread keeps
//   s = sum 2^((x - m) c)   and, for the entropy,   t = sum 2^((x - m) c) (x - m) c
// and rescales both when m grows, so one pass over the row gives
//   lse = m / temperature + ln s,   log p_v = ((x_v - m) c - log2 s) ln 2,   H = (log2 s - t / s) ln 2.
// The difference is formed before the scaling: a row filled with the type's lowest value then has differences of 0 and
// not of infinity minus infinity.  m starts at the lowest finite fp32 value, so a logit of minus infinity has the weight
// 2^-inf = 0 and a row of them ends with s = 0.  A NaN or an infinite logit makes s NaN (infinity minus itself), which
// is how such a row is recognised.  All sums are fp32 over at most a few hundred terms a thread, then a tree.
#include <float.h>
#include <math.h>

#include "common.cuh"

namespace camera {

namespace {

constexpr int V_THREADS = 512;
constexpr int V_WARPS = V_THREADS / 32;
constexpr int V_UNROLL = 4;                // 16-byte loads in flight per thread
constexpr int V_CAND = 1024;               // candidates for the top alternatives kept in shared memory
constexpr float D_FLOOR = -150.f;          // 2^-150 is 0 in fp32: a floor for exponents that multiply a zero weight

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A row of `n` logits as the threads walk it: up to 15 bytes of single elements before the first 16-byte boundary,
// whole 16-byte vectors, single elements after the last.  Vector v belongs to thread v % V_THREADS, head and tail
// element i to thread i.
template <typename T>
struct Row {
  static constexpr int N = Vec16<T>::N;
  const T* p;
  int n, head, n_vec, tail;
  __device__ __forceinline__ Row(const T* row, int len) : p(row), n(len) {
    const int mis = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    head = mis ? min(N - mis, len) : 0;
    n_vec = (len - head) / N;
    tail = len - head - n_vec * N;
  }
  __device__ __forceinline__ const T* vec(int v) const { return p + head + (size_t)v * N; }
  __device__ __forceinline__ int vec_index(int v) const { return head + v * N; }
  __device__ __forceinline__ int tail_index(int i) const { return head + n_vec * N + i; }
};

__device__ __forceinline__ uint4 ld_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
template <typename T> __device__ __forceinline__ void unpack(const uint4& v, float* out);
template <> __device__ __forceinline__ void unpack<float>(const uint4& v, float* out) {
  out[0] = __uint_as_float(v.x); out[1] = __uint_as_float(v.y); out[2] = __uint_as_float(v.z); out[3] = __uint_as_float(v.w);
}
template <> __device__ __forceinline__ void unpack<__nv_bfloat16>(const uint4& v, float* out) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    out[2 * i] = __uint_as_float(w[i] << 16);
    out[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// The running sums of one thread (or of a whole row).
struct Stats {
  float m, s, t, r;      // r: the part of s from tokens outside the teacher's list
  __device__ __forceinline__ void init() { m = -FLT_MAX; s = 0.f; t = 0.f; r = 0.f; }
  template <bool ENT, bool REST>
  __device__ __forceinline__ void raise(float to, float c) {      // to >= m
    const float d = fmaxf((m - to) * c, D_FLOOR), f = ex2((m - to) * c);
    if (ENT) t = f * fmaf(d, s, t);
    s *= f;
    if (REST) r *= f;
    m = to;
  }
  template <bool ENT>
  __device__ __forceinline__ float add(float x, float c) {        // x <= m
    const float d = (x - m) * c, e = ex2(d);
    s += e;
    if (ENT) t = fmaf(e, fmaxf(d, D_FLOOR), t);
    return e;
  }
  template <bool ENT, bool REST>
  __device__ __forceinline__ void merge(const Stats& o, float c) {
    const float to = fmaxf(m, o.m);
    Stats b = o;
    raise<ENT, REST>(to, c);
    b.raise<ENT, REST>(to, c);
    s += b.s;
    if (ENT) t += b.t;
    if (REST) r += b.r;
  }
};

// One thread's share of the row.  listed: a bit per element of the row that is on the teacher's list (REST only).
template <typename T, bool ENT, bool REST>
__device__ __forceinline__ Stats walk_row(const Row<T>& row, float c, const uint32_t* listed) {
  constexpr int N = Row<T>::N;
  Stats st;
  st.init();
  auto single = [&](int i) {
    const float x = to_f32<T>(row.p[i]);
    if (x > st.m) st.raise<ENT, REST>(x, c);
    const float e = st.add<ENT>(x, c);
    if (REST && !((listed[i >> 5] >> (i & 31)) & 1u)) st.r += e;
  };
  if ((int)threadIdx.x < row.head) single(threadIdx.x);
  if ((int)threadIdx.x < row.tail) single(row.tail_index(threadIdx.x));
  for (int v0 = threadIdx.x; v0 < row.n_vec; v0 += V_UNROLL * V_THREADS) {
    uint4 raw[V_UNROLL];
#pragma unroll
    for (int u = 0; u < V_UNROLL; ++u) {
      const int v = v0 + u * V_THREADS;
      if (v < row.n_vec) raw[u] = ld_stream(row.vec(v));
    }
#pragma unroll
    for (int u = 0; u < V_UNROLL; ++u) {
      const int v = v0 + u * V_THREADS;
      if (v >= row.n_vec) break;
      float x[N];
      unpack<T>(raw[u], x);
      float top = x[0];
#pragma unroll
      for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
      if (top > st.m) st.raise<ENT, REST>(top, c);
      float e[N], es = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float d = (x[i] - st.m) * c;
        e[i] = ex2(d);
        es += e[i];
        if (ENT) st.t = fmaf(e[i], fmaxf(d, D_FLOOR), st.t);
      }
      st.s += es;
      if (REST) {
        const int i0 = row.vec_index(v);
        const uint32_t bits = __funnelshift_r(listed[i0 >> 5], listed[(i0 >> 5) + 1], i0 & 31) & ((1u << N) - 1);
        if (bits) {             // the others are added up again: subtracting the listed ones would cancel
          es = 0.f;
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (!((bits >> i) & 1u)) es += e[i];
        }
        st.r += es;
      }
    }
  }
  return st;
}

// Joins the threads' sums; every thread gets the row's.
template <bool ENT, bool REST>
__device__ __forceinline__ Stats join(Stats st, float c, Stats* part) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    Stats b;
    b.m = __shfl_xor_sync(0xffffffffu, st.m, o);
    b.s = __shfl_xor_sync(0xffffffffu, st.s, o);
    if (ENT) b.t = __shfl_xor_sync(0xffffffffu, st.t, o);
    if (REST) b.r = __shfl_xor_sync(0xffffffffu, st.r, o);
    st.merge<ENT, REST>(b, c);
  }
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = st;
  __syncthreads();
  st = part[0];
  for (int w = 1; w < V_WARPS; ++w) st.merge<ENT, REST>(part[w], c);
  return st;
}

// Order-preserving image of a float (both zeros alike) and the 64-bit key by which alternatives are ranked: larger value
// first, then lower index.
__device__ __forceinline__ uint32_t value_key(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ unsigned long long rank_key(float x, int i) {
  return ((unsigned long long)value_key(x) << 32) | (uint32_t)~i;
}
constexpr uint32_t KEY_NEG_INF = 0x007fffffu;     // value_key(-inf)

struct TopScratch {
  uint32_t group_key[V_THREADS];         // largest value of every thread's share
  int active[V_THREADS];                 // the shares that can hold an alternative
  unsigned long long cand[V_CAND];
  int n_active, n_cand, count;
};

// Calls f(index, value) for every element of the shares listed in sc.active[0 .. n_active).
template <typename T, typename F>
__device__ __forceinline__ void for_active(const Row<T>& row, const TopScratch& sc, F f) {
  constexpr int N = Row<T>::N;
  const int per = (row.n_vec + V_THREADS - 1) / V_THREADS + 1;      // the last "vector" stands for head and tail
  const int total = sc.n_active * per;
  for (int q = threadIdx.x; q < total; q += V_THREADS) {
    const int g = sc.active[q / per], k = q % per;
    if (k == per - 1) {
      if (g < row.head) f(g, to_f32<T>(row.p[g]));
      if (g < row.tail) f(row.tail_index(g), to_f32<T>(row.p[row.tail_index(g)]));
      continue;
    }
    const int v = g + k * V_THREADS;
    if (v >= row.n_vec) continue;
    float x[N];
    unpack<T>(ld_stream(row.vec(v)), x);
#pragma unroll
    for (int i = 0; i < N; ++i) f(row.vec_index(v) + i, x[i]);
  }
}

// The (up to) n elements of the row with the largest keys, logits of minus infinity left out, as sc.cand[0 .. sc.n_cand)
// in any order; at least n of them (if the row has as many), possibly a few more.
// A share whose maximum is below the n-th largest of the shares' maxima holds none of the n largest elements, so only
// about n of the V_THREADS shares are read again.  The threshold is found by bisection on the key bits; where the
// elements at or above it outgrow the candidate list (long runs of equal logits), the bisection goes on over the
// elements' 64-bit keys, which are all distinct.
template <typename T>
__device__ __forceinline__ void collect_top(const Row<T>& row, float own_max, bool own_any, int n, TopScratch& sc) {
  const uint32_t mine = own_any ? value_key(own_max) : 0u;
  uint32_t lo = KEY_NEG_INF + 1, hi = 0xffffffffu;    // invariant: count(>= lo) is enough (or lo is the lowest), count(>= hi) is not
  __syncthreads();
  while (hi - lo > 1) {
    const uint32_t mid = lo + (hi - lo) / 2;
    const int cnt = __syncthreads_count(mine >= mid);
    if (cnt >= n) { lo = mid; if (cnt <= n + n / 4) break; } else hi = mid;
  }
  if (threadIdx.x == 0) { sc.n_active = 0; sc.n_cand = 0; }
  __syncthreads();
  if (mine >= lo) sc.active[atomicAdd(&sc.n_active, 1)] = threadIdx.x;
  __syncthreads();
  unsigned long long klo = (unsigned long long)lo << 32, khi = ~0ull;
  for (int attempt = 0; attempt < 2; ++attempt) {
    for_active(row, sc, [&](int i, float x) {
      const unsigned long long k = rank_key(x, i);
      if (k >= klo) {
        const int at = atomicAdd(&sc.n_cand, 1);
        if (at < V_CAND) sc.cand[at] = k;
      }
    });
    __syncthreads();
    if (sc.n_cand <= V_CAND) return;
    // More than fit: raise klo until n .. V_CAND elements are left.  64 halvings of the key range always get there.
    for (int it = 0; it < 64; ++it) {
      const unsigned long long mid = klo + (khi - klo) / 2;
      __syncthreads();
      if (threadIdx.x == 0) { sc.count = 0; sc.n_cand = 0; }
      __syncthreads();
      int c = 0;
      for_active(row, sc, [&](int i, float x) { c += rank_key(x, i) >= mid; });
      if (c) atomicAdd(&sc.count, c);
      __syncthreads();
      const int all = sc.count;
      if (all >= n) { klo = mid; if (all <= V_CAND) break; } else khi = mid;
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) sc.n_cand = V_CAND;      // only if the logits changed while they were read
  __syncthreads();
}

struct LogprobArgs {
  const void* logits;
  long long ld;
  int vocab, top_n;
  float c, inv_tau;         // log2(e) / temperature, 1 / temperature
  const long long* targets;
  float *logprob, *entropy, *top_logprob;
  int* top_idx;
};

constexpr float LN2 = 0.693147180559945309f;

template <typename T, bool ENT>
__global__ void __launch_bounds__(V_THREADS) k_token_logprobs(const LogprobArgs a) {
  __shared__ Stats part[V_WARPS];
  __shared__ TopScratch sc;
  const long long r = blockIdx.x;
  const Row<T> row(static_cast<const T*>(a.logits) + r * a.ld, a.vocab);
  const Stats own = walk_row<T, ENT, false>(row, a.c, nullptr);
  const Stats st = join<ENT, false>(own, a.c, part);
  const float log2s = log2f(st.s);
  if (threadIdx.x == 0) {
    if (a.logprob) {
      const long long t = a.targets[r];
      float lp = 0.f;
      if (t >= 0 && t < a.vocab) {
        lp = (to_f32<T>(row.p[t]) - st.m) * a.inv_tau - log2s * LN2;
        if (st.s == 0.f) lp = -INFINITY;
      }
      a.logprob[r] = lp;
    }
    if (ENT) a.entropy[r] = st.s == 0.f ? 0.f : (log2s - st.t / st.s) * LN2;
  }
  if (a.top_n == 0) return;
  int* const out_i = a.top_idx + r * a.top_n;
  float* const out_v = a.top_logprob + r * a.top_n;
  const bool usable = st.s > 0.f;                 // false for a NaN
  if (usable) collect_top(row, own.m, own.s > 0.f, a.top_n, sc);
  const int n_cand = usable ? sc.n_cand : 0;
  for (int q = threadIdx.x; q < n_cand; q += V_THREADS) {
    const unsigned long long k = sc.cand[q];
    int rank = 0;
    for (int j = 0; j < n_cand; ++j) rank += sc.cand[j] > k;
    if (rank < a.top_n) {
      const int i = (int)~(uint32_t)k;
      out_i[rank] = i;
      out_v[rank] = (to_f32<T>(row.p[i]) - st.m) * a.inv_tau - log2s * LN2;
    }
  }
  for (int q = n_cand + threadIdx.x; q < a.top_n; q += V_THREADS) {
    out_i[q] = -1;
    out_v[q] = st.s == 0.f || usable ? -INFINITY : NAN;
  }
}

// ---------------------------------------------------------------------------------------------- distillation
// Teacher: a list of k tokens with log-probabilities.  p is their softmax over the list, or, with the rest as one more
// class (TAIL), p = exp(logprob) and rest = 1 - sum p.  Student: q = softmax(x / temperature) over the vocabulary.
//   loss   = sum p (ln p - ln q) [+ rest (ln rest - ln R)],  R = the student's share outside the list
//   d loss / d x_v = (q_v - p_v) / temperature on the list,  q_v / temperature outside; with the rest as a class the
//   latter is q_v (1 - rest / R) / temperature, because a token outside moves the rest's share as well.
// R is summed over the tokens outside (a bitmap in shared memory says which they are), not formed as 1 - Q: once the
// student is right, R is small and the difference would be noise.  The k terms of the list are taken in double: they are
// few, and the loss is a difference of nearly equal logarithms by the end of the training.
struct DistillArgs {
  const void* logits;
  long long ld;
  int vocab, k;
  float c, inv_tau;
  const int* idx;
  const float* logprob;
  const float* d_loss;
  float *loss, *lse, *log_tail;       // outputs of the forward pass, inputs of the backward pass
  void* grad;
  long long ld_grad;
};
enum { DISTILL_FORWARD = 0, DISTILL_BACKWARD = 1, DISTILL_STEP = 2 };

struct TeacherList {
  int idx[CAMERA_MAX_TOP];            // -1: no such entry
  float p[CAMERA_MAX_TOP];
  float log_p[CAMERA_MAX_TOP];
  float x[CAMERA_MAX_TOP];            // the student's logits of the listed tokens
  double rest;
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// One warp reads the row's list and turns it into probabilities.
template <bool TAIL>
__device__ __forceinline__ void load_teacher(const DistillArgs& a, long long r, TeacherList& tl) {
  const int lane = threadIdx.x & 31;
  float top = -INFINITY;
  for (int j = lane; j < a.k; j += 32) {
    int i = a.idx[r * a.k + j];
    float lp = a.logprob[r * a.k + j];
    if (i < 0 || i >= a.vocab) { i = -1; lp = -INFINITY; }
    tl.idx[j] = i;
    tl.log_p[j] = lp;
    top = fmaxf(top, lp);
  }
  double sum = 0.0;
  if (TAIL) {
    for (int j = lane; j < a.k; j += 32) {
      const double p = exp((double)tl.log_p[j]);
      tl.p[j] = (float)p;
      sum += p;
    }
    sum = warp_sum(sum);
    if (lane == 0) tl.rest = 1.0 - sum < 0.0 ? 0.0 : 1.0 - sum;      // keeps a NaN
  } else {
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == -INFINITY) top = 0.f;                                  // nothing on the list
    for (int j = lane; j < a.k; j += 32) sum += exp((double)(tl.log_p[j] - top));
    sum = warp_sum(sum);
    const double log_sum = log(sum);
    for (int j = lane; j < a.k; j += 32) {
      const double lp = (double)(tl.log_p[j] - top) - log_sum;
      tl.p[j] = sum > 0.0 || sum != sum ? (float)exp(lp) : 0.f;
      tl.log_p[j] = (float)lp;
    }
    if (lane == 0) tl.rest = 0.0;
  }
}

// Writes scale * 2^((x - m) c - off) for every element of the row.
template <typename T>
__device__ __forceinline__ void write_row(const Row<T>& row, T* out, float m, float c, float off, float scale) {
  constexpr int N = Row<T>::N;
  auto grad = [&](float x) { return scale * ex2((x - m) * c - off); };
  auto put = [&](int i, float v) {
    if constexpr (sizeof(T) == 2) out[i] = __float2bfloat16_rn(v); else out[i] = v;
  };
  if ((int)threadIdx.x < row.head) put(threadIdx.x, grad(to_f32<T>(row.p[threadIdx.x])));
  if ((int)threadIdx.x < row.tail) {
    const int i = row.tail_index(threadIdx.x);
    put(i, grad(to_f32<T>(row.p[i])));
  }
  const bool vec_out = (reinterpret_cast<uintptr_t>(out + row.head) & 15) == 0;
  for (int v0 = threadIdx.x; v0 < row.n_vec; v0 += V_UNROLL * V_THREADS) {
    uint4 raw[V_UNROLL];
#pragma unroll
    for (int u = 0; u < V_UNROLL; ++u) {
      const int v = v0 + u * V_THREADS;
      if (v < row.n_vec) raw[u] = ld_stream(row.vec(v));
    }
#pragma unroll
    for (int u = 0; u < V_UNROLL; ++u) {
      const int v = v0 + u * V_THREADS;
      if (v >= row.n_vec) break;
      float x[N];
      unpack<T>(raw[u], x);
#pragma unroll
      for (int i = 0; i < N; ++i) x[i] = grad(x[i]);
      const int i0 = row.vec_index(v);
      if (vec_out) {
        uint4 o;
        if constexpr (sizeof(T) == 2) {
          __nv_bfloat162 h[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
          o = *reinterpret_cast<const uint4*>(h);
        } else {
          o = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
        }
        *reinterpret_cast<uint4*>(out + i0) = o;
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) put(i0 + i, x[i]);
      }
    }
  }
}

template <typename T, int MODE, bool TAIL>
__global__ void __launch_bounds__(V_THREADS) k_distill(const DistillArgs a) {
  constexpr bool STATS = MODE != DISTILL_BACKWARD;
  constexpr bool GRAD = MODE != DISTILL_FORWARD;
  constexpr bool REST = STATS && TAIL;
  extern __shared__ uint32_t listed[];               // REST: a bit per token, set on the list
  __shared__ Stats part[V_WARPS];
  __shared__ TeacherList tl;
  const long long r = blockIdx.x;
  const Row<T> row(static_cast<const T*>(a.logits) + r * a.ld, a.vocab);
  T* const out = GRAD ? static_cast<T*>(a.grad) + r * a.ld_grad : nullptr;
  const int tid = threadIdx.x;
  const float w = GRAD ? a.d_loss[r] * a.inv_tau : 0.f;
  if (GRAD && a.d_loss[r] == 0.f) {                   // a row that does not count: its logits are not looked at
    for (int i = tid; i < a.vocab; i += V_THREADS) {
      if constexpr (sizeof(T) == 2) out[i] = __float2bfloat16_rn(0.f); else out[i] = 0.f;
    }
    if (STATS && tid == 0) a.loss[r] = 0.f;
    return;
  }
  if (REST)
    for (int i = tid; i < (a.vocab >> 5) + 2; i += V_THREADS) listed[i] = 0u;
  if (tid < 32) load_teacher<TAIL>(a, r, tl);
  __syncthreads();
  const int li = tid < a.k ? tl.idx[tid] : -1;
  if (REST) {
    if (li >= 0) atomicOr(&listed[li >> 5], 1u << (li & 31));
    __syncthreads();
  }
  if (tid < a.k) tl.x[tid] = li >= 0 ? to_f32<T>(row.p[li]) : 0.f;     // read before the gradient may overwrite it
  float m, off, coef = 1.f;
  bool empty;
  if (STATS) {
    Stats st = join<false, REST>(walk_row<T, false, REST>(row, a.c, listed), a.c, part);
    // no distribution: every logit minus infinity, or all of them beyond fp32's range once scaled
    empty = st.s == 0.f || st.m * a.c < -FLT_MAX;
    m = st.m;
    off = log2f(st.s);
    if (REST && tl.rest != 0.0) coef = st.r > 0.f || st.r != st.r ? (float)(1.0 - tl.rest * ((double)st.s / (double)st.r)) : 0.f;
    if (tid < 32) {
      double loss = 0.0;
      for (int j = tid; j < a.k; j += 32) {
        const float p = tl.p[j];
        if (tl.idx[j] < 0 || p == 0.f) continue;
        loss += (double)p * ((double)tl.log_p[j] - (double)((tl.x[j] - m) * a.c - off) * 0.6931471805599453);
      }
      loss = warp_sum(loss);
      if (tid == 0) {
        if (REST && tl.rest != 0.0 && (st.r > 0.f || st.r != st.r))
          loss += tl.rest * (log(tl.rest) - (double)(log2f(st.r) - off) * 0.6931471805599453);
        a.loss[r] = empty ? 0.f : (float)loss;
        if (MODE == DISTILL_FORWARD) {
          if (a.lse) a.lse[r] = empty ? -INFINITY : (m * a.c + off) * LN2;
          if (TAIL && a.log_tail) a.log_tail[r] = empty || st.r == 0.f ? -INFINITY : (m * a.c + log2f(st.r)) * LN2;
        }
      }
    }
  } else {
    __syncthreads();                                 // the listed logits are read before any of them is overwritten
    const float lse = a.lse[r];
    empty = lse == -INFINITY;
    m = 0.f;
    off = lse * 1.44269504088896341f;
    if (TAIL && tl.rest != 0.0) {
      const float lt = a.log_tail[r];
      coef = lt == -INFINITY ? 0.f : (float)(1.0 - tl.rest * exp((double)lse - (double)lt));
    }
  }
  if (!GRAD) return;
  if (empty) {
    for (int i = tid; i < a.vocab; i += V_THREADS) {
      if constexpr (sizeof(T) == 2) out[i] = __float2bfloat16_rn(0.f); else out[i] = 0.f;
    }
    return;
  }
  write_row<T>(row, out, m, a.c, off, w * coef);
  __syncthreads();
  if (li >= 0) {
    const float g = w * (ex2((tl.x[tid] - m) * a.c - off) - tl.p[tid]);
    if constexpr (sizeof(T) == 2) out[li] = __float2bfloat16_rn(g); else out[li] = g;
  }
}

template <int MODE>
cudaError_t launch_distill(const DistillArgs& a, int dtype, bool tail, long long rows, cudaStream_t st) {
  const size_t smem = tail && MODE != DISTILL_BACKWARD ? ((size_t)(a.vocab >> 5) + 2) * 4 : 0;
  auto go = [&](auto kern) {
    if (smem > 32 * 1024) {
      const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
      if (e != cudaSuccess) return e;
    }
    kern<<<(unsigned)rows, V_THREADS, smem, st>>>(a);
    return cudaGetLastError();
  };
  if (dtype == CAMERA_BF16) return tail ? go(k_distill<__nv_bfloat16, MODE, true>) : go(k_distill<__nv_bfloat16, MODE, false>);
  return tail ? go(k_distill<float, MODE, true>) : go(k_distill<float, MODE, false>);
}

int check_logits(const void* logits, int dtype, int64_t ld, int64_t n_rows, int32_t vocab, float temperature) {
  if (dtype != CAMERA_F32 && dtype != CAMERA_BF16) return CAMERA_ERR_INVALID_ARG;
  if (n_rows < 0 || vocab < 1 || ld < vocab || !(temperature > 0.f) || isinf(temperature)) return CAMERA_ERR_INVALID_ARG;
  if (vocab > CAMERA_MAX_VOCAB || n_rows > 0x7fffffff) return CAMERA_ERR_UNSUPPORTED_SHAPE;
  if (n_rows > 0 && (logits == nullptr || (reinterpret_cast<uintptr_t>(logits) & (dtype == CAMERA_BF16 ? 1 : 3))))
    return CAMERA_ERR_INVALID_ARG;
  return CAMERA_OK;
}

int check_distill(const camera_distill_t* d) {
  if (d == nullptr) return CAMERA_ERR_INVALID_ARG;
  const int rc = check_logits(d->logits, d->dtype, d->ld, d->n_rows, d->vocab, d->temperature);
  if (rc != CAMERA_OK) return rc;
  if (d->k < 1 || (d->flags & ~(uint32_t)CAMERA_DISTILL_TAIL)) return CAMERA_ERR_INVALID_ARG;
  if (d->k > CAMERA_MAX_TOP) return CAMERA_ERR_UNSUPPORTED_SHAPE;
  if (d->n_rows > 0 && (d->teacher_idx == nullptr || d->teacher_logprob == nullptr)) return CAMERA_ERR_INVALID_ARG;
  return CAMERA_OK;
}

bool grad_ok(const camera_distill_t* d, const void* grad, int64_t ld) {
  const uintptr_t mask = d->dtype == CAMERA_BF16 ? 1 : 3;
  return grad != nullptr && ld >= d->vocab && (reinterpret_cast<uintptr_t>(grad) & mask) == 0 &&
         (grad != d->logits || ld == d->ld);          // in place: the same rows
}

DistillArgs distill_args(const camera_distill_t* d) {
  DistillArgs a;
  a.logits = d->logits; a.ld = d->ld; a.vocab = d->vocab; a.k = d->k;
  a.c = 1.44269504088896341f / d->temperature; a.inv_tau = 1.f / d->temperature;
  a.idx = d->teacher_idx; a.logprob = d->teacher_logprob;
  a.d_loss = nullptr; a.loss = a.lse = a.log_tail = nullptr; a.grad = nullptr; a.ld_grad = 0;
  return a;
}

}  // namespace
}  // namespace camera

extern "C" int camera_token_logprobs(const void* logits, int32_t dtype, int64_t ld, int64_t n_rows, int32_t vocab,
                                     const int64_t* targets, int32_t top_n, float temperature, float* logprob,
                                     float* entropy, int32_t* top_idx, float* top_logprob, void* cuda_stream) {
  using namespace camera;
  const int rc = check_logits(logits, dtype, ld, n_rows, vocab, temperature);
  if (rc != CAMERA_OK) return rc;
  if (top_n < 0 || (targets == nullptr) != (logprob == nullptr)) return CAMERA_ERR_INVALID_ARG;
  if (top_n > CAMERA_MAX_TOP) return CAMERA_ERR_UNSUPPORTED_SHAPE;
  if (n_rows == 0) return CAMERA_OK;
  if (top_n > 0 && (top_idx == nullptr || top_logprob == nullptr)) return CAMERA_ERR_INVALID_ARG;
  LogprobArgs a{logits, ld, vocab, top_n, 1.44269504088896341f / temperature, 1.f / temperature, reinterpret_cast<const long long*>(targets),
                logprob, entropy, top_logprob, top_idx};
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const unsigned grid = (unsigned)n_rows;
  if (dtype == CAMERA_BF16) {
    if (entropy) k_token_logprobs<__nv_bfloat16, true><<<grid, V_THREADS, 0, st>>>(a);
    else k_token_logprobs<__nv_bfloat16, false><<<grid, V_THREADS, 0, st>>>(a);
  } else {
    if (entropy) k_token_logprobs<float, true><<<grid, V_THREADS, 0, st>>>(a);
    else k_token_logprobs<float, false><<<grid, V_THREADS, 0, st>>>(a);
  }
  return cudaGetLastError() == cudaSuccess ? CAMERA_OK : CAMERA_ERR_CUDA;
}

extern "C" int camera_distill_forward(const camera_distill_t* d, float* loss, float* lse, float* log_tail, void* cuda_stream) {
  using namespace camera;
  const int rc = check_distill(d);
  if (rc != CAMERA_OK) return rc;
  if (d->n_rows == 0) return CAMERA_OK;
  if (loss == nullptr) return CAMERA_ERR_INVALID_ARG;
  DistillArgs a = distill_args(d);
  a.loss = loss; a.lse = lse; a.log_tail = log_tail;
  return launch_distill<DISTILL_FORWARD>(a, d->dtype, d->flags & CAMERA_DISTILL_TAIL, d->n_rows,
                                         static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? CAMERA_OK : CAMERA_ERR_CUDA;
}

extern "C" int camera_distill_backward(const camera_distill_t* d, const float* d_loss, const float* lse, const float* log_tail,
                                       void* d_logits, int64_t d_ld, void* cuda_stream) {
  using namespace camera;
  const int rc = check_distill(d);
  if (rc != CAMERA_OK) return rc;
  if (d->n_rows == 0) return CAMERA_OK;
  if (d_loss == nullptr || lse == nullptr || (log_tail == nullptr && (d->flags & CAMERA_DISTILL_TAIL)) ||
      !grad_ok(d, d_logits, d_ld))
    return CAMERA_ERR_INVALID_ARG;
  DistillArgs a = distill_args(d);
  a.d_loss = d_loss; a.lse = const_cast<float*>(lse); a.log_tail = const_cast<float*>(log_tail);
  a.grad = d_logits; a.ld_grad = d_ld;
  return launch_distill<DISTILL_BACKWARD>(a, d->dtype, d->flags & CAMERA_DISTILL_TAIL, d->n_rows,
                                          static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? CAMERA_OK : CAMERA_ERR_CUDA;
}

extern "C" int camera_distill_step(const camera_distill_t* d, const float* d_loss, float* loss, void* d_logits, int64_t d_ld,
                                   void* cuda_stream) {
  using namespace camera;
  const int rc = check_distill(d);
  if (rc != CAMERA_OK) return rc;
  if (d->n_rows == 0) return CAMERA_OK;
  if (d_loss == nullptr || loss == nullptr || !grad_ok(d, d_logits, d_ld)) return CAMERA_ERR_INVALID_ARG;
  DistillArgs a = distill_args(d);
  a.d_loss = d_loss; a.loss = loss; a.grad = d_logits; a.ld_grad = d_ld;
  return launch_distill<DISTILL_STEP>(a, d->dtype, d->flags & CAMERA_DISTILL_TAIL, d->n_rows,
                                      static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? CAMERA_OK : CAMERA_ERR_CUDA;
}
