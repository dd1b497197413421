// Operators over rows of vocabulary logits: the log-probability of a given token with the entropy and the top
// alternatives of its distribution, and the distillation loss against a teacher's top log-probabilities with its gradient.
//
// With z = x / temperature and c = log2(e) / temperature, a thread takes a reference m (x c for the largest x of the
// first chunk it reads that has a logit above -126 / c: a mask at the front of its share does not count) and sums over its
// share of the row
//   s = sum 2^(x c - m)   and, for the entropy,   t = sum 2^(x c - m) (x c - m);
// the threads' sums are joined by scaling with 2^(m_i - max m).  One pass over the row then gives
//   ln sum exp z = (m + log2 s) ln 2,   log p_v = (x_v c - m - log2 s) ln 2,   H = (log2 s - t / s) ln 2.
// The reference does not follow the maximum closely: fp32 holds 2^(x c - m) for any x c up to m + 127, and scaling loses
// no precision in s.  Only the entropy wants it within a few powers of two of the largest logit, because log2 s and t / s
// cancel (4095 rows: error of the entropies against 64 bits 9.6e-6 without, 6e-7 with): where it is asked for, a thread
// raises its reference when a chunk's maximum exceeds it by more than 2^REF_SLACK.  A row whose sum ends outside
// [2^-60, 2^120] (logits far above a share's first, all of them the type's lowest value, NaN, infinity: nothing an
// ordinary row does) is walked again with differences formed before the scaling and a running maximum (walk_careful; two to
// four times an ordinary row's time: 2048 rows of 151936 bf16 logits around -200, log-probabilities 107 -> 402 us,
// distillation step 289 -> 1055 us).
// All sums are fp32, over a few hundred terms a thread (4096 at the largest vocabulary), then a tree in a fixed order.
//
// Bound by reading the logits once; the arithmetic comes close behind (an exponential per logit: 16 a clock and SM), so
// the multiply-adds run in pairs (f32x2) and the loop holds nothing else.  Few rows are split over the CTAs of a cluster,
// which exchange their sums (and alternatives) through distributed shared memory.
#include <float.h>
#include <math.h>

#include <atomic>
#include <type_traits>

#include "common.cuh"
#include "launch.cuh"
#include "umma_pair.cuh"

namespace camera {

namespace {

constexpr int V_THREADS = 256;
constexpr int V_WARPS = V_THREADS / 32;
constexpr long long STEP_L2_BYTES = 60ll << 20;   // half of L2
constexpr int V_MAX_LG = 3, V_MAX_SPLIT = 1 << V_MAX_LG;       // CTAs that can share a row
constexpr float D_FLOOR = -150.f;          // 2^-150 is 0 in fp32: a floor for exponents that multiply a zero weight
constexpr float D_PART = -100.f;           // the most a sum is scaled down in one step
constexpr float REF_FLOOR = -126.f;        // references start here
constexpr float REF_SLACK = 3.f;
constexpr float SHARE_FLOOR = -1022.f;     // log2 of the smallest share outside a teacher's list that counts
constexpr float LN2 = 0.693147180559945309f;
constexpr float LOG2E = 1.44269504088896341f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {      // NaN if either is
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)),
        "l"(*reinterpret_cast<unsigned long long*>(&c)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(r)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
  return *reinterpret_cast<float2*>(&r);
}

__device__ __forceinline__ uint4 ld_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// What depends on the element type: how a 16-byte vector becomes pairs of floats, its maximum, minus infinity.
template <typename T> struct Elem;
template <> struct Elem<float> {
  static constexpr int N = 4;
  static constexpr uint32_t NEG_INF = 0xff800000u;
  __device__ __forceinline__ static void pairs(const uint4& v, float2* x) {
    x[0] = make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
    x[1] = make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
  }
  // maxima in the raw form; NaN is passed over
  __device__ __forceinline__ static uint32_t max_word(uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }
  __device__ __forceinline__ static uint32_t max_vec(const uint4& v) { return max_word(max_word(v.x, v.y), max_word(v.z, v.w)); }
  __device__ __forceinline__ static float max_of(uint32_t w) { return __uint_as_float(w); }
  __device__ __forceinline__ static float put(float v) { return v; }
  __device__ __forceinline__ static uint4 pack(const float2* x) {
    return make_uint4(__float_as_uint(x[0].x), __float_as_uint(x[0].y), __float_as_uint(x[1].x), __float_as_uint(x[1].y));
  }
};
template <> struct Elem<__nv_bfloat16> {
  static constexpr int N = 8;
  static constexpr uint32_t NEG_INF = 0xff80ff80u;
  __device__ __forceinline__ static void pairs(const uint4& v, float2* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
  __device__ __forceinline__ static uint32_t max_word(uint32_t a, uint32_t b) {      // of two pairs, each its own maximum
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  __device__ __forceinline__ static uint32_t max_vec(const uint4& v) { return max_word(max_word(v.x, v.y), max_word(v.z, v.w)); }
  __device__ __forceinline__ static float max_of(uint32_t w) {
    return fmaxf(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
  __device__ __forceinline__ static __nv_bfloat16 put(float v) { return __float2bfloat16_rn(v); }
  __device__ __forceinline__ static uint4 pack(const float2* x) {
    __nv_bfloat162 h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __float22bfloat162_rn(x[i]);
    return *reinterpret_cast<const uint4*>(h);
  }
};
// A row of `n` logits, or the part of it that CTA `part` of 2^lg walks: single elements before the first 16-byte
// boundary (part 0), whole 16-byte vectors [v_begin, v_end), single elements after the last (last part).  Vector v belongs to
// thread (v - v_begin) % V_THREADS, single element i of head or tail to thread i.
template <typename T>
struct Row {
  static constexpr int N = Elem<T>::N;
  const T* p;
  int first;                 // index of the first element of vector 0
  int head, v_begin, v_end, tail, tail_at;
  __device__ __forceinline__ Row(const T* row, int n, int part, int lg) : p(row) {
    const int mis = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    first = mis ? min(N - mis, n) : 0;
    const int n_vec = (n - first) / N;
    v_begin = (n_vec * part) >> lg;
    v_end = (n_vec * (part + 1)) >> lg;
    head = part == 0 ? first : 0;
    tail_at = first + n_vec * N;
    tail = part + 1 == 1 << lg ? n - tail_at : 0;
  }
  __device__ __forceinline__ const T* vec(int v) const { return p + first + (size_t)v * N; }
  __device__ __forceinline__ int vec_index(int v) const { return first + v * N; }
  __device__ __forceinline__ bool holds(int i) const {       // is element i of the row in this part?
    if (i < first) return head != 0;
    if (i >= tail_at) return tail != 0;
    const int v = (i - first) / N;
    return v >= v_begin && v < v_end;
  }
};

// Sums of a thread, a CTA or a row.  ref: the reference of s, in powers of two (or, of a careful walk, in logits).  ENT: t is
// the entropy's sum.  REST: s counts the tokens outside the teacher's list alone, l those on it against a reference t of
// their own, so that neither is lost where the other is larger by any factor.
struct Sums {
  float ref, s, t, l;
};
template <bool REST>
__device__ __forceinline__ Sums no_sums() { return Sums{-FLT_MAX, 0.f, REST ? -FLT_MAX : 0.f, 0.f}; }
// 2^d (d <= 0) times v.  A share whose reference is far below the largest may all the same hold the largest weights (up to
// 2^127 of them: logits that start with a mask), so a factor below fp32's range is applied in two parts; at once it would be
// flushed to 0 and the share lost.
__device__ __forceinline__ float scale_down(float v, float d) {
  const float d0 = fmaxf(d, D_PART);
  return v * ex2(d0) * ex2(d - d0);                          // the last is 1 unless d is below D_PART
}
// s and (ENT) t brought to the reference `to` >= ref; l to `to` >= t.
template <bool CAREFUL, bool ENT>
__device__ __forceinline__ void raise(Sums& a, float to, float c) {
  const float d = CAREFUL ? (a.ref - to) * c : a.ref - to;
  if (ENT) a.t = scale_down(fmaf(fmaxf(d, D_FLOOR), a.s, a.t), d);
  a.s = scale_down(a.s, d);
  a.ref = to;
}
template <bool CAREFUL>
__device__ __forceinline__ void raise_listed(Sums& a, float to, float c) {
  a.l = scale_down(a.l, CAREFUL ? (a.t - to) * c : a.t - to);
  a.t = to;
}

// The rows first, first + stride, .. whose weight is not 0 (null: all rows).  Weights are read one row ahead, so that
// nothing waits for one.
struct RowWalk {
  int at;
  float ahead;
  __device__ __forceinline__ void begin(const float* weight, int rows, int first) {
    at = first;
    ahead = weight != nullptr && at < rows ? weight[at] : 1.f;
  }
  __device__ __forceinline__ int next(const float* weight, int rows, int stride) {
    while (at < rows) {
      const float w = ahead;
      const int r = at;
      at += stride;
      if (weight != nullptr && at < rows) ahead = weight[at];
      if (w != 0.f) return r;
    }
    return rows;
  }
};

// Chunks of PER vectors a thread, SLOTS of them in the ring.
template <int PER_, int SLOTS_>
struct Ring {
  static constexpr int PER = PER_, SLOTS = SLOTS_;
  static constexpr int CHUNK = PER * V_THREADS;              // vectors
  static constexpr int BYTES = SLOTS * CHUNK * 16;
};
using RingStream = Ring<8, 3>;       // 96 KB: two CTAs fit an SM
using RingDistill = Ring<4, 6>;      // the same bytes in smaller pieces: registers for the second pass

// A quarter of a warp copies 128 bytes at a time: off a 128-byte boundary in shared memory each such piece takes two
// requests of L2 (300 rows of 151936 fp32 logits, gradient alone: 3.6 -> 6.4 million requests, 74 -> 84 us).
constexpr int RING_ALIGN = 128;

// The logits' way into the CTA: every thread copies its own 16-byte vectors with cp.async into its own places of a ring
// in shared memory, over the ends of rows: while the sums of a row are joined and its results written, the next row is on
// its way.  A thread reads only what it copied itself, so there is nothing to wait for but its own copies
// (cp.async.wait_group) and no barrier.  One copy group is committed per chunk consumed.  twice: every row is sent two
// times in a row, for the pass that sums it and the pass that writes its gradient.
template <typename T, typename RG>
struct Feed {
  const T* logits;
  long long ld;
  const float* weight;               // rows with weight 0 are passed over (null: none are)
  int rows, stride, vocab, part, lg;
  int r;                             // row the next chunk belongs to
  bool twice, again;                 // every row comes twice in a row; the second time now
  uint32_t dst0, dst;                // this thread's place in slot 0 and in the next slot
  const T* src;                      // this thread's first vector of the next chunk
  int whole;                         // vectors from the chunk's first to the end of the part
  RowWalk walk;
  __device__ __forceinline__ void begin(int first, bool twice_ = false) {
    dst = dst0;
    twice = twice_; again = false; r = -1;
    walk.begin(weight, rows, first);
    open();
  }
  __device__ __forceinline__ void open() {
    if (twice && !again && r >= 0) {
      again = true;
    } else {
      again = false;
      r = walk.next(weight, rows, stride);
    }
    if (r >= rows) return;
    const Row<T> row(logits + r * ld, vocab, part, lg);
    src = row.vec(row.v_begin) + (size_t)threadIdx.x * Row<T>::N;
    whole = row.v_end - row.v_begin;
  }
  __device__ __forceinline__ void copy(int u) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + (uint32_t)(u * V_THREADS * 16)),
                 "l"(src + (size_t)u * V_THREADS * Row<T>::N)
                 : "memory");
  }
  __device__ __forceinline__ void issue() {
    if (r < rows) {
      if (whole >= RG::CHUNK) {
#pragma unroll
        for (int u = 0; u < RG::PER; ++u) copy(u);
      } else {
#pragma unroll
        for (int u = 0; u < RG::PER; ++u)
          if ((int)threadIdx.x + u * V_THREADS < whole) copy(u);
      }
      src += (size_t)RG::CHUNK * Row<T>::N;
      whole -= RG::CHUNK;
      dst += RG::CHUNK * 16;
      if (dst == dst0 + RG::BYTES) dst = dst0;
      if (whole <= 0) open();
    }
    commit();
  }
  __device__ __forceinline__ static void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
  // the oldest chunk not yet consumed has landed
  __device__ __forceinline__ static void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(RG::SLOTS - 1) : "memory"); }
};
// Chunks of a part, one at least; and the offset in the ring behind the chunk at `at`.
template <typename RG>
__device__ __forceinline__ int row_chunks(int n_vec) { return n_vec <= RG::CHUNK ? 1 : (n_vec + RG::CHUNK - 1) / RG::CHUNK; }
template <typename RG>
__device__ __forceinline__ int next_chunk(int at) { return at + RG::CHUNK * 16 == RG::BYTES ? 0 : at + RG::CHUNK * 16; }

// PER vectors of this thread from the ring.
template <typename RG>
__device__ __forceinline__ void read_chunk(const uint8_t* mine, int at, uint4* raw) {
#pragma unroll
  for (int u = 0; u < RG::PER; ++u) raw[u] = *reinterpret_cast<const uint4*>(mine + at + u * V_THREADS * 16);
}

// One thread's share of the row, whose chunks arrive in the ring from offset `at` on (moved past the row).  mark (REST): a
// bit per vector of the part, set where it holds a token of the teacher's list; such vectors are left out.  TOP: top[u]
// receives the largest logit of its vectors u of all chunks, single elements counted to u = 0 (minus infinity if there
// are none).
template <typename T, typename RG, bool ENT, bool REST, bool TOP>
__device__ __forceinline__ Sums walk_row(const Row<T>& row, float c, Feed<T, RG>& feed, const uint8_t* ring, int& at,
                                         const uint32_t* mark, const int* list, int k, float* top) {
  constexpr int N = Elem<T>::N;
  constexpr uint32_t NI = Elem<T>::NEG_INF;
  const uint4 nothing = make_uint4(NI, NI, NI, NI);          // minus infinity has no weight
  const int tid = threadIdx.x;
  uint32_t big[TOP ? RG::PER : 1];                           // running maxima in the raw form
  if (TOP) {
#pragma unroll
    for (int u = 0; u < RG::PER; ++u) big[u] = NI;
  }
  float2 s2 = make_float2(0.f, 0.f), t2 = make_float2(0.f, 0.f);
  const float2 c2 = make_float2(c, c);
  float2 ref2 = make_float2(-REF_FLOOR, -REF_FLOOR);         // minus the reference
  float single[2] = {-INFINITY, -INFINITY}, listed[2] = {-INFINITY, -INFINITY};     // of this thread: off and on the list
  if (tid < row.head) single[0] = to_f32<T>(row.p[tid]);
  if (tid < row.tail) single[1] = to_f32<T>(row.p[row.tail_at + tid]);
  if (REST) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      if (tid >= (q == 0 ? row.head : row.tail)) continue;
      const int i = q == 0 ? tid : row.tail_at + tid;
      bool on = false;
      for (int j = 0; j < k; ++j) on |= list[j] == i;
      if (on) { listed[q] = single[q]; single[q] = -INFINITY; }
    }
  }
  const uint8_t* const mine = ring + tid * 16;
  if (REST) mark += tid >> 5;
  float raise_at = REF_FLOOR;                                // a maximum above this becomes the reference
  float seen = -INFINITY;                                    // REST: the largest before one did
  int left = row.v_end - row.v_begin;                        // vectors of the part not yet walked
  do {
    uint4 raw[RG::PER];
    Feed<T, RG>::wait();
    read_chunk<RG>(mine, at, raw);
    at = next_chunk<RG>(at);
    if (left < RG::CHUNK) {
#pragma unroll
      for (int u = 0; u < RG::PER; ++u)
        if (tid + u * V_THREADS >= left) raw[u] = nothing;
    }
    if (REST) {
      uint32_t word[RG::PER], any = 0;
#pragma unroll
      for (int u = 0; u < RG::PER; ++u) { word[u] = mark[u * (V_THREADS / 32)]; any |= word[u]; }
      if (any) {                                             // the same in the whole warp
#pragma unroll
        for (int u = 0; u < RG::PER; ++u)
          if ((word[u] >> (tid & 31)) & 1u) raw[u] = nothing;
      }
      mark += RG::CHUNK / 32;
    }
    if (ENT || TOP || raise_at == REF_FLOOR) {
      uint32_t chunk = NI;
#pragma unroll
      for (int u = 0; u < RG::PER; ++u) {
        const uint32_t w = Elem<T>::max_vec(raw[u]);
        if (TOP) big[u] = Elem<T>::max_word(big[u], w);
        chunk = Elem<T>::max_word(chunk, w);
      }
      const float m = fmaxf(Elem<T>::max_of(chunk), fmaxf(single[0], single[1])) * c;
      if (REST) seen = fmaxf(seen, m);
      // the first logits above the floor, or for the entropy's digits (see above) larger ones further on
      if (m > raise_at) {
        const float d = -ref2.x - m, f = ex2(d), dd = fmaxf(d, D_FLOOR);
        const float2 f2 = make_float2(f, f), dd2 = make_float2(dd, dd);
        if (ENT) t2 = mul2(f2, fma2(dd2, s2, t2));
        s2 = mul2(s2, f2);
        ref2 = make_float2(-m, -m);
        raise_at = ENT ? m + REF_SLACK : INFINITY;
      }
    }
#pragma unroll
    for (int u = 0; u < RG::PER; ++u) {
      float2 x[N / 2];
      Elem<T>::pairs(raw[u], x);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        float2 d = fma2(x[i], c2, ref2);
        if (ENT) d = make_float2(max_nan(d.x, D_FLOOR), max_nan(d.y, D_FLOOR));
        x[i] = make_float2(ex2(d.x), ex2(d.y));
        if (ENT) t2 = fma2(x[i], d, t2);
        s2 = add2(s2, x[i]);
      }
    }
    feed.issue();
    left -= RG::CHUNK;
  } while (left > 0);
  Sums st;
  st.ref = -ref2.x;
  st.s = s2.x + s2.y;
  st.t = ENT ? t2.x + t2.y : 0.f;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    if (tid >= (q == 0 ? row.head : row.tail)) continue;
    float d = fmaf(single[q], c, ref2.x);
    if (ENT) d = max_nan(d, D_FLOOR);
    const float e = ex2(d);
    if (ENT) st.t = fmaf(e, d, st.t);
    st.s += e;
  }
  if (REST) {
    if (st.s == 0.f) st.ref = fmaxf(seen, -FLT_MAX);         // how far below the floor everything lies (see sums_ordinary)
    st.t = fmaxf(fmaxf(listed[0], listed[1]) * c, REF_FLOOR);
    st.l = ex2(fmaf(listed[0], c, -st.t)) + ex2(fmaf(listed[1], c, -st.t));
  }
  if (TOP) {
#pragma unroll
    for (int u = 0; u < RG::PER; ++u) top[u] = Elem<T>::max_of(big[u]);
    top[0] = fmaxf(top[0], fmaxf(single[0], single[1]));
  }
  return st;
}

// The same from global memory, with a running maximum and differences formed before the scaling: right for any row, and
// how a NaN or an infinite logit (infinity minus itself) shows as a NaN sum, a row of minus infinities as s = 0.  Only
// elements of marked vectors (see walk_row) and single ones are looked for on the list.
template <typename T, bool ENT, bool REST>
__device__ __noinline__ Sums walk_careful(const Row<T> row, float c, const uint32_t* mark, const int* list, int k) {
  constexpr int N = Elem<T>::N;
  Sums st = no_sums<REST>();
  auto one = [&](float x, int i, bool look) {
    if (REST && look) {
      bool on = false;
      for (int j = 0; j < k; ++j) on |= list[j] == i;
      if (on) {
        if (x > st.t) raise_listed<true>(st, x, c);
        st.l += ex2((x - st.t) * c);
        return;
      }
    }
    if (x > st.ref) raise<true, ENT>(st, x, c);
    const float d = (x - st.ref) * c, e = ex2(d);
    st.s += e;
    if (ENT) st.t = fmaf(e, fmaxf(d, D_FLOOR), st.t);
  };
  if ((int)threadIdx.x < row.head) one(to_f32<T>(row.p[threadIdx.x]), threadIdx.x, true);
  if ((int)threadIdx.x < row.tail) one(to_f32<T>(row.p[row.tail_at + threadIdx.x]), row.tail_at + threadIdx.x, true);
  for (int v = row.v_begin + threadIdx.x; v < row.v_end; v += V_THREADS) {
    const uint4 raw = ld_stream(row.vec(v));
    const int at = v - row.v_begin;
    const bool look = REST && ((mark[at >> 5] >> (at & 31)) & 1u);
    float2 x[N / 2];
    Elem<T>::pairs(raw, x);
#pragma unroll
    for (int i = 0; i < N; ++i) one(i & 1 ? x[i >> 1].y : x[i >> 1].x, row.vec_index(v) + i, look);
  }
  return st;
}

// Shared memory of a CTA that joins sums.
struct JoinScratch {
  Sums warp[2][2 * V_WARPS];       // joins alternate, so that none overwrites what another thread still reads
  alignas(16) Sums cta[2][V_MAX_SPLIT];    // of the CTAs that share the row, written by each of them (see Exchange)
  unsigned long long bars[3];
};
// The sums of WIDTH neighbouring lanes joined, in all of them.
template <int WIDTH, bool CAREFUL, bool ENT, bool REST>
__device__ __forceinline__ Sums join_lanes(Sums st, float c) {
  float to = st.ref, to_l = st.t;
#pragma unroll
  for (int o = WIDTH / 2; o; o >>= 1) {
    to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, o));
    if (REST) to_l = fmaxf(to_l, __shfl_xor_sync(0xffffffffu, to_l, o));
  }
  raise<CAREFUL, ENT>(st, to, c);
  if (REST) raise_listed<CAREFUL>(st, to_l, c);
#pragma unroll
  for (int o = WIDTH / 2; o; o >>= 1) {
    st.s += __shfl_xor_sync(0xffffffffu, st.s, o);
    if (ENT) st.t += __shfl_xor_sync(0xffffffffu, st.t, o);
    if (REST) st.l += __shfl_xor_sync(0xffffffffu, st.l, o);
  }
  return st;
}
// Sums of the CTA from those of its threads, the same in every thread.  WARPS: how many warps there are.
template <bool CAREFUL, bool ENT, bool REST, int WARPS>
__device__ __forceinline__ Sums join_cta(Sums st, float c, int& join_turn, JoinScratch& js) {
  constexpr int WIDTH = WARPS <= V_WARPS ? V_WARPS : 2 * V_WARPS;
  Sums* const slots = js.warp[join_turn];
  join_turn ^= 1;
  st = join_lanes<32, CAREFUL, ENT, REST>(st, c);
  if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = st;
  __syncthreads();
  const int from = threadIdx.x % WIDTH;
  st = no_sums<REST>();
  if (from < WARPS) st = slots[from];
  return join_lanes<WIDTH, CAREFUL, ENT, REST>(st, c);
}
// The CTAs of a cluster may write to each other's shared memory once all of them run: each says so when it starts and
// waits for the others where it first needs them.  Without .aligned, which asks for warps whose threads execute the
// barrier together.
__device__ __forceinline__ void cluster_started() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_all_started() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier() {
  __syncwarp();
  cluster_started();
  cluster_all_started();
}
// How the CTAs that share a row exchange their sums: each writes its own into every CTA with a store that counts its bytes
// on that CTA's barrier, and waits until all have come in.  (A cluster barrier would also wait for the gradients written
// so far.)  Exchanges alternate between two places: a CTA sends the sums of exchange i + 2 only after those of i + 1 have
// come in from everyone, who had read exchange i's by then.
// A wait has a limit.  It cannot run out while the cluster's CTAs run; where one does, the whole CTA takes note (failed),
// sends and waits no more, and gives NaN for this row and those it has left.  The others then miss its sums and fail
// at their next exchange in turn, so that every CTA ends.  One that failed leaves last (see exchange_leave).
struct Exchange {
  uint32_t bar;                      // three mbarriers: two for sums in turn, one for alternatives (first CTA)
  uint32_t phase[2], top_phase;
  int turn;
  bool failed;                       // the same in the whole CTA
  unsigned long long limit_ns;
};
__device__ __forceinline__ void exchange_init(Exchange& ex, unsigned long long* bars, unsigned long long limit_ns) {
  ex.bar = smem_u32(bars);
  ex.phase[0] = ex.phase[1] = ex.top_phase = 0;
  ex.turn = 0;
  ex.failed = false;
  ex.limit_ns = limit_ns;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 3; ++i) mbar_init(ex.bar + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
}
// What the barrier counts has come in: one warp waits, all threads of the CTA agree on the outcome.  The clock is read
// rarely (a read takes about as long as the exchange, and the CTA would wait for it).
__device__ __forceinline__ bool exchange_wait(Exchange& ex, uint32_t bar, uint32_t phase) {
  bool ok = true;
  if (threadIdx.x < 32) {
    unsigned long long t0 = 0;
    unsigned spins = 0;
    while (!(ok = mbar_try_wait_cluster(bar, phase))) {
      if ((++spins & 31u) != 0u) continue;
      const unsigned long long now = globaltimer_ns();
      if (t0 == 0) t0 = now;
      else if (now - t0 > ex.limit_ns) break;
    }
  }
  ex.failed = __syncthreads_or(!ok);
  if (!ex.failed) mbar_try_wait_cluster(bar, phase);         // over by now: every thread acquires what came in
  return !ex.failed;
}
// At the end of the kernel: a CTA that failed may still be written to by others that have not, and stays until all of them
// have failed as well or are gone (the barrier counts those that ended), and what they sent has landed.
__device__ __forceinline__ void exchange_leave(const Exchange& ex) {
  if (!ex.failed) return;
  cluster_barrier();
  const unsigned long long t0 = globaltimer_ns();
  while (globaltimer_ns() - t0 < 2000000ull) __nanosleep(1000);
}
template <bool CAREFUL, bool ENT, bool REST>
__device__ __forceinline__ Sums join_parts(const Sums* cta, int parts, float c) {
  const int lane = threadIdx.x % V_MAX_SPLIT;
  Sums st = no_sums<REST>();
  if (lane < parts) st = cta[lane];
  return join_lanes<V_MAX_SPLIT, CAREFUL, ENT, REST>(st, c);
}
// The row's sums from this CTA's (in every thread of it), NaN if the exchange failed.
template <bool CAREFUL, bool ENT, bool REST>
__device__ __forceinline__ Sums exchange_sums(const Sums& own, int part, int parts, float c, Exchange& ex, JoinScratch& js) {
  const uint32_t bar = ex.bar + 8 * ex.turn;
  if (!ex.failed) {
    if (threadIdx.x == 0) mbar_expect_tx(bar, (uint32_t)parts * sizeof(Sums));
    __syncwarp();
    if ((int)threadIdx.x < parts) {
      asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                   ::"r"(map_to_cta(smem_u32(&js.cta[ex.turn][part]), threadIdx.x)), "r"(__float_as_uint(own.ref)),
                   "r"(__float_as_uint(own.s)), "r"(__float_as_uint(own.t)), "r"(__float_as_uint(own.l)),
                   "r"(map_to_cta(bar, threadIdx.x))
                   : "memory");
    }
    exchange_wait(ex, bar, ex.phase[ex.turn]);
  }
  if (ex.failed) return Sums{0.f, NAN, NAN, NAN};
  const Sums st = join_parts<CAREFUL, ENT, REST>(js.cta[ex.turn], parts, c);
  ex.phase[ex.turn] ^= 1;
  ex.turn ^= 1;
  return st;
}
__device__ __forceinline__ bool in_range(float s) { return s >= 0x1p-60f && s <= 0x1p120f; }
// REST: no bound below for l beside an ordinary s; what the walk's floor flushes there is nothing against s.  Nor has s one
// where it is 0 and the largest logit outside the list, ref then, is so far below the list that a whole vocabulary of it
// makes no share (a student whose other logits are masked).
template <bool REST>
__device__ __forceinline__ bool sums_ordinary(const Sums& st) {
  if (!REST) return in_range(st.s);
  return st.s == 0.f ? in_range(st.l) && st.ref + 20.f < st.t + SHARE_FLOOR : in_range(st.s) && st.l <= 0x1p120f;
}
static_assert(CAMERA_MAX_VOCAB <= 1 << 20, "2^20 tokens at most");

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
constexpr int V_BINS = 256;

// The key of an alternative back as its logit.
__device__ __forceinline__ float key_value(unsigned long long key) {
  const uint32_t k = (uint32_t)(key >> 32);
  return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// CAND: candidates kept in shared memory.  A CTA that shares its row with others has fewer to look through and needs room
// for the others' alternatives.
template <int CAND_, int SHARES_>
struct TopScratch {
  static constexpr int CAND = CAND_, SHARES = SHARES_;
  int hist[V_BINS];
  uint16_t active[SHARES];               // the shares that can hold an alternative
  alignas(16) unsigned long long cand[CAND];
  float w_max[V_WARPS], w_min[V_WARPS];
  int last_bin, n_bins, n_active, n_cand, count;
  uint32_t floor_key;                    // smallest of the active shares' maxima
};

// Calls f(index, value) for every element of the shares listed in sc.active[0 .. n_active).  Share u V_THREADS + t: vectors
// u V_THREADS + t of every chunk; the single elements of thread t belong to share t.
template <typename T, typename RG, typename SC, typename F>
__device__ __forceinline__ void for_active(const Row<T>& row, const SC& sc, F f) {
  constexpr int N = Elem<T>::N, BATCH = 4;
  const unsigned per = (unsigned)row_chunks<RG>(row.v_end - row.v_begin);
  const unsigned total = (unsigned)sc.n_active * per;
  for (unsigned q0 = threadIdx.x; q0 < total; q0 += BATCH * V_THREADS) {
    uint4 raw[BATCH];
    int at[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const unsigned q = q0 + u * V_THREADS;
      at[u] = -1;
      if (q < total) {
        const unsigned g = q / per;
        const int v = row.v_begin + sc.active[g] + (int)(q - g * per) * RG::CHUNK;
        if (v < row.v_end) { at[u] = row.vec_index(v); raw[u] = ld_stream(row.vec(v)); }
      }
    }
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      if (at[u] < 0) continue;
      float2 x[N / 2];
      Elem<T>::pairs(raw[u], x);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) { f(at[u] + 2 * i, x[i].x); f(at[u] + 2 * i + 1, x[i].y); }
    }
  }
  for (int q = threadIdx.x; q < sc.n_active; q += V_THREADS) {
    const int g = sc.active[q];
    if (g < row.head) f(g, to_f32<T>(row.p[g]));
    if (g < row.tail) f(row.tail_at + g, to_f32<T>(row.p[row.tail_at + g]));
  }
}
__device__ __forceinline__ int sum_cta(int v, int* total) {       // *total is 0 before and stays the sum until reset
  v = __reduce_add_sync(0xffffffffu, v);
  if ((threadIdx.x & 31) == 0 && v) atomicAdd(total, v);
  __syncthreads();
  return *total;
}

// The (up to) n elements of this CTA's part with the largest keys, logits of minus infinity left out, as
// sc.cand[0 .. sc.n_cand) in any order; at least n of them (if there are as many), possibly more.
// A share whose maximum is below the n-th largest of the shares' maxima holds none of the n largest elements, so only
// about n of the SHARES shares are read again (2 to 6 % of the row; one share a thread would make it 8 times as much).  A
// histogram of the maxima between their least and their largest finds the threshold; where its bins are too coarse (one
// logit far above the rest), bisection over the key bits does.  Where the elements at or above the threshold outgrow the
// candidate list (long runs of equal logits), the bisection goes on over the elements' 64-bit keys, which are all
// distinct.
template <typename T, typename RG, typename SC>
__device__ __noinline__ void collect_top(const Row<T> row, const float* own_max, int n, SC& sc) {
  constexpr int CAND = SC::CAND, PER = RG::PER;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float own[PER];
#pragma unroll
  for (int u = 0; u < PER; ++u) own[u] = own_max[u];
  static_assert(V_BINS <= V_THREADS, "one bin per thread to clear");
  if (tid < V_BINS) sc.hist[tid] = 0;
  if (tid == 0) { sc.n_active = 0; sc.n_cand = 0; sc.floor_key = 0xffffffffu; sc.last_bin = V_BINS - 1; }
  float hi = -INFINITY, lo = INFINITY;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    hi = fmaxf(hi, own[u]);
    if (own[u] > -INFINITY) lo = fminf(lo, own[u]);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
  }
  if (lane == 0) { sc.w_max[warp] = hi; sc.w_min[warp] = lo; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < V_WARPS; ++w) { hi = fmaxf(hi, sc.w_max[w]); lo = fminf(lo, sc.w_min[w]); }
  if (!(hi > -INFINITY)) return;                       // nothing but minus infinity in this part (uniform)
  const float range = hi - lo;
  const float scale = range > 0.f && range < FLT_MAX ? (V_BINS - 1) / range : 0.f;
  // falls as the maximum grows
  auto bin_of = [&](float m) { return min(V_BINS - 1, (int)((hi - m) * scale)); };
#pragma unroll
  for (int u = 0; u < PER; ++u)
    if (own[u] > -INFINITY) atomicAdd(&sc.hist[bin_of(own[u])], 1);
  __syncthreads();
  if (warp == 0) {
    int c[V_BINS / 32], sum = 0;
#pragma unroll
    for (int i = 0; i < V_BINS / 32; ++i) { c[i] = sc.hist[lane * (V_BINS / 32) + i]; sum += c[i]; }
    int before = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += v;
    }
    if (lane == 31) sc.n_bins = before;                // shares with anything in them, unless a bin reaches n
    before -= sum;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < V_BINS / 32; ++i) {
      if (before < n && before + c[i] >= n) { sc.last_bin = lane * (V_BINS / 32) + i; sc.n_bins = before + c[i]; }
      before += c[i];
    }
  }
  __syncthreads();
  const int last_bin = sc.last_bin, n_active = sc.n_bins;
  uint32_t from = KEY_NEG_INF + 1;                     // shares with a maximum of at least this key, in a bin up to last_bin
  if (n_active > 2 * n + 64) {
    uint32_t to = 0xffffffffu;
    while (to - from > 1) {                            // at most 32 rounds
      const uint32_t mid = from + (to - from) / 2;
      __syncthreads();
      if (tid == 0) sc.count = 0;
      __syncthreads();
      int c = 0;
#pragma unroll
      for (int u = 0; u < PER; ++u) c += value_key(own[u]) >= mid;
      const int cnt = sum_cta(c, &sc.count);
      if (cnt >= n) { from = mid; if (cnt <= n + n / 4) break; } else to = mid;
    }
  }
  uint32_t least = 0xffffffffu;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    const uint32_t key = value_key(own[u]);
    if (own[u] > -INFINITY && key >= from && bin_of(own[u]) <= last_bin) {
      sc.active[atomicAdd(&sc.n_active, 1)] = (uint16_t)(u * V_THREADS + tid);
      least = min(least, key);
    }
  }
  if (least != 0xffffffffu) atomicMin(&sc.floor_key, least);
  __syncthreads();
  // fewer shares than n with anything in them: their elements below the shares' maxima count as well
  unsigned long long klo = (unsigned long long)(n_active < n ? KEY_NEG_INF + 1 : sc.floor_key) << 32, khi = ~0ull;
  for (int attempt = 0; attempt < 2; ++attempt) {
    for_active<T, RG>(row, sc, [&](int i, float x) {
      const unsigned long long k = rank_key(x, i);
      if (k >= klo) {
        const int at = atomicAdd(&sc.n_cand, 1);
        if (at < CAND) sc.cand[at] = k;
      }
    });
    __syncthreads();
    if (sc.n_cand <= CAND) return;
    // More than fit: raise klo until n .. CAND elements are left.  64 halvings of the key range always get there.
    for (int it = 0; it < 64; ++it) {
      const unsigned long long mid = klo + (khi - klo) / 2;
      __syncthreads();
      if (tid == 0) { sc.count = 0; sc.n_cand = 0; }
      __syncthreads();
      int c = 0;
      for_active<T, RG>(row, sc, [&](int i, float x) { c += rank_key(x, i) >= mid; });
      const int all = sum_cta(c, &sc.count);
      if (all >= n) { klo = mid; if (all <= CAND) break; } else khi = mid;
    }
    __syncthreads();
  }
  if (tid == 0) sc.n_cand = CAND;        // only if the logits changed while they were read
  __syncthreads();
}
// How many of the n keys are larger than k.
__device__ __forceinline__ int rank_among(const unsigned long long* keys, int n, unsigned long long k) {
  int rank = 0, j = 0;
  for (; j + 4 <= n; j += 4) {
    const ulonglong2 a = *reinterpret_cast<const ulonglong2*>(keys + j), b = *reinterpret_cast<const ulonglong2*>(keys + j + 2);
    rank += (a.x > k) + (a.y > k) + (b.x > k) + (b.y > k);
  }
  for (; j < n; ++j) rank += keys[j] > k;
  return rank;
}

struct LogprobArgs {
  const void* logits;
  long long ld;
  int rows, vocab, top_n;
  int lg;                   // 2^lg CTAs share a row
  float c, inv_tau;         // log2(e) / temperature, 1 / temperature
  unsigned long long wait_limit_ns;
  const long long* targets;
  float *logprob, *entropy, *top_logprob;
  int* top_idx;
};

// How log-probabilities and probabilities come from a row's logits: log2 q_v = x c - k, or for a row walked carefully
// (x - m) c - log2s.
struct Softmax {
  float c, inv_tau, k, m, log2s;
  bool careful;
  __device__ __forceinline__ Softmax(const Sums& st, bool careful_, float c_, float inv_tau_) : c(c_), inv_tau(inv_tau_), careful(careful_) {
    log2s = log2f(st.s);
    m = st.ref;
    k = st.ref + log2s;
  }
  __device__ __forceinline__ float q(float x) const { return ex2(careful ? (x - m) * c - log2s : fmaf(x, c, -k)); }
  __device__ __forceinline__ float logprob(float x) const {
    if (careful) return (x - m) * inv_tau - log2s * LN2;
    const float d = fmaf(x, c, -m);
    return d < -1e30f ? x * inv_tau - m * LN2 : (d - log2s) * LN2;     // x c may be beyond fp32's range; log2s does not count
  }
};

// A CTA, or (SPLIT) the CTAs of a cluster together, take row after row: blockIdx.x is the CTA's part of the row,
// blockIdx.y its first row.  Two CTAs an SM with ring chunks of 32 KB: one selects alternatives while the other
// reads.  4095 rows of 151936 bf16 logits with entropy take 227 to 241 us (5.2 to 5.5 TB/s of logits), 2048 such rows with
// 64 alternatives 152 us; one row with 8 alternatives 10.6 us of the GPU, 13.9 us a call.
template <typename T, bool ENT, bool TOP, bool SPLIT>
__global__ void __launch_bounds__(V_THREADS, 2) k_token_logprobs(const LogprobArgs a) {
  using RG = RingStream;
  extern __shared__ __align__(RING_ALIGN) uint8_t ring[];
  __shared__ JoinScratch js;
  using Scratch = TopScratch<SPLIT ? 512 : 1024, RG::PER * V_THREADS>;
  __shared__ typename std::conditional<TOP, Scratch, int>::type sc_raw;
  unsigned long long* const merged = reinterpret_cast<unsigned long long*>(ring + RG::BYTES);   // TOP && SPLIT: the parts' best; 0: none
  const int lg = SPLIT ? a.lg : 0, part = SPLIT ? blockIdx.x : 0, parts = 1 << lg;
  const int tid = threadIdx.x;
  Exchange ex;
  ex.failed = false;
  if (SPLIT) {
    exchange_init(ex, js.bars, a.wait_limit_ns);
    cluster_started();
  }
  bool started = !SPLIT;
  Feed<T, RG> feed;
  feed.logits = static_cast<const T*>(a.logits);
  feed.ld = a.ld; feed.weight = nullptr;
  feed.rows = a.rows; feed.stride = gridDim.y; feed.vocab = a.vocab; feed.part = part; feed.lg = lg;
  feed.dst0 = smem_u32(ring) + tid * 16;
  feed.begin(blockIdx.y);
#pragma unroll
  for (int i = 0; i < RG::SLOTS; ++i) feed.issue();
  int at = 0, join_turn = 0;
  const bool first = part == 0 && tid == 0;
  long long target = first && a.logprob && (int)blockIdx.y < a.rows ? a.targets[blockIdx.y] : -1;
  for (int r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const Row<T> row(static_cast<const T*>(a.logits) + r * a.ld, a.vocab, part, lg);
    // the target's logit, and the next row's target, on their way during the walk
    const bool wanted = target >= 0 && target < a.vocab;
    const float x_target = wanted ? to_f32<T>(row.p[target]) : 0.f;
    if (first && a.logprob && r + (int)gridDim.y < a.rows) target = a.targets[r + gridDim.y];
    float top[RG::PER];
    Sums st = walk_row<T, RG, ENT, false, TOP>(row, a.c, feed, ring, at, nullptr, nullptr, 0, top);
    st = join_cta<false, ENT, false, V_WARPS>(st, a.c, join_turn, js);
    if (SPLIT) {
      if (!started) { cluster_all_started(); started = true; }
      st = exchange_sums<false, ENT, false>(st, part, parts, a.c, ex, js);
    }
    const bool careful = !ex.failed && !sums_ordinary<false>(st);
    if (careful) {
      st = join_cta<true, ENT, false, V_WARPS>(walk_careful<T, ENT, false>(row, a.c, nullptr, nullptr, 0), a.c, join_turn, js);
      if (SPLIT) st = exchange_sums<true, ENT, false>(st, part, parts, a.c, ex, js);
    }
    const Softmax sm(st, careful, a.c, a.inv_tau);
    if (first) {
      if (a.logprob) a.logprob[r] = !wanted ? 0.f : st.s == 0.f ? -INFINITY : sm.logprob(x_target);
      if (ENT) a.entropy[r] = st.s == 0.f ? 0.f : (sm.log2s - st.t / st.s) * LN2;
    }
    if constexpr (TOP) {
      Scratch& sc = sc_raw;
      bool usable = st.s > 0.f;                          // false for a NaN
      int n_cand = 0, n_out = 0;
      const unsigned long long* cand = sc.cand;
      if (usable) {
        collect_top<T, RG, Scratch>(row, top, a.top_n, sc);
        __syncthreads();
        n_cand = n_out = sc.n_cand;
        if (SPLIT) {                                     // this part's best n go to the first CTA, n from every part
          const uint32_t bar = ex.bar + 16;
          if (first) mbar_expect_tx(bar, (uint32_t)(parts * a.top_n * 8));
          for (int q = tid; q < max(n_cand, a.top_n); q += V_THREADS) {
            const unsigned long long k = q < n_cand ? cand[q] : 0ull;
            const int rank = q < n_cand ? rank_among(cand, n_cand, k) : q;
            if (rank < a.top_n) {
              asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];"
                           ::"r"(map_to_cta(smem_u32(&merged[part * a.top_n + rank]), 0)), "l"(k), "r"(map_to_cta(bar, 0))
                           : "memory");
            }
          }
          cand = merged;
          n_cand = n_out = parts * a.top_n;
          // the next row's alternatives come after its sums, which the others have not had from this CTA before it is
          // through with these
          if (part == 0) {
            if (!exchange_wait(ex, bar, ex.top_phase)) { usable = false; n_cand = n_out = 0; }
            ex.top_phase ^= 1;
          }
        }
      }
      if (part == 0) {
        int* const out_i = a.top_idx + (long long)r * a.top_n;
        float* const out_v = a.top_logprob + (long long)r * a.top_n;
        for (int q = tid; q < n_cand; q += V_THREADS) {
          const unsigned long long k = cand[q];
          if (SPLIT && k == 0) continue;
          const int rank = rank_among(cand, n_cand, k);
          if (rank < a.top_n) {
            out_i[rank] = (int)~(uint32_t)k;
            out_v[rank] = sm.logprob(key_value(k));
          }
        }
        if (SPLIT && usable) {                           // how many there are in all
          int have = 0;
          for (int q = tid; q < n_cand; q += V_THREADS) have += cand[q] != 0;
          n_out = have;
#pragma unroll
          for (int o = 16; o; o >>= 1) n_out += __shfl_xor_sync(0xffffffffu, n_out, o);
          if ((tid & 31) == 0) sc.hist[tid >> 5] = n_out;
          __syncthreads();
          n_out = 0;
          for (int w = 0; w < V_WARPS; ++w) n_out += sc.hist[w];
        }
        for (int q = n_out + tid; q < a.top_n; q += V_THREADS) {
          out_i[q] = -1;
          out_v[q] = st.s == 0.f || usable ? -INFINITY : NAN;
        }
      }
    }
  }
  if (SPLIT && !started) cluster_all_started();
  if (SPLIT) exchange_leave(ex);
}

// ---------------------------------------------------------------------------------------------- distillation
// Teacher: a list of k tokens with log-probabilities.  p is their softmax over the list, or, with the rest as one more
// class (TAIL), p = exp(logprob) and rest = 1 - sum p.  Student: q = softmax(x / temperature) over the vocabulary.
//   loss   = sum p (ln p - ln q) [+ rest (ln rest - ln R)],  R = the student's share outside the list
//   d loss / d x_v = (M q_v - p_v) / temperature on the list,  M q_v / temperature outside,  M = sum p [+ rest]; with the
//   rest as a class the latter is q_v (M - rest / R) / temperature, because a token outside moves the rest's share as well.  It is formed as
//   (q_v / R) (M R - rest): the student's distribution over the tokens outside, whose weights are of ordinary size however
//   small R is, times a factor that cannot overflow.
// M is 1 for an ordinary list, 0 for one without an entry (its loss is 0 whatever the logits), above 1 where the listed
// probabilities add to more (rest is 0 then), and sum p alone where the student has nothing outside and the rest's term is
// dropped.
// R is summed over the tokens outside, not formed as 1 - Q: once the student is right, R is small and the difference would
// be noise.  It has its own reference, so that it holds down to SHARE_FLOOR; below that (float64's normal range, in which
// the term is a number) the student counts as having nothing outside.  The 16-byte vectors that hold listed tokens are marked, left out by the walk and summed apart.  The k terms of the list are taken in double: they are
// few, and the loss is a difference of nearly equal logarithms by the end of the training.
struct DistillArgs {
  const void* logits;
  long long ld;
  int rows, vocab, k;
  int lg;                   // 2^lg CTAs share a row
  int in_place;             // the gradient takes the logits' room
  int mark_words;           // of one set of marks: a bit per vector of a part, rounded up to whole chunks
  float c, inv_tau;
  unsigned long long wait_limit_ns;
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
  double mass, rest;                  // sum of p; NaN if the list holds one
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
    if (i < 0 || i >= a.vocab) {        // no entry; a NaN stays (-1 / NaN: the teacher's row held one)
      i = -1;
      if (lp == lp) lp = -INFINITY;
    }
    tl.idx[j] = i;
    tl.log_p[j] = lp;
    top = fmaxf(top, lp);
  }
  double sum = 0.0;
  if (TAIL) {
    for (int j = lane; j < a.k; j += 32) {
      const float p = expf(tl.log_p[j]);
      tl.p[j] = p;
      sum += (double)p;                 // 1 - sum would lose the rest's digits in fp32
    }
    sum = warp_sum(sum);
    if (lane == 0) {
      tl.mass = sum;
      tl.rest = 1.0 - sum < 0.0 ? 0.0 : 1.0 - sum;                    // keeps a NaN
    }
  } else {
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == -INFINITY) top = 0.f;                                  // nothing on the list
    for (int j = lane; j < a.k; j += 32) sum += (double)expf(tl.log_p[j] - top);
    sum = warp_sum(sum);
    const float log_sum = logf((float)sum);
    for (int j = lane; j < a.k; j += 32) {
      const float lp = tl.log_p[j] - top - log_sum;
      tl.p[j] = sum > 0.0 || sum != sum ? expf(lp) : 0.f;
      tl.log_p[j] = lp;
    }
    if (lane == 0) {
      tl.mass = sum > 0.0 ? 1.0 : sum;
      tl.rest = 0.0;
    }
  }
}

// Marks the part's vectors that hold listed tokens and sums them, listed and other elements apart, each against their own
// reference (one warp).  Each such vector is looked after by its first entry on the list.
template <typename T>
__device__ __forceinline__ Sums mark_list(const Row<T>& row, const TeacherList& tl, int k, float c, uint32_t* mark) {
  constexpr int N = Elem<T>::N;
  Sums st{REF_FLOOR, 0.f, REF_FLOOR, 0.f};
  float seen = -INFINITY;
  for (int j = threadIdx.x & 31; j < k; j += 32) {
    const int i = tl.idx[j];
    if (i < row.first || i >= row.tail_at) continue;
    const int v = (i - row.first) / N, i0 = row.vec_index(v);
    if (v < row.v_begin || v >= row.v_end) continue;
    const uint4 raw = ld_stream(row.vec(v));
    uint32_t listed = 0;
    bool mine = true;
    for (int l = 0; l < k; ++l) {
      const unsigned off = (unsigned)(tl.idx[l] - i0);
      if (off < (unsigned)N) {
        listed |= 1u << off;
        mine &= l >= j;
      }
    }
    if (!mine) continue;
    const int at = v - row.v_begin;
    atomicOr(mark + (at >> 5), 1u << (at & 31));
    float2 x[N / 2];
    Elem<T>::pairs(raw, x);
    float m = -INFINITY, m_l = -INFINITY;
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const float v_q = q & 1 ? x[q >> 1].y : x[q >> 1].x;
      if ((listed >> q) & 1u) m_l = fmaxf(m_l, v_q); else m = fmaxf(m, v_q);
    }
    m *= c;
    m_l *= c;
    seen = fmaxf(seen, m);
    if (m > st.ref) raise<false, false>(st, m, c);
    if (m_l > st.t) raise_listed<false>(st, m_l, c);
#pragma unroll
    for (int q = 0; q < N; ++q) {
      const bool on = (listed >> q) & 1u;
      const float e = ex2(fmaf(q & 1 ? x[q >> 1].y : x[q >> 1].x, c, on ? -st.t : -st.ref));
      if (on) st.l += e; else st.s += e;
    }
  }
  if (st.s == 0.f) st.ref = fmaxf(seen, -FLT_MAX);
  return st;
}
template <typename T>
__device__ __forceinline__ void unmark_list(const Row<T>& row, const TeacherList& tl, int k, uint32_t* mark) {
  for (int j = threadIdx.x & 31; j < k; j += 32) {
    const int i = tl.idx[j];
    if (i < row.first || i >= row.tail_at) continue;
    const int v = (i - row.first) / Row<T>::N;
    if (v >= row.v_begin && v < row.v_end) mark[(v - row.v_begin) >> 5] = 0u;
  }
}
template <typename T>
__device__ __forceinline__ void store_vec(T* o, const float2* x, bool aligned) {
  constexpr int N = Elem<T>::N;
  if (aligned) {
    __stcs(reinterpret_cast<uint4*>(o), Elem<T>::pack(x));
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) { o[2 * i] = Elem<T>::put(x[i].x); o[2 * i + 1] = Elem<T>::put(x[i].y); }
  }
}
template <typename T>
__device__ __forceinline__ void zero_row(const Row<T>& row, T* out) {
  const int tid = threadIdx.x;
  const bool aligned = (reinterpret_cast<uintptr_t>(out + row.first) & 15) == 0;
  const float2 zero[Elem<T>::N / 2] = {};
  if (tid < row.head) out[tid] = Elem<T>::put(0.f);
  if (tid < row.tail) out[row.tail_at + tid] = Elem<T>::put(0.f);
  for (int v = row.v_begin + tid; v < row.v_end; v += V_THREADS) store_vec<T>(out + row.vec_index(v), zero, aligned);
}

// Writes scale * q_v (or 0: blank) for every element of the part, whose vectors arrive in the ring from offset `at` on
// (moved past them).
template <typename T, typename RG>
__device__ __forceinline__ void write_row(const Row<T>& row, T* out, const Softmax& sm, float scale, bool blank, Feed<T, RG>& feed,
                                          const uint8_t* ring, int& at) {
  constexpr int N = Elem<T>::N;
  const int tid = threadIdx.x;
  float single[2] = {0.f, 0.f};
  if (tid < row.head) single[0] = to_f32<T>(row.p[tid]);
  if (tid < row.tail) single[1] = to_f32<T>(row.p[row.tail_at + tid]);
  const bool aligned = (reinterpret_cast<uintptr_t>(out + row.first) & 15) == 0;
  const float2 c2 = make_float2(sm.c, sm.c), k2 = make_float2(-sm.k, -sm.k), s2 = make_float2(scale, scale);
  const uint8_t* const mine = ring + tid * 16;
  T* o = out + row.vec_index(row.v_begin + tid);
  const bool plain = aligned && !blank && !sm.careful;
  int left = row.v_end - row.v_begin;
  do {
    uint4 raw[RG::PER];
    Feed<T, RG>::wait();
    read_chunk<RG>(mine, at, raw);
    at = next_chunk<RG>(at);
    if (plain && left >= RG::CHUNK) {        // no branch among the vectors: their exponentials overlap
#pragma unroll
      for (int u = 0; u < RG::PER; ++u) {
        float2 x[N / 2];
        Elem<T>::pairs(raw[u], x);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
          const float2 d = fma2(x[i], c2, k2);
          x[i] = mul2(make_float2(ex2(d.x), ex2(d.y)), s2);
        }
        raw[u] = Elem<T>::pack(x);
      }
#pragma unroll
      for (int u = 0; u < RG::PER; ++u) __stcs(reinterpret_cast<uint4*>(o + (size_t)u * V_THREADS * N), raw[u]);
    } else {
#pragma unroll
      for (int u = 0; u < RG::PER; ++u) {
        if (left <= u * V_THREADS + tid) continue;
        float2 x[N / 2];
        Elem<T>::pairs(raw[u], x);
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
          x[i] = blank ? make_float2(0.f, 0.f) : make_float2(scale * sm.q(x[i].x), scale * sm.q(x[i].y));
        store_vec<T>(o + (size_t)u * V_THREADS * N, x, aligned);
      }
    }
    o += (size_t)RG::CHUNK * N;
    feed.issue();
    left -= RG::CHUNK;
  } while (left > 0);
  if (tid < row.head) out[tid] = Elem<T>::put(blank ? 0.f : scale * sm.q(single[0]));
  if (tid < row.tail) out[row.tail_at + tid] = Elem<T>::put(blank ? 0.f : scale * sm.q(single[1]));
}

// A CTA, or (SPLIT) the CTAs of a cluster together, take row after row, like k_token_logprobs.  STEP sends every row
// through the ring twice, once to sum it and once to write the gradient; the second time it comes from L2 (see Feed).  The
// last warp looks after the teacher's lists: while the others sum a row it brings in the next row's, and while they write
// the gradient it forms the loss.  4096 rows of 151936 bf16 logits with 64 entries: 584 us; reading the logits and writing the
// gradient once would be 381 us, the rest is that a CTA sums and writes in turn, with a join in between.  250 rows of 32003 fp32
// logits, loss alone: 12.3 us of the GPU, 13.6 us a call, most of it the first row's list, sums and logarithms one after the other.
constexpr int VD_THREADS = V_THREADS + 32;
constexpr int VD_LISTS = 3;

template <typename T, int MODE, bool TAIL, bool SPLIT>
__global__ void __launch_bounds__(VD_THREADS, 2) k_distill(const DistillArgs a) {
  constexpr bool STATS = MODE != DISTILL_BACKWARD;
  constexpr bool GRAD = MODE != DISTILL_FORWARD;
  constexpr bool REST = STATS && TAIL;
  using RG = RingDistill;
  extern __shared__ __align__(RING_ALIGN) uint8_t ring[];     // the ring, then (REST) two sets of marks
  __shared__ JoinScratch js;
  __shared__ TeacherList lists[VD_LISTS];
  const int lg = SPLIT ? a.lg : 0, part = SPLIT ? blockIdx.x : 0, parts = 1 << lg;
  const int tid = threadIdx.x;
  const bool lister = tid >= V_THREADS;
  const T* const logits = static_cast<const T*>(a.logits);
  uint32_t* const marks = reinterpret_cast<uint32_t*>(ring + RG::BYTES);
  Exchange ex;
  ex.failed = false;
  if (SPLIT) {
    exchange_init(ex, js.bars, a.wait_limit_ns);
    cluster_started();
  }
  bool started = !SPLIT;
  if (REST)
    for (int i = tid; i < 2 * a.mark_words; i += VD_THREADS) marks[i] = 0u;
  Feed<T, RG> feed;
  feed.logits = logits;
  feed.ld = a.ld; feed.weight = GRAD ? a.d_loss : nullptr;
  feed.rows = a.rows; feed.stride = gridDim.y; feed.vocab = a.vocab; feed.part = part; feed.lg = lg;
  feed.dst0 = smem_u32(ring) + tid * 16;
  feed.begin(lister ? a.rows : (int)blockIdx.y, MODE == DISTILL_STEP);
#pragma unroll
  for (int i = 0; i < RG::SLOTS; ++i) feed.issue();
  if (GRAD && !lister) {                              // rows that do not count: their logits are not looked at
    for (int r = blockIdx.y; r < a.rows; r += gridDim.y) {
      if (a.d_loss[r] != 0.f) continue;
      zero_row<T>(Row<T>(logits + r * a.ld, a.vocab, part, lg), static_cast<T*>(a.grad) + r * a.ld_grad);
      if (STATS && part == 0 && tid == 0) a.loss[r] = 0.f;
    }
  }
  Sums listed{REF_FLOOR, 0.f, REF_FLOOR, 0.f}, listed_next = listed;    // the lister's: of the vectors with listed tokens
  auto bring_list = [&](int r, TeacherList& tl, uint32_t* mark) {
    if (r >= a.rows) return;
    const Row<T> row(logits + r * a.ld, a.vocab, part, lg);
    load_teacher<TAIL>(a, r, tl);
    __syncwarp();
    for (int j = tid & 31; j < a.k; j += 32) {
      const int i = tl.idx[j];
      tl.x[j] = i >= 0 ? to_f32<T>(row.p[i]) : 0.f;
    }
    if (REST) listed_next = mark_list<T>(row, tl, a.k, a.c, mark);
  };
  RowWalk walk;
  walk.begin(feed.weight, a.rows, blockIdx.y);
  int r = walk.next(feed.weight, a.rows, gridDim.y);
  __syncthreads();
  if (lister) bring_list(r, lists[0], marks);
  if (!STATS && SPLIT && a.in_place) {
    // nobody writes to the first row before every CTA has its listed logits
    cluster_all_started();
    started = true;
    cluster_barrier();
  } else {
    __syncthreads();
  }
  int at = 0, turn = 0, join_turn = 0, list = 0;
  while (r < a.rows) {
    const int r_next = walk.next(feed.weight, a.rows, gridDim.y);
    const Row<T> row(logits + r * a.ld, a.vocab, part, lg);
    const TeacherList& tl = lists[list];
    const int list_next = list + 1 == VD_LISTS ? 0 : list + 1;
    uint32_t* const mark = marks + turn * a.mark_words;
    Sums st = no_sums<REST>();
    bool careful = false, empty;
    if (lister) {
      listed = listed_next;
      bring_list(r_next, lists[list_next], marks + (turn ^ 1) * a.mark_words);
    }
    if (STATS) {
      if (!lister) st = walk_row<T, RG, false, REST, false>(row, a.c, feed, ring, at, mark, tl.idx, a.k, nullptr);
      else if (REST) st = listed;
      st = join_cta<false, false, REST, V_WARPS + 1>(st, a.c, join_turn, js);
      if (SPLIT) {
        if (!started) { cluster_all_started(); started = true; }
        st = exchange_sums<false, false, REST>(st, part, parts, a.c, ex, js);
      }
      // a reference that large would swallow digits of log2 s where the two are added (Softmax::k)
      careful = !ex.failed && (!sums_ordinary<REST>(st) || (st.s != 0.f && fabsf(st.ref) > 4096.f) || (REST && fabsf(st.t) > 4096.f));
      if (careful) {
        st = no_sums<REST>();
        if (!lister) st = walk_careful<T, false, REST>(row, a.c, mark, tl.idx, a.k);
        st = join_cta<true, false, REST, V_WARPS + 1>(st, a.c, join_turn, js);
        if (SPLIT) st = exchange_sums<true, false, REST>(st, part, parts, a.c, ex, js);
      }
    }
    // of the whole row; with the rest as a class from both sums
    Sums all = st;
    if (REST) {
      all.ref = fmaxf(st.ref, st.t);
      const float unit = careful ? a.c : 1.f;
      all.s = scale_down(st.s, (st.ref - all.ref) * unit) + scale_down(st.l, (st.t - all.ref) * unit);
    }
    Softmax sm(all, careful, a.c, a.inv_tau);
    // Outside the list the gradient is `scale` times the weight by `out`; M is `mass`
    Softmax out = sm;
    float mass = (float)tl.mass, scale = mass;
    if (STATS) {
      // no distribution: every logit minus infinity, or all of them beyond fp32's range once scaled
      empty = all.s == 0.f || (careful && all.ref * a.c < -FLT_MAX);
      const float to_rest = st.ref - all.ref;                            // REST: ln R = this (scaled) + ln(st.s / all.s)
      const bool rest = REST && tl.rest != 0.0 &&
                        !((careful ? to_rest * a.c : to_rest) + log2f(st.s) - sm.log2s < SHARE_FLOOR);       // a NaN counts
      if (rest) {
        mass = (float)(tl.mass + tl.rest);
        out = Softmax(st, careful, a.c, a.inv_tau);
        scale = mass * scale_down(st.s / all.s, careful ? to_rest * a.c : to_rest) - (float)tl.rest;
      }
      if (lister) {
        if (REST) unmark_list<T>(row, tl, a.k, mark);
        if (part == 0) {
          double loss = 0.0;
          for (int j = tid & 31; j < a.k; j += 32) {
            const float p = tl.p[j], x = tl.x[j];
            if (tl.idx[j] < 0 || p == 0.f) continue;
            const float d = careful ? (x - sm.m) * a.inv_tau * LOG2E : fmaf(x, a.c, -sm.m);
            loss += (double)p * ((double)tl.log_p[j] - ((double)d - (double)sm.log2s) * 0.6931471805599453);
          }
          loss = warp_sum(loss);
          if (tid == V_THREADS) {
            if (rest)
              loss += tl.rest * (log(tl.rest) - log((double)st.s / (double)all.s) -
                                 (double)to_rest * (careful ? (double)a.inv_tau : 0.6931471805599453));
            if (tl.mass != tl.mass || all.s != all.s) loss = NAN;       // also where no entry brought it in
            a.loss[r] = empty ? 0.f : (float)loss;
            if (MODE == DISTILL_FORWARD) {
              const float to_ln = careful ? a.inv_tau : LN2;
              if (a.lse) a.lse[r] = empty ? -INFINITY : sm.m * to_ln + sm.log2s * LN2;
              if (TAIL && a.log_tail) a.log_tail[r] = empty || st.s == 0.f ? -INFINITY : st.ref * to_ln + log2f(st.s) * LN2;
            }
          }
        }
      }
    } else {
      const float lse = a.lse[r];
      empty = lse == -INFINITY;
      sm.k = out.k = lse * LOG2E;
      if (TAIL && tl.rest != 0.0) {
        const float lt = a.log_tail[r], d = (lt - lse) * LOG2E;
        if (!(d < SHARE_FLOOR)) {
          mass = (float)(tl.mass + tl.rest);
          out.k = lt * LOG2E;
          scale = mass * ex2(d) - (float)tl.rest;
        }
      }
    }
    if (GRAD) {
      // In place: the barriers so far have seen every CTA of the row read its listed logits.
      T* const grad = static_cast<T*>(a.grad) + r * a.ld_grad;
      const float w = a.d_loss[r] * a.inv_tau;
      const float on_list = tid < a.k ? w * (mass * sm.q(tl.x[tid]) - tl.p[tid]) : 0.f;
      if (!lister) {
        write_row<T, RG>(row, grad, out, w * scale, empty, feed, ring, at);
      }
      if (!STATS && SPLIT && a.in_place) cluster_barrier(); else __syncthreads();
      if (tid < a.k && !empty) {
        const int i = tl.idx[tid];
        if (i >= 0 && row.holds(i)) grad[i] = Elem<T>::put(on_list);
      }
    }
    r = r_next;
    turn ^= 1;
    list = list_next;
  }
  if (SPLIT && !started) cluster_all_started();
  if (SPLIT) exchange_leave(ex);
}

// ------------------------------------------------------------------------------------------------ launches
// CTAs that share a row when there are few: as many as keep the grid within two CTAs an SM and two vectors a thread.
int split_for(int rows, int n_vec, int sms) {
  int lg = 0;
  while (1 << lg < V_MAX_SPLIT && (long long)rows << (lg + 1) <= 2ll * sms && n_vec >> lg >= 4 * V_THREADS) ++lg;
  return lg;
}

// Clusters of 2^lg CTAs that run at one time (a cluster needs SMs of one GPC, so they do not always fill the GPU).  Kept per
// kernel, device and size of cluster for the last amount of shared memory asked about (bytes << 32 | clusters); an answer
// of the driver that is none is not kept.
template <auto KERN>
int clusters_at_once(cudaLaunchConfig_t& cfg, int lg) {
  static std::atomic<unsigned long long> known[KNOWN_DEVICES][V_MAX_LG + 1];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 1; }
  const bool keep = dev < KNOWN_DEVICES;
  const unsigned long long seen = keep ? known[dev][lg].load(std::memory_order_relaxed) : 0;
  if (seen != 0 && seen >> 32 == cfg.dynamicSmemBytes) return (int)(seen & 0xffffffffu);
  if (cudaOccupancyMaxActiveClusters(&n, KERN, &cfg) != cudaSuccess || n < 1) { cudaGetLastError(); return 1; }
  if (keep) known[dev][lg].store((unsigned long long)cfg.dynamicSmemBytes << 32 | (unsigned)n, std::memory_order_relaxed);
  return n;
}

// MOST: the most shared memory a launch of this kernel takes.
template <auto KERN, int MOST, typename A>
cudaError_t launch_rows(const A& args, int threads, int smem, int sms, cudaStream_t st) {
  const cudaError_t e = allow_smem<KERN, MOST>();
  if (e != cudaSuccess) return e;
  const int split = 1 << args.lg;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)split, (unsigned)args.rows);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)split; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = split > 1 ? 1 : 0;
  // two CTAs fit an SM (one where long rows need more marks); each walks rows until none is left
  int clusters = 2 * sms / split;
  if (split > 1 && args.rows > clusters / 2) clusters = clusters_at_once<KERN>(cfg, args.lg);
  if (args.rows > clusters) cfg.gridDim.y = (unsigned)clusters;
  return cudaLaunchKernelEx(&cfg, KERN, args);
}

template <typename T, bool ENT, bool TOP>
cudaError_t launch_logprobs(LogprobArgs& a, cudaStream_t st) {
  const int sms = sm_count();
  a.lg = split_for(a.rows, a.vocab / Elem<T>::N, sms);
  constexpr int RING = RingStream::BYTES, MOST = RING + (TOP ? V_MAX_SPLIT * CAMERA_MAX_TOP * 8 : 0);
  return a.lg == 0 ? launch_rows<k_token_logprobs<T, ENT, TOP, false>, RING>(a, V_THREADS, RING, sms, st)
                   : launch_rows<k_token_logprobs<T, ENT, TOP, true>, MOST>(a, V_THREADS, RING + (a.top_n * 8 << a.lg), sms, st);
}
template <typename T>
cudaError_t launch_logprobs(LogprobArgs& a, cudaStream_t st) {
  if (a.entropy) return a.top_n ? launch_logprobs<T, true, true>(a, st) : launch_logprobs<T, true, false>(a, st);
  return a.top_n ? launch_logprobs<T, false, true>(a, st) : launch_logprobs<T, false, false>(a, st);
}

// Words of one set of marks for parts of n_vec >> lg vectors, or one more.
constexpr int mark_words(int n_vec, int lg) { return ((n_vec >> lg) + RingDistill::CHUNK) / RingDistill::CHUNK * (RingDistill::CHUNK / 32); }

template <typename T, int MODE, bool TAIL>
cudaError_t launch_distill(DistillArgs& a, cudaStream_t st) {
  constexpr bool REST = TAIL && MODE != DISTILL_BACKWARD;
  const int sms = sm_count(), n_vec = a.vocab / Elem<T>::N;
  a.lg = split_for(a.rows, n_vec, sms);
  // A step reads its rows again from L2: two CTAs share a row where the rows of all CTAs would not stay there beside the
  // gradients on their way out (4096 rows of 151936 bf16 logits, 90 MB in flight: 602 us unshared, 584 us in pairs; in
  // fours 817 us, the CTAs then wait for each other more often than the reads gain).  The loss alone is as fast either way
  // and takes the same split, so that both calls give the same bits.
  if (MODE != DISTILL_BACKWARD && a.lg == 0 && 2ll * sms * n_vec * 16 > STEP_L2_BYTES) a.lg = 1;
  a.mark_words = REST ? mark_words(n_vec, a.lg) : 0;
  const int smem = RingDistill::BYTES + 8 * a.mark_words;
  constexpr int MOST = RingDistill::BYTES + (REST ? 8 * mark_words(CAMERA_MAX_VOCAB / Elem<T>::N, 0) : 0);
  return a.lg == 0 ? launch_rows<k_distill<T, MODE, TAIL, false>, MOST>(a, VD_THREADS, smem, sms, st)
                   : launch_rows<k_distill<T, MODE, TAIL, true>, MOST>(a, VD_THREADS, smem, sms, st);
}
template <int MODE>
cudaError_t launch_distill(DistillArgs& a, int dtype, bool tail, cudaStream_t st) {
  if (dtype == CAMERA_BF16)
    return tail ? launch_distill<__nv_bfloat16, MODE, true>(a, st) : launch_distill<__nv_bfloat16, MODE, false>(a, st);
  return tail ? launch_distill<float, MODE, true>(a, st) : launch_distill<float, MODE, false>(a, st);
}

int check_logits(const void* logits, int dtype, int64_t ld, int64_t n_rows, int32_t vocab, float temperature) {
  if (dtype != CAMERA_F32 && dtype != CAMERA_BF16) return CAMERA_ERR_INVALID_ARG;
  if (n_rows < 0 || vocab < 1 || ld < vocab || !(temperature > 0.f) || isinf(temperature) || isinf(LOG2E / temperature))
    return CAMERA_ERR_INVALID_ARG;
  if (vocab > CAMERA_MAX_VOCAB || n_rows > 0x3fffffff) return CAMERA_ERR_UNSUPPORTED_SHAPE;
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
  a.logits = d->logits; a.ld = d->ld; a.rows = (int)d->n_rows; a.lg = 0; a.in_place = 0; a.mark_words = 0; a.vocab = d->vocab; a.k = d->k;
  a.c = 1.44269504088896341f / d->temperature; a.inv_tau = 1.f / d->temperature;
  a.wait_limit_ns = current_wait_limit_ns();
  a.idx = d->teacher_idx; a.logprob = d->teacher_logprob;
  a.d_loss = nullptr; a.loss = a.lse = a.log_tail = nullptr; a.grad = nullptr; a.ld_grad = 0;
  return a;
}

// The status of a call from its launch's; an error is the call's, and not left for the caller's next check to find.
int launch_status(cudaError_t e) {
  if (e == cudaSuccess) return CAMERA_OK;
  cudaGetLastError();
  return CAMERA_ERR_CUDA;
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
  LogprobArgs a{logits, ld, (int)n_rows, vocab, top_n, 0, 1.44269504088896341f / temperature, 1.f / temperature,
                current_wait_limit_ns(), reinterpret_cast<const long long*>(targets),
                logprob, entropy, top_logprob, top_idx};
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  return launch_status(dtype == CAMERA_BF16 ? launch_logprobs<__nv_bfloat16>(a, st) : launch_logprobs<float>(a, st));
}

extern "C" int camera_distill_forward(const camera_distill_t* d, float* loss, float* lse, float* log_tail, void* cuda_stream) {
  using namespace camera;
  const int rc = check_distill(d);
  if (rc != CAMERA_OK) return rc;
  if (d->n_rows == 0) return CAMERA_OK;
  if (loss == nullptr) return CAMERA_ERR_INVALID_ARG;
  DistillArgs a = distill_args(d);
  a.loss = loss; a.lse = lse; a.log_tail = log_tail;
  return launch_status(launch_distill<DISTILL_FORWARD>(a, d->dtype, d->flags & CAMERA_DISTILL_TAIL, static_cast<cudaStream_t>(cuda_stream)));
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
  a.grad = d_logits; a.ld_grad = d_ld; a.in_place = d_logits == d->logits;
  return launch_status(launch_distill<DISTILL_BACKWARD>(a, d->dtype, d->flags & CAMERA_DISTILL_TAIL, static_cast<cudaStream_t>(cuda_stream)));
}

extern "C" int camera_distill_step(const camera_distill_t* d, const float* d_loss, float* loss, void* d_logits, int64_t d_ld,
                                   void* cuda_stream) {
  using namespace camera;
  const int rc = check_distill(d);
  if (rc != CAMERA_OK) return rc;
  if (d->n_rows == 0) return CAMERA_OK;
  if (d_loss == nullptr || loss == nullptr || !grad_ok(d, d_logits, d_ld)) return CAMERA_ERR_INVALID_ARG;
  DistillArgs a = distill_args(d);
  a.d_loss = d_loss; a.loss = loss; a.grad = d_logits; a.ld_grad = d_ld; a.in_place = d_logits == d->logits;
  return launch_status(launch_distill<DISTILL_STEP>(a, d->dtype, d->flags & CAMERA_DISTILL_TAIL, static_cast<cudaStream_t>(cuda_stream)));
}
