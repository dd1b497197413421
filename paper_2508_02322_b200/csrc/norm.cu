// Layer norm and root-mean-square norm of rows, with the residual sum, and their backward pass.
//   z = x + r, rounded to the dtype of x;  mu = mean z (0 for RMS);  s = (mean (z - mu)^2 + eps)^-1/2
//   y = (z - mu) s w + b
//   h = (z - mu) s, g = dy w:  dx = s (g - mean g - h mean(g h)) + d_sum (no mean g for RMS),  dw = sum_rows dy h,
//   db = sum_rows dy
// A row is held in the registers of a group of warps: it is read once, the sums are taken in two passes over registers
// (the second around the mean, so that a large mean costs no digits), and the next row of the group is on its way
// meanwhile.  All sums are fp32.
#include "common.cuh"
#include "launch.cuh"
#include "rowgroup.cuh"

namespace camera {

namespace {

constexpr int NORM_MAX_D = 32768;          // 32 warps x 32 elements a thread
constexpr int BACKWARD_ROWS = 2;            // a group's rows, at least
constexpr int FORWARD_THREADS = 1024;      // threads an SM may hold of the forward kernel
constexpr int BACKWARD_THREADS = 512;       // threads an SM holds of the backward kernel (128 registers each)
// Rows of a group in flight, of N 16-byte loads a thread and matrix: what 196 KB hold of the backward pass's three matrices for 512
// threads (16384 x 3584 bf16: 2 stages 96 us, 3 stages 94, 4 stages 95).
template <int N> constexpr int NORM_STAGES = N <= 2 ? 3 : N <= 8 ? 8 / N : 1;
// The same of the forward pass's two.
template <int N, int THREADS> constexpr int FORWARD_STAGES = THREADS <= 512 ? NORM_STAGES<N> : N <= 2 ? 3 : 1;
constexpr int NORM_GROUP_THREADS = 256;    // groups of fewer threads share a CTA up to this

struct NormArgs {
  const void *x, *r;                       // forward: x and the residual; backward: z and d_sum
  const void* dy;
  void *sum, *y;                           // backward: y is dx
  long long x_ld, r_ld, dy_ld, sum_ld, y_ld;
  long long rows;
  int d, warps;                            // warps that share a row
  const void *w, *b;
  bool w_f32, rms;
  float eps;
  float *mean, *rstd;                      // backward: inputs
  float* part;                             // backward: [groups][1 or 2][d] shares of dw and db
  bool want_w, want_b;
};

template <int W>
__device__ __forceinline__ void load_weight(const void* p, bool f32, int c, float absent, float (&out)[W]) {
  if (p == nullptr) {
#pragma unroll
    for (int i = 0; i < W; ++i) out[i] = absent;
  } else if (f32) {
    constexpr int V = W >= 4 ? 4 : 1;
#pragma unroll
    for (int k = 0; k < W; k += V) {
      const Pack<float, V> t = *reinterpret_cast<const Pack<float, V>*>(static_cast<const float*>(p) + c + k);
#pragma unroll
      for (int i = 0; i < V; ++i) out[k + i] = t.v[i];
    }
  } else {
    reinterpret_cast<const Pack<__nv_bfloat16, W>*>(static_cast<const __nv_bfloat16*>(p) + c)->get(out);
  }
}

// The weights of the columns a thread owns, as pairs; columns past the end have weight 0.
template <int W, int N>
__device__ __forceinline__ void own_weights(const void* p, bool f32, int d, int threads, int t, float absent, F2 (&out)[N * W / 2]) {
  float f[N * W];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int c = (j * threads + t) * W;
    float w[W];
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0.f;
    if (c < d) load_weight<W>(p, f32, c, absent, w);
#pragma unroll
    for (int i = 0; i < W; ++i) f[j * W + i] = w[i];
  }
#pragma unroll
  for (int i = 0; i < N * W / 2; ++i) out[i] = f2(f[2 * i], f[2 * i + 1]);
}

// W elements a load (16 bytes, or 1 element where rows or the width are not aligned for that), N loads a thread and matrix.
// Columns past the end read as zeros.  RING: the next rows travel through shared memory, each thread copying (cp.async) what it
// will read itself, so that a wait is the thread's own and the rows in flight cost no registers.
template <typename T, int W, int N, bool BIAS, bool RING, int THREADS>
__global__ void __launch_bounds__(THREADS, 1) k_norm_forward(const NormArgs q) {
  using P = Pack<T, W>;
  constexpr int E2 = N * W / 2, STAGES = FORWARD_STAGES<N, THREADS>;
  constexpr bool OWN_W = THREADS <= 512 && N * W <= 16;                  // weights in registers, or loaded again for each use
  extern __shared__ __align__(16) uint8_t ring[];
  const int threads = 32 * q.warps, group = threadIdx.x / threads, t = threadIdx.x - group * threads;
  const int groups = blockDim.x / threads;
  const long long step = (long long)gridDim.x * groups;
  const T* const x = static_cast<const T*>(q.x);
  const T* const r = static_cast<const T*>(q.r);
  int buf = 0, stage = 0;
  F2 w[E2], b[BIAS ? E2 : 1];
  if (OWN_W) {
    own_weights<W, N>(q.w, q.w_f32, q.d, threads, t, 1.f, w);
    if constexpr (BIAS) own_weights<W, N>(q.b, q.w_f32, q.d, threads, t, 0.f, b);
  }
  const int parts = r != nullptr ? 2 : 1, line = N * 16 * (int)blockDim.x;
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + 16 * threadIdx.x;
  auto issue = [&](int stage, long long row) {
    if (row < q.rows) {
      const T* const src[2] = {x + row * q.x_ld, r + row * q.r_ld};
#pragma unroll
      for (int p = 0; p < 2; ++p)
        if (p < parts) {
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const int c = (j * threads + t) * W, at = c < q.d ? c : 0;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(mine + (stage * parts + p) * line + j * 16 * blockDim.x),
                         "l"(src[p] + at), "r"(c < q.d ? 16 : 0)
                         : "memory");
          }
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  const long long first = (long long)blockIdx.x * groups + group;
  if constexpr (RING)
    for (int s = 0; s < STAGES; ++s) issue(s, first + s * step);
  for (long long row = first; row < q.rows; row += step) {
    P px[N], pr[N];
    if constexpr (RING) {
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
      const uint8_t* const at = ring + 16 * threadIdx.x + stage * parts * line;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        px[j] = *reinterpret_cast<const P*>(at + j * 16 * blockDim.x);
        if (r != nullptr) pr[j] = *reinterpret_cast<const P*>(at + line + j * 16 * blockDim.x);
      }
      issue(stage, row + STAGES * step);
      if (++stage == STAGES) stage = 0;
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int c = (j * threads + t) * W;
        px[j] = pr[j] = P();
        if (c < q.d) {
          px[j] = *reinterpret_cast<const P*>(x + row * q.x_ld + c);
          if (r != nullptr) pr[j] = *reinterpret_cast<const P*>(r + row * q.r_ld + c);
        }
      }
    }
    F2 z[E2];
    to_pairs<P, W, N>(px, z);
    if (r != nullptr) {
      F2 v[E2];
      to_pairs<P, W, N>(pr, v);
#pragma unroll
      for (int i = 0; i < E2; ++i) z[i] = add2(z[i], v[i]);
      from_pairs<P, W, N>(z, px);
      to_pairs<P, W, N>(px, z);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int c = (j * threads + t) * W;
        if (c < q.d) *reinterpret_cast<P*>(static_cast<T*>(q.sum) + row * q.sum_ld + c) = px[j];
      }
    }
    float s[1], lo, hi, mu = 0.f;
    F2 acc = f2(0.f, 0.f);
    if (!q.rms) {
#pragma unroll
      for (int i = 0; i < E2; ++i) acc = add2(acc, z[i]);
      split(acc, lo, hi);
      s[0] = lo + hi;
      group_sum(s, q.warps, group, buf);
      mu = s[0] / (float)q.d;
      // around the mean; columns past the end stay zero
      float f[N * W];
#pragma unroll
      for (int i = 0; i < E2; ++i) split(add2(z[i], f2(-mu, -mu)), f[2 * i], f[2 * i + 1]);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if ((j * threads + t) * W >= q.d) {
#pragma unroll
          for (int i = 0; i < W; ++i) f[j * W + i] = 0.f;
        }
#pragma unroll
      for (int i = 0; i < E2; ++i) z[i] = f2(f[2 * i], f[2 * i + 1]);
    }
    acc = f2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < E2; ++i) acc = fma2(z[i], z[i], acc);
    split(acc, lo, hi);
    s[0] = lo + hi;
    group_sum(s, q.warps, group, buf);
    const float rstd = 1.f / sqrtf(s[0] / (float)q.d + q.eps);
    if (t == 0) {
      if (q.mean != nullptr) q.mean[row] = mu;
      if (q.rstd != nullptr) q.rstd[row] = rstd;
    }
    if (!OWN_W) {
      own_weights<W, N>(q.w, q.w_f32, q.d, threads, t, 1.f, w);
      if constexpr (BIAS) own_weights<W, N>(q.b, q.w_f32, q.d, threads, t, 0.f, b);
    }
    const F2 rs = f2(rstd, rstd);
#pragma unroll
    for (int i = 0; i < E2; ++i) z[i] = BIAS ? fma2(mul2(z[i], rs), w[i], b[BIAS ? i : 0]) : mul2(mul2(z[i], rs), w[i]);
    from_pairs<P, W, N>(z, px);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = (j * threads + t) * W;
      if (c < q.d) *reinterpret_cast<P*>(static_cast<T*>(q.y) + row * q.y_ld + c) = px[j];
    }
  }
}

// A thread keeps the columns it owns for all rows of its group, so their weights and their shares of dw and db stay in its
// registers; the groups' shares are added up by k_norm_reduce in a fixed order.  Columns past the end read as zeros, which add
// nothing.  RING: the next rows travel through shared memory, each thread copying (cp.async) what it will read itself, so that
// a wait is the thread's own and the rows in flight cost no registers; without it (elements, which cp.async cannot copy one at
// a time) the next row waits in registers.
template <typename T, int W, int N, bool BIAS, bool RING, int THREADS>
__global__ void __launch_bounds__(THREADS, 1) k_norm_backward(const NormArgs q) {
  using P = Pack<T, W>;
  constexpr int E2 = N * W / 2;
  constexpr bool AHEAD = !RING && N * W <= 16;
  constexpr int STAGES = NORM_STAGES<N>;
  extern __shared__ __align__(16) uint8_t ring[];
  const int threads = 32 * q.warps, group = threadIdx.x / threads, t = threadIdx.x - group * threads;
  const int groups = blockDim.x / threads;
  const long long step = (long long)gridDim.x * groups;
  const T* const x = static_cast<const T*>(q.x);
  const T* const r = static_cast<const T*>(q.r);
  const T* const dy = static_cast<const T*>(q.dy);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int buf = 0;
  P now[3][RING ? 1 : N], next[3][AHEAD ? N : 1];
  constexpr bool OWN_W = N * W <= 16;                  // weights in registers, or loaded again for each use
  F2 dw[E2], db[BIAS ? E2 : 1], w[E2];
#pragma unroll
  for (int i = 0; i < E2; ++i) dw[i] = db[BIAS ? i : 0] = f2(0.f, 0.f);
  if (OWN_W) own_weights<W, N>(q.w, q.w_f32, q.d, threads, t, 1.f, w);
  const long long first = (long long)blockIdx.x * groups + group;
  auto load = [&](P (*to)[RING ? 1 : N], long long row) {
#pragma unroll
    for (int j = 0; j < (RING ? 0 : N); ++j) {
      const int c = (j * threads + t) * W;
      to[0][j] = to[1][j] = to[2][j] = P();
      if (c < q.d) {
        to[0][j] = *reinterpret_cast<const P*>(x + row * q.x_ld + c);
        to[1][j] = *reinterpret_cast<const P*>(dy + row * q.dy_ld + c);
        if (r != nullptr) to[2][j] = *reinterpret_cast<const P*>(r + row * q.r_ld + c);
      }
    }
  };
  const int parts = r != nullptr ? 3 : 2, line = N * 16 * (int)blockDim.x;
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + 16 * threadIdx.x;
  auto issue = [&](int stage, long long row) {
    if (row < q.rows) {
      const T* const src[3] = {x + row * q.x_ld, dy + row * q.dy_ld, r + row * q.r_ld};
#pragma unroll
      for (int p = 0; p < 3; ++p)
        if (p < parts) {
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const int c = (j * threads + t) * W, at = c < q.d ? c : 0;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(mine + (stage * parts + p) * line + j * 16 * blockDim.x),
                         "l"(src[p] + at), "r"(c < q.d ? 16 : 0)
                         : "memory");
          }
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  int stage = 0;
  // the thread's elements of matrix p (x, dy, d_sum) of this row, from where they wait
  auto get = [&](int p, F2 (&out)[E2]) {
    P v[N];
    const uint8_t* const at = ring + 16 * threadIdx.x + (stage * parts + p) * line;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if constexpr (RING) v[j] = *reinterpret_cast<const P*>(at + j * 16 * blockDim.x);
      else v[j] = now[p][j];
    }
    to_pairs<P, W, N>(v, out);
  };
  float rstd_next = 0.f, mu_next = 0.f;
  auto stats = [&](long long row) {
    if (row < q.rows) {
      rstd_next = q.rstd[row];
      mu_next = q.rms ? 0.f : q.mean[row];
    }
  };
  stats(first);
  if constexpr (RING) {
    for (int s = 0; s < STAGES; ++s) issue(s, first + s * step);
  } else if constexpr (AHEAD) {
    if (first < q.rows) load(next, first);
  }
  for (long long row = first; row < q.rows; row += step) {
    const float rstd = rstd_next, mu = mu_next;
    stats(row + step);
    if constexpr (RING) {
      asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
    } else if constexpr (AHEAD) {
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int j = 0; j < N; ++j) now[p][j] = next[p][j];
      if (row + step < q.rows) load(next, row + step);
    } else {
      load(now, row);
    }
    const F2 minus_mu = f2(-mu, -mu), rs = f2(rstd, rstd);
    F2 s0 = f2(0.f, 0.f), s1 = f2(0.f, 0.f);
    {
      F2 c[E2], d[E2];
      get(0, c);
      get(1, d);
      if (!OWN_W) own_weights<W, N>(q.w, q.w_f32, q.d, threads, t, 1.f, w);
#pragma unroll
      for (int i = 0; i < E2; ++i) {
        c[i] = add2(c[i], minus_mu);
        dw[i] = fma2(mul2(d[i], rs), c[i], dw[i]);
        if (BIAS) db[i] = add2(db[i], d[i]);
        const F2 g = mul2(d[i], w[i]);
        s0 = add2(s0, g);
        s1 = fma2(g, c[i], s1);
      }
    }
    if (q.y != nullptr) {
      float s[2], lo, hi;
      split(s0, lo, hi);
      s[0] = lo + hi;
      split(s1, lo, hi);
      s[1] = lo + hi;
      group_sum(s, q.warps, group, buf);
      // dx = s g - s mean g - c s^2 mean(g h),  mean(g h) = s mean(g c)
      const float k1 = q.rms ? 0.f : -rstd * (s[0] / (float)q.d), k2 = -rstd * rstd * (rstd * (s[1] / (float)q.d));
      const F2 k1s = f2(k1, k1), k2s = f2(k2, k2);
      F2 c[E2], d[E2];
      get(0, c);
      get(1, d);
      if (!OWN_W) own_weights<W, N>(q.w, q.w_f32, q.d, threads, t, 1.f, w);
#pragma unroll
      for (int i = 0; i < E2; ++i) c[i] = fma2(mul2(d[i], w[i]), rs, fma2(add2(c[i], minus_mu), k2s, k1s));
      if (r != nullptr) {
        get(2, d);
#pragma unroll
        for (int i = 0; i < E2; ++i) c[i] = add2(c[i], d[i]);
      }
      P out[N];
      from_pairs<P, W, N>(c, out);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int at = (j * threads + t) * W;
        if (at < q.d) *reinterpret_cast<P*>(static_cast<T*>(q.y) + row * q.y_ld + at) = out[j];
      }
    }
    if constexpr (RING) {
      issue(stage, row + STAGES * step);
      if (++stage == STAGES) stage = 0;
    }
  }
  // [groups][wanted][d]
  const int wanted = q.want_w + q.want_b;
  float* const part = q.part + first * wanted * q.d;
#pragma unroll
  for (int which = 0; which < (BIAS ? 2 : 1); ++which) {
    if (!(which ? q.want_b : q.want_w)) continue;
    float f[N * W];
#pragma unroll
    for (int i = 0; i < E2; ++i) split(which ? db[i] : dw[i], f[2 * i], f[2 * i + 1]);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = (j * threads + t) * W;
      if (c < q.d) {
        constexpr int V = W >= 4 ? 4 : 1;
#pragma unroll
        for (int k = 0; k < W; k += V) {
          Pack<float, V> a;
#pragma unroll
          for (int i = 0; i < V; ++i) a.v[i] = f[j * W + k + i];
          *reinterpret_cast<Pack<float, V>*>(part + (which ? (wanted - 1) * q.d : 0) + c + k) = a;
        }
      }
    }
  }
}

constexpr int REDUCE_WARPS = 32;
struct NormReduce { const float* part; int groups, d, wanted; float *dw, *db; };
// Columns of the groups' shares added up: a lane takes a column, the warps take every 32nd group.
__global__ void __launch_bounds__(32 * REDUCE_WARPS) k_norm_reduce(const NormReduce q) {
  __shared__ float sums[REDUCE_WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, which = blockIdx.y;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float* const out = which || q.dw == nullptr ? q.db : q.dw;
  float s = 0.f;
  if (c < q.d) {
    const float* p = q.part + (long long)which * q.d + c;
#pragma unroll 8
    for (int g = warp; g < q.groups; g += REDUCE_WARPS) s += p[(long long)g * q.wanted * q.d];
  }
  sums[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < q.d) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < REDUCE_WARPS; ++i) s += sums[i][lane];
    out[c] = s;
  }
}

// ------------------------------------------------------------------------------------------------ host side
struct NormShape { int warps, groups_per_cta, ctas; };

// Warps a row and groups a CTA for `per` elements a thread; threads_sm: threads an SM holds of the kernel.
NormShape norm_shape(long long rows, int d, int per, int threads_sm, long long rows_per_group) {
  NormShape s;
  s.warps = (d + 32 * per - 1) / (32 * per);
  s.groups_per_cta = NORM_GROUP_THREADS / (32 * s.warps);
  if (s.groups_per_cta < 1) s.groups_per_cta = 1;
  const int sms = sm_count();
  const long long want = (rows + rows_per_group - 1) / rows_per_group;       // groups
  while (s.groups_per_cta > 1 && (want + s.groups_per_cta - 1) / s.groups_per_cta < sms) --s.groups_per_cta;
  const int per_sm = threads_sm / (32 * s.warps * s.groups_per_cta);
  const long long most = (long long)sms * (per_sm > 1 ? per_sm : 1), need = (want + s.groups_per_cta - 1) / s.groups_per_cta;
  s.ctas = (int)(need < most ? need : most);
  return s;
}

// Elements a thread holds in the backward pass, and the groups that leave shares of dw and db.
int backward_per(int d) { return d <= 16 * 512 ? 16 : 32; }
// Rows a group takes at least: a group's shares cost the second kernel as much as a few of its rows do here, more where rows are
// read by elements.
NormShape backward_shape(long long rows, int d, bool vec) {
  return norm_shape(rows, d, backward_per(d), BACKWARD_THREADS, vec ? 2 * BACKWARD_ROWS : BACKWARD_ROWS);
}

template <typename T, int W, int N, bool BIAS, bool RING, int THREADS>
cudaError_t forward_as(const NormArgs& a, cudaStream_t st) {
  NormArgs q = a;
  const NormShape s = norm_shape(q.rows, q.d, N * W, RING ? FORWARD_THREADS : 1024, 1);
  q.warps = s.warps;
  const int threads = 32 * s.warps * s.groups_per_cta;
  int smem = 0;
  if constexpr (RING) {
    constexpr int MOST = FORWARD_STAGES<N, THREADS> * 2 * N * 16 * THREADS;
    static_assert(MOST <= 226 * 1024, "shared memory of an SM");
    const cudaError_t e = allow_smem<k_norm_forward<T, W, N, BIAS, RING, THREADS>, MOST>();
    if (e != cudaSuccess) return e;
    smem = FORWARD_STAGES<N, THREADS> * (q.r != nullptr ? 2 : 1) * N * threads * 16;
  }
  k_norm_forward<T, W, N, BIAS, RING, THREADS><<<s.ctas, threads, smem, st>>>(q);
  return cudaGetLastError();
}
template <typename T, bool BIAS>
cudaError_t forward_typed(const NormArgs& q, bool vec, cudaStream_t st) {
  constexpr int W = 16 / (int)sizeof(T);
  // Few rows: 8 elements a thread, so that a row's loads and sums are spread over most threads.
  if (q.rows <= 2 * sm_count() && q.d <= 8 * 1024)
    return vec ? forward_as<T, W, 8 / W, BIAS, false, 1024>(q, st) : forward_as<T, 1, 8, BIAS, false, 1024>(q, st);
  if (q.d <= 16 * 512) return vec ? forward_as<T, W, 16 / W, BIAS, true, 512>(q, st) : forward_as<T, 1, 16, BIAS, false, 512>(q, st);
  if (q.d <= 16 * 1024 && vec) return forward_as<T, W, 16 / W, BIAS, true, 1024>(q, st);
  if (q.d <= 32 * 512) return forward_as<T, 1, 32, BIAS, false, 512>(q, st);
  return vec ? forward_as<T, W, 32 / W, BIAS, false, 1024>(q, st) : forward_as<T, 1, 32, BIAS, false, 1024>(q, st);
}

template <typename T, int W, int N, bool BIAS, int THREADS>
cudaError_t backward_as(const NormArgs& a, const NormShape& s, cudaStream_t st) {
  constexpr bool RING = W * sizeof(T) == 16 && THREADS <= 512;
  NormArgs q = a;
  q.warps = s.warps;
  const int threads = 32 * s.warps * s.groups_per_cta;
  int smem = 0;
  if constexpr (RING) {
    constexpr int MOST = NORM_STAGES<N> * 3 * N * 16 * THREADS;
    static_assert(MOST <= 226 * 1024, "shared memory of an SM");
    const cudaError_t e = allow_smem<k_norm_backward<T, W, N, BIAS, RING, THREADS>, MOST>();
    if (e != cudaSuccess) return e;
    smem = NORM_STAGES<N> * (q.r != nullptr ? 3 : 2) * N * threads * 16;
  }
  return launch_chained(k_norm_backward<T, W, N, BIAS, RING, THREADS>, q, s.ctas, 1, 1, threads, smem, false, st);
}
template <typename T, bool BIAS>
cudaError_t backward_typed(const NormArgs& q, const NormShape& s, bool vec, cudaStream_t st) {
  constexpr int W = 16 / (int)sizeof(T);
  if (backward_per(q.d) == 16) return vec ? backward_as<T, W, 16 / W, BIAS, 512>(q, s, st) : backward_as<T, 1, 16, BIAS, 512>(q, s, st);
  if (s.warps <= 16) return vec ? backward_as<T, W, 32 / W, BIAS, 512>(q, s, st) : backward_as<T, 1, 32, BIAS, 512>(q, s, st);
  return vec ? backward_as<T, W, 32 / W, BIAS, 1024>(q, s, st) : backward_as<T, 1, 32, BIAS, 1024>(q, s, st);
}

int check_norm(const camera_norm_t* n) {
  if (n == nullptr || n->n_rows < 0 || n->d < 1 || (n->dtype != CAMERA_BF16 && n->dtype != CAMERA_F32) ||
      (n->weight_dtype != CAMERA_BF16 && n->weight_dtype != CAMERA_F32) || (n->flags & ~(uint32_t)CAMERA_NORM_RMS) || !(n->eps >= 0.f) ||
      !(n->eps < 3.0e38f) || n->ld < n->d)
    return CAMERA_ERR_INVALID_ARG;
  if (n->d > NORM_MAX_D) return CAMERA_ERR_UNSUPPORTED_SHAPE;
  const uintptr_t wm = n->weight_dtype == CAMERA_BF16 ? 1 : 3;
  if ((reinterpret_cast<uintptr_t>(n->weight) | reinterpret_cast<uintptr_t>(n->bias)) & wm) return CAMERA_ERR_INVALID_ARG;
  return CAMERA_OK;
}
bool rows_ok(const void* p, long long ld, const camera_norm_t* n) {
  return p != nullptr && ld >= n->d && (reinterpret_cast<uintptr_t>(p) & (n->dtype == CAMERA_BF16 ? 1 : 3)) == 0;
}

#define NORM_CK(...)            \
  do {                          \
    if ((__VA_ARGS__) != cudaSuccess) { \
      cudaGetLastError();       \
      return CAMERA_ERR_CUDA;   \
    }                           \
  } while (0)

size_t norm_part_bytes(const NormShape& s, int d) { return (size_t)s.ctas * s.groups_per_cta * 2 * d * 4; }
// At least that for any alignment, and no less for more rows, so that a workspace serves every smaller call: groups are what the rows
// ask for, rounded up to whole CTAs, or as many as the GPU holds at one time.
size_t norm_part_bound(int64_t rows, int d) {
  const int warps = (d + 32 * backward_per(d) - 1) / (32 * backward_per(d));
  const int64_t want = (rows + BACKWARD_ROWS - 1) / BACKWARD_ROWS + NORM_GROUP_THREADS / 32, most = (int64_t)sm_count() * (BACKWARD_THREADS / 32 / warps > 1 ? BACKWARD_THREADS / 32 / warps : 1);
  return (size_t)(want < most ? want : most) * 2 * d * 4;
}

}  // namespace
}  // namespace camera

extern "C" int camera_norm_forward(const camera_norm_t* n, const void* residual, int64_t residual_ld, void* sum, int64_t sum_ld,
                                   void* y, int64_t y_ld, float* mean, float* rstd, void* cuda_stream) {
  using namespace camera;
  const int rc = check_norm(n);
  if (rc != CAMERA_OK) return rc;
  if ((residual == nullptr) != (sum == nullptr)) return CAMERA_ERR_INVALID_ARG;
  if (n->n_rows == 0) return CAMERA_OK;
  if (!rows_ok(n->x, n->ld, n) || !rows_ok(y, y_ld, n) ||
      (residual != nullptr && (!rows_ok(residual, residual_ld, n) || !rows_ok(sum, sum_ld, n))))
    return CAMERA_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(mean) | reinterpret_cast<uintptr_t>(rstd)) & 3) return CAMERA_ERR_INVALID_ARG;
  NormArgs q = {};
  q.x = n->x; q.r = residual; q.sum = sum; q.y = y;
  q.x_ld = n->ld; q.r_ld = residual_ld; q.sum_ld = sum_ld; q.y_ld = y_ld;
  q.rows = n->n_rows; q.d = n->d;
  q.w = n->weight; q.b = n->bias; q.w_f32 = n->weight_dtype == CAMERA_F32;
  q.rms = n->flags & CAMERA_NORM_RMS; q.eps = n->eps; q.mean = mean; q.rstd = rstd;
  const int size = n->dtype == CAMERA_BF16 ? 2 : 4;
  const bool vec = (n->d * size) % 16 == 0 && vec_ok(q.x, q.x_ld, size) && vec_ok(q.r, q.r_ld, size) && vec_ok(q.sum, q.sum_ld, size) &&
                   vec_ok(q.y, q.y_ld, size) && vec_ok(q.w, 0, 1) && vec_ok(q.b, 0, 1);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (size == 2) NORM_CK(q.b != nullptr ? forward_typed<__nv_bfloat16, true>(q, vec, st) : forward_typed<__nv_bfloat16, false>(q, vec, st));
  else NORM_CK(q.b != nullptr ? forward_typed<float, true>(q, vec, st) : forward_typed<float, false>(q, vec, st));
  return CAMERA_OK;
}

extern "C" size_t camera_norm_backward_workspace_bytes(int64_t n_rows, int32_t d) {
  if (n_rows < 0 || d < 1 || d > camera::NORM_MAX_D) return 0;
  return 256 + camera::norm_part_bound(n_rows, d);
}

extern "C" int camera_norm_backward(const camera_norm_t* n, const void* dy, int64_t dy_ld, const float* mean, const float* rstd,
                                    const void* d_sum, int64_t d_sum_ld, void* dx, int64_t dx_ld, float* d_weight, float* d_bias,
                                    void* workspace, size_t workspace_bytes, void* cuda_stream) {
  using namespace camera;
  const int rc = check_norm(n);
  if (rc != CAMERA_OK) return rc;
  const bool want_w = d_weight != nullptr || d_bias != nullptr;
  if (n->n_rows > 0 && dx == nullptr && (!want_w || d_sum != nullptr)) return CAMERA_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(mean) | reinterpret_cast<uintptr_t>(rstd) | reinterpret_cast<uintptr_t>(d_weight) |
       reinterpret_cast<uintptr_t>(d_bias)) & 3)
    return CAMERA_ERR_INVALID_ARG;
  const bool rms = n->flags & CAMERA_NORM_RMS;
  if (n->n_rows > 0 && (!rows_ok(n->x, n->ld, n) || !rows_ok(dy, dy_ld, n) || (dx != nullptr && !rows_ok(dx, dx_ld, n)) ||
                        (d_sum != nullptr && !rows_ok(d_sum, d_sum_ld, n)) || rstd == nullptr || (mean == nullptr && !rms)))
    return CAMERA_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (n->n_rows == 0) {                         // sums over no row
    if (d_weight != nullptr) NORM_CK(cudaMemsetAsync(d_weight, 0, (size_t)4 * n->d, st));
    if (d_bias != nullptr) NORM_CK(cudaMemsetAsync(d_bias, 0, (size_t)4 * n->d, st));
    return CAMERA_OK;
  }
  NormArgs q = {};
  q.x = n->x; q.r = d_sum; q.dy = dy; q.y = dx;
  q.x_ld = n->ld; q.r_ld = d_sum_ld; q.dy_ld = dy_ld; q.y_ld = dx_ld;
  q.rows = n->n_rows; q.d = n->d;
  q.w = n->weight; q.w_f32 = n->weight_dtype == CAMERA_F32;
  q.rms = rms; q.mean = const_cast<float*>(mean); q.rstd = const_cast<float*>(rstd);
  q.part = static_cast<float*>(workspace); q.want_w = d_weight != nullptr; q.want_b = d_bias != nullptr;
  const int size = n->dtype == CAMERA_BF16 ? 2 : 4;
  const bool vec = (n->d * size) % 16 == 0 && vec_ok(q.x, q.x_ld, size) && vec_ok(q.r, q.r_ld, size) && vec_ok(q.dy, q.dy_ld, size) &&
                   vec_ok(q.y, q.y_ld, size) && vec_ok(q.w, 0, 1);
  const NormShape s = backward_shape(q.rows, q.d, vec);
  if (want_w && (workspace == nullptr || workspace_bytes < norm_part_bytes(s, q.d) || (reinterpret_cast<uintptr_t>(workspace) & 255)))
    return CAMERA_ERR_WORKSPACE;
  if (size == 2) NORM_CK(q.want_b ? backward_typed<__nv_bfloat16, true>(q, s, vec, st) : backward_typed<__nv_bfloat16, false>(q, s, vec, st));
  else NORM_CK(q.want_b ? backward_typed<float, true>(q, s, vec, st) : backward_typed<float, false>(q, s, vec, st));
  if (want_w) {
    const NormReduce r = {q.part, s.ctas * s.groups_per_cta, q.d, q.want_w + q.want_b, d_weight, d_bias};
    NORM_CK(launch_chained(k_norm_reduce, r, (q.d + 31) / 32, r.wanted, 1, 32 * REDUCE_WARPS, 0, true, st));
  }
  return CAMERA_OK;
}
