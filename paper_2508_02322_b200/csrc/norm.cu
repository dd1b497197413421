// Layer norm and root-mean-square norm of rows, with the residual sum, and their backward pass.
//   z = x + r, rounded to the dtype of x;  mu = mean z (0 for RMS);  s = (mean (z - mu)^2 + eps)^-1/2
//   y = (z - mu) s w + b
//   h = (z - mu) s, g = dy w:  dx = s (g - mean g - h mean(g h)) + d_sum (no mean g for RMS),  dw = sum_rows dy h,
//   db = sum_rows dy
// A row is held by the threads of a group of warps: it is read once, the sums are taken in two passes over what they hold
// (the second around the mean, so that a large mean costs no digits), and up to 8192 columns the next rows of the group are on
// their way meanwhile.  All sums are fp32.
// Bound: HBM.  16384 x 3584 bf16, root mean square, with residual: forward 88 us, backward with d_sum and weight gradient 84 us by itself
// and 92 us among other calls, 470 MB each, 5.3 and 5.1 to 5.6 TB/s (copy 6.5).  One row: 2.5 us, which is a load, two barriers and a store.
// Longer rows: registers.  Of 8193 to 16384 columns one row is in flight (6000 rows of 12288 bf16: forward 0.55, backward 0.39 of the copy
// rate); beyond, 32 elements a thread beside their weights do not fit 64 registers: the forward kernels keep 270 to 2120 bytes a thread in
// local memory (20480 columns: 0.38, backward 0.37).
#include "common.cuh"
#include "launch.cuh"
#include "rowgroup.cuh"

namespace camera {

namespace {

constexpr int NORM_MAX_D = 32768;          // 32 warps x 32 elements a thread
constexpr int NORM_BOTH_D = 28672;         // up to here shared memory holds shares of dw and db
constexpr int BACKWARD_ROWS = 2;           // a group's rows in the backward pass, at least
// Rows of a group worked on together, so that their sums and barriers overlap: two in the backward pass (16384 x 3584 bf16: 90 us by
// one, 83 by two) and in the forward pass of layer norms with their two sums (12743 x 4608 bf16 with bias and residual: 125 and 105),
// one in that of root-mean-square norms (16384 x 3584: 86 and 89).
template <int THREADS> constexpr int BACKWARD_TOGETHER = THREADS > 512 ? 1 : 2;
// Rows of a group in flight, of N 16-byte loads a thread and matrix: what 196 KB hold of the backward pass's three matrices for 512
// threads; one where a CTA has up to 1024 for a long row.
template <int N, int THREADS, int E> constexpr int NORM_STAGES = THREADS > 512 && E > 8 ? 1 : N <= 2 ? 4 : 2;
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
  float* part;                             // backward: [CTAs][1 or 2][d] shares of dw and db
  bool want_w, want_b;
  float *dw, *db;                          // where one CTA writes them itself; or null
};

// W elements from p on: at once, or (LOOSE) one by one, from any address.
template <bool LOOSE, typename T, int W>
__device__ __forceinline__ Pack<T, W> load_pack(const T* p) {
  if constexpr (LOOSE && sizeof(T) == 2) {
    const uint16_t* const e = reinterpret_cast<const uint16_t*>(p);
    Pack<T, W> v;
#pragma unroll
    for (int i = 0; i < W / 2; ++i) v.v[i] = (uint32_t)e[2 * i] | (uint32_t)e[2 * i + 1] << 16;
    return v;
  } else if constexpr (LOOSE) {
    Pack<T, W> v;
#pragma unroll
    for (int i = 0; i < W; ++i) v.v[i] = p[i];
    return v;
  } else {
    return *reinterpret_cast<const Pack<T, W>*>(p);
  }
}

// 16 bytes on their way to shared memory (zeros where there are none), in words if LOOSE.
template <bool LOOSE>
__device__ __forceinline__ void copy_pack(uint32_t to, const void* from, bool there) {
  if constexpr (LOOSE) {
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + i), "l"(static_cast<const char*>(from) + i), "r"(there ? 4 : 0) : "memory");
  } else {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
  }
}

template <bool LOOSE, int W>
__device__ __forceinline__ void load_weight(const void* p, bool f32, int c, float absent, float (&out)[W]) {
  if (p == nullptr) {
#pragma unroll
    for (int i = 0; i < W; ++i) out[i] = absent;
  } else if (f32) {
    constexpr int V = W >= 4 ? 4 : W;
#pragma unroll
    for (int k = 0; k < W; k += V) {
      const Pack<float, V> t = load_pack<LOOSE, float, V>(static_cast<const float*>(p) + c + k);
#pragma unroll
      for (int i = 0; i < V; ++i) out[k + i] = t.v[i];
    }
  } else {
    load_pack<LOOSE, __nv_bfloat16, W>(static_cast<const __nv_bfloat16*>(p) + c).get(out);
  }
}

// The weights of the columns a thread owns, as pairs; columns past the end have weight 0.
template <bool LOOSE, int W, int N>
__device__ __forceinline__ void own_weights(const void* p, bool f32, int d, int threads, int t, float absent, F2 (&out)[N * W / 2]) {
  float f[N * W];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int c = (j * threads + t) * W;
    float w[W];
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0.f;
    if (c < d) load_weight<LOOSE, W>(p, f32, c, absent, w);
#pragma unroll
    for (int i = 0; i < W; ++i) f[j * W + i] = w[i];
  }
#pragma unroll
  for (int i = 0; i < N * W / 2; ++i) out[i] = f2(f[2 * i], f[2 * i + 1]);
}

// W elements a load (16 bytes, or 1 element where rows or the width are not aligned for that), N loads a thread and matrix.
// Columns past the end read as zeros.  RING: the next rows travel through shared memory, each thread copying (cp.async) what it
// will read itself, so that a wait is the thread's own and the rows in flight cost no registers.
template <typename T, int W, int N, bool BIAS, bool RING, bool LOOSE, int THREADS, int ROWS>
__global__ void __launch_bounds__(THREADS, 1) k_norm_forward(const NormArgs q) {
  using P = Pack<T, W>;
  constexpr int E2 = N * W / 2, STAGES = NORM_STAGES<N, THREADS, N * W>;
  constexpr bool OWN_W = N * W <= 8 || (THREADS <= 512 && N * W <= 16);   // weights in registers, or loaded again for each use
  constexpr bool AHEAD = !RING && (N * W <= 8 || THREADS <= 512);         // the next row waits in registers
  extern __shared__ __align__(16) uint8_t ring[];
  const int threads = 32 * q.warps, group = threadIdx.x / threads, t = threadIdx.x - group * threads;
  const int groups = blockDim.x / threads;
  const long long step = (long long)gridDim.x * groups;
  const T* const x = static_cast<const T*>(q.x);
  const T* const r = static_cast<const T*>(q.r);
  int buf = 0, stage = 0;
  F2 w[E2], b[BIAS ? E2 : 1];
  if (OWN_W) {
    own_weights<LOOSE, W, N>(q.w, q.w_f32, q.d, threads, t, 1.f, w);
    if constexpr (BIAS) own_weights<LOOSE, W, N>(q.b, q.w_f32, q.d, threads, t, 0.f, b);
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
            copy_pack<false>(mine + (stage * parts + p) * line + j * 16 * blockDim.x, src[p] + at, c < q.d);
          }
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  P nx[N], nr[N];
  auto load = [&](long long row) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = (j * threads + t) * W;
      nx[j] = nr[j] = P();
      if (c < q.d) {
        nx[j] = load_pack<LOOSE, T, W>(x + row * q.x_ld + c);
        if (r != nullptr) nr[j] = load_pack<LOOSE, T, W>(r + row * q.r_ld + c);
      }
    }
  };
  const long long first = (long long)blockIdx.x * groups + group;
  if constexpr (RING) {
    for (int s = 0; s < STAGES; ++s) issue(s, first + s * step);
  } else if constexpr (AHEAD) {
    if (first < q.rows) load(first);
  }
  for (long long row0 = first; row0 < q.rows; row0 += ROWS * step) {
    F2 z[ROWS][E2];
    float mu[ROWS], s[ROWS], lo, hi;
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const long long row = row0 + k * step;
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
        if (!AHEAD) load(row);
#pragma unroll
        for (int j = 0; j < N; ++j) { px[j] = nx[j]; pr[j] = nr[j]; }
        if (AHEAD && row + step < q.rows) load(row + step);
      }
      to_pairs<P, W, N>(px, z[k]);
      if (r != nullptr) {
        F2 v[E2];
        to_pairs<P, W, N>(pr, v);
#pragma unroll
        for (int i = 0; i < E2; ++i) z[k][i] = add2(z[k][i], v[i]);
        from_pairs<P, W, N>(z[k], px);
        to_pairs<P, W, N>(px, z[k]);
        if (row < q.rows) {
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const int c = (j * threads + t) * W;
            if (c < q.d) *reinterpret_cast<P*>(static_cast<T*>(q.sum) + row * q.sum_ld + c) = px[j];
          }
        }
      }
      mu[k] = 0.f;
      F2 acc = f2(0.f, 0.f);
#pragma unroll
      for (int i = 0; i < E2; ++i) acc = q.rms ? fma2(z[k][i], z[k][i], acc) : add2(acc, z[k][i]);
      split(acc, lo, hi);
      s[k] = lo + hi;
    }
    group_sum(s, q.warps, group, buf);
    if (!q.rms) {
#pragma unroll
      for (int k = 0; k < ROWS; ++k) {
        mu[k] = s[k] / (float)q.d;
        // around the mean; columns past the end stay zero
        float f[N * W];
#pragma unroll
        for (int i = 0; i < E2; ++i) split(add2(z[k][i], f2(-mu[k], -mu[k])), f[2 * i], f[2 * i + 1]);
#pragma unroll
        for (int j = 0; j < N; ++j)
          if ((j * threads + t) * W >= q.d) {
#pragma unroll
            for (int i = 0; i < W; ++i) f[j * W + i] = 0.f;
          }
        F2 acc = f2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < E2; ++i) {
          z[k][i] = f2(f[2 * i], f[2 * i + 1]);
          acc = fma2(z[k][i], z[k][i], acc);
        }
        split(acc, lo, hi);
        s[k] = lo + hi;
      }
      group_sum(s, q.warps, group, buf);
    }
    if (!OWN_W) {
      own_weights<LOOSE, W, N>(q.w, q.w_f32, q.d, threads, t, 1.f, w);
      if constexpr (BIAS) own_weights<LOOSE, W, N>(q.b, q.w_f32, q.d, threads, t, 0.f, b);
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const long long row = row0 + k * step;
      if (row >= q.rows) break;
      const float rstd = 1.f / sqrtf(s[k] / (float)q.d + q.eps);
      if (t == 0) {
        if (q.mean != nullptr) q.mean[row] = mu[k];
        if (q.rstd != nullptr) q.rstd[row] = rstd;
      }
      const F2 rs = f2(rstd, rstd);
      P out[N];
#pragma unroll
      for (int i = 0; i < E2; ++i) z[k][i] = BIAS ? fma2(mul2(z[k][i], rs), w[i], b[BIAS ? i : 0]) : mul2(mul2(z[k][i], rs), w[i]);
      from_pairs<P, W, N>(z[k], out);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int c = (j * threads + t) * W;
        if (c < q.d) *reinterpret_cast<P*>(static_cast<T*>(q.y) + row * q.y_ld + c) = out[j];
      }
    }
  }
}

// A thread keeps the columns it owns for all rows of its group, so their weights and their shares of dw and db stay in its
// registers (in its own places of shared memory where a row is long); the groups of a CTA add theirs up in shared memory, the CTAs'
// shares are added up by k_norm_reduce, all in a fixed order (a share per group: 39156 x 90 bf16 37 us, one per CTA 20).  Columns past the end read as zeros, which add nothing.  RING as above; without it both passes over a row load it.
template <typename T, int W, int N, bool BIAS, bool RING, bool LOOSE, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 256 ? 4 : 1) k_norm_backward(const NormArgs q) {
  using P = Pack<T, W>;
  constexpr bool LONG = THREADS > 512 && N * W >= 16;
  constexpr int E2 = N * W / 2, STAGES = NORM_STAGES<N, THREADS, N * W>;
  constexpr int G = W == 1 ? 2 : 1, PR = W == 1 ? 1 : W / 2;           // packs worked on at a time, and their pairs
  constexpr int ROWS = BACKWARD_TOGETHER<THREADS>;
  extern __shared__ __align__(16) uint8_t ring[];
  const int threads = 32 * q.warps, group = threadIdx.x / threads, t = threadIdx.x - group * threads;
  const int groups = blockDim.x / threads;
  const long long step = (long long)gridDim.x * groups;
  const T* const src[3] = {static_cast<const T*>(q.x), static_cast<const T*>(q.dy), static_cast<const T*>(q.r)};
  const long long ld[3] = {q.x_ld, q.dy_ld, q.r_ld};
  const bool has_r = q.r != nullptr;
  const int parts = has_r ? 3 : 2, line = N * 16 * (int)blockDim.x;
  const long long first = (long long)blockIdx.x * groups + group;
  const int wanted = q.want_w + q.want_b;
  float* const part = q.part + (long long)blockIdx.x * wanted * q.d;
  // LONG: pair i of the thread's share of dw at i * blockDim.x + threadIdx.x, db's behind it, or in memory where there is no room
  F2* const acc = reinterpret_cast<F2*>(ring + (RING ? STAGES * parts * line : 0)) + threadIdx.x;
  F2* const acc_b = acc + E2 * blockDim.x;
  const bool far = LONG && BIAS && q.d > NORM_BOTH_D;
  const bool direct = q.dw != nullptr || q.db != nullptr;
  float* const to_w = direct ? q.dw : part;
  float* const part_b = direct ? q.db : part + (wanted - 1) * q.d;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int buf = 0, stage = 0;
  F2 dw[LONG ? 1 : E2], db[BIAS && !LONG ? E2 : 1], w[LONG ? 1 : E2];
#pragma unroll
  for (int i = 0; i < (LONG ? 1 : E2); ++i) dw[i] = db[BIAS && !LONG ? i : 0] = f2(0.f, 0.f);
  if constexpr (LONG) {
    for (int i = 0; i < E2; ++i) {
      acc[i * blockDim.x] = f2(0.f, 0.f);
      if (BIAS && !far) acc_b[i * blockDim.x] = f2(0.f, 0.f);
    }
    if (far)
      for (int j = 0; j < N; ++j)
        for (int i = 0; i < W; ++i)
          if ((j * threads + t) * W + i < q.d) part_b[(j * threads + t) * W + i] = 0.f;
  } else {
    own_weights<LOOSE, W, N>(q.w, q.w_f32, q.d, threads, t, 1.f, w);
  }
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + 16 * threadIdx.x;
  auto issue = [&](int stage, long long row) {
    if (row < q.rows) {
#pragma unroll
      for (int p = 0; p < 3; ++p)
        if (p < parts) {
#pragma unroll
          for (int j = 0; j < N; ++j) {
            const int c = (j * threads + t) * W, at = c < q.d ? c : 0;
            copy_pack<LOOSE>(mine + (stage * parts + p) * line + j * 16 * blockDim.x, src[p] + row * ld[p] + at, c < q.d);
          }
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // pairs of packs j .. j + G - 1 of matrix p (x, dy, d_sum) of this row, from where they wait
  auto get = [&](int p, int j, int k_row, long long row, F2 (&out)[PR]) {
    P v[G];
#pragma unroll
    for (int k = 0; k < G; ++k) {
      if constexpr (RING) {
        v[k] = *reinterpret_cast<const P*>(ring + 16 * threadIdx.x + ((stage + k_row) % STAGES * parts + p) * line + (j + k) * 16 * blockDim.x);
      } else {
        const int c = ((j + k) * threads + t) * W;
        v[k] = P();
        if (c < q.d) v[k] = load_pack<LOOSE, T, W>(src[p] + row * ld[p] + c);
      }
    }
    to_pairs<P, W, G>(v, out);
  };
  auto weights = [&](int j, F2 (&out)[PR]) {
    if constexpr (LONG) {
      float f[G * W];
#pragma unroll
      for (int k = 0; k < G; ++k) {
        const int c = ((j + k) * threads + t) * W;
        float v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = 0.f;
        if (c < q.d) load_weight<LOOSE, W>(q.w, q.w_f32, c, 1.f, v);
#pragma unroll
        for (int i = 0; i < W; ++i) f[k * W + i] = v[i];
      }
#pragma unroll
      for (int i = 0; i < PR; ++i) out[i] = f2(f[2 * i], f[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < PR; ++i) out[i] = w[j / G * PR + i];
    }
  };
  float rstd_next[ROWS], mu_next[ROWS];
  auto stats = [&](long long row0) {
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const long long row = row0 + k * step;
      rstd_next[k] = row < q.rows ? q.rstd[row] : 0.f;
      mu_next[k] = row < q.rows && !q.rms ? q.mean[row] : 0.f;
    }
  };
  stats(first);
  if constexpr (RING)
    for (int s = 0; s < STAGES; ++s) issue(s, first + s * step);
  for (long long row0 = first; row0 < q.rows; row0 += ROWS * step) {
    float rstd[ROWS], s[2 * ROWS];
    F2 minus_mu[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      rstd[k] = rstd_next[k];
      minus_mu[k] = f2(-mu_next[k], -mu_next[k]);
    }
    stats(row0 + ROWS * step);
    if constexpr (RING) asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - ROWS) : "memory");
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const long long row = row0 + k * step;
      F2 s0 = f2(0.f, 0.f), s1 = f2(0.f, 0.f);
      if (row < q.rows) {
        const F2 rs = f2(rstd[k], rstd[k]);
#pragma unroll
        for (int j = 0; j < N; j += G) {
          F2 c[PR], d[PR], wj[PR];
          get(0, j, k, row, c);
          get(1, j, k, row, d);
          weights(j, wj);
#pragma unroll
          for (int i = 0; i < PR; ++i) {
            const int at = j / G * PR + i;
            c[i] = add2(c[i], minus_mu[k]);
            const F2 g = mul2(d[i], wj[i]), dr = mul2(d[i], rs);
            s0 = add2(s0, g);
            s1 = fma2(g, c[i], s1);
            if constexpr (LONG) {
              acc[at * blockDim.x] = fma2(dr, c[i], acc[at * blockDim.x]);
              if (BIAS && !far) acc_b[at * blockDim.x] = add2(acc_b[at * blockDim.x], d[i]);
              if (far) {
                float lo, hi;
                split(d[i], lo, hi);
                const int c0 = (j * threads + t) * W + 2 * i, c1 = W == 1 ? c0 + threads : c0 + 1;
                if (c0 < q.d) part_b[c0] += lo;
                if (c1 < q.d) part_b[c1] += hi;
              }
            } else {
              dw[at] = fma2(dr, c[i], dw[at]);
              if (BIAS) db[at] = add2(db[at], d[i]);
            }
          }
        }
      }
      float lo, hi;
      split(s0, lo, hi);
      s[2 * k] = lo + hi;
      split(s1, lo, hi);
      s[2 * k + 1] = lo + hi;
    }
    if (q.y != nullptr) {
      group_sum(s, q.warps, group, buf);
#pragma unroll
      for (int k = 0; k < ROWS; ++k) {
        const long long row = row0 + k * step;
        if (row >= q.rows) break;
        // dx = s g - s mean g - c s^2 mean(g h),  mean(g h) = s mean(g c)
        const float k1 = q.rms ? 0.f : -rstd[k] * (s[2 * k] / (float)q.d), k2 = -rstd[k] * rstd[k] * (rstd[k] * (s[2 * k + 1] / (float)q.d));
        const F2 k1s = f2(k1, k1), k2s = f2(k2, k2), rs = f2(rstd[k], rstd[k]);
#pragma unroll
        for (int j = 0; j < N; j += G) {
          F2 c[PR], d[PR], wj[PR];
          get(0, j, k, row, c);
          get(1, j, k, row, d);
          weights(j, wj);
#pragma unroll
          for (int i = 0; i < PR; ++i) c[i] = fma2(mul2(d[i], wj[i]), rs, fma2(add2(c[i], minus_mu[k]), k2s, k1s));
          if (has_r) {
            get(2, j, k, row, d);
#pragma unroll
            for (int i = 0; i < PR; ++i) c[i] = add2(c[i], d[i]);
          }
          P out[G];
          from_pairs<P, W, G>(c, out);
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const int at = ((j + g) * threads + t) * W;
            if (at < q.d) *reinterpret_cast<P*>(static_cast<T*>(q.y) + row * q.y_ld + at) = out[g];
          }
        }
      }
    }
    if constexpr (RING) {
#pragma unroll
      for (int k = 0; k < ROWS; ++k) {
        issue(stage, row0 + (STAGES + k) * step);
        if (++stage == STAGES) stage = 0;
      }
    }
  }
  float* const shares = reinterpret_cast<float*>(ring);
  for (int g = 0; g < groups; ++g) {
    if (groups > 1) __syncthreads();
    if (g != group) continue;
#pragma unroll
    for (int which = 0; which < (BIAS ? 2 : 1); ++which) {
      if (!(which ? q.want_b : q.want_w)) continue;
      const int at = which ? (wanted - 1) * q.d : 0;
      if (which && far) continue;
      float f[N * W];
#pragma unroll
      for (int i = 0; i < E2; ++i) {
        F2 v;
        if constexpr (LONG) v = (which ? acc_b : acc)[i * blockDim.x];
        else v = which ? db[BIAS ? i : 0] : dw[i];
        split(v, f[2 * i], f[2 * i + 1]);
      }
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int c = (j * threads + t) * W;
        if (c < q.d) {
          constexpr int V = W >= 4 ? 4 : W;
#pragma unroll
          for (int k = 0; k < W; k += V) {
            Pack<float, V> a;
#pragma unroll
            for (int i = 0; i < V; ++i) a.v[i] = f[j * W + k + i];
            Pack<float, V>* const here = reinterpret_cast<Pack<float, V>*>(shares + at + c + k);
            if (g > 0) {
              const Pack<float, V> before = *here;
#pragma unroll
              for (int i = 0; i < V; ++i) a.v[i] += before.v[i];
            }
            if (g + 1 < groups) *here = a;
            else *reinterpret_cast<Pack<float, V>*>((which ? part_b : to_w) + c + k) = a;
          }
        }
      }
    }
  }
}

constexpr int REDUCE_WARPS = 32;
struct NormReduce { const float* part; int ctas, d, wanted; float *dw, *db; };
// Columns of the CTAs' shares added up: a lane takes a column, the warps take every 32nd CTA.
__global__ void __launch_bounds__(32 * REDUCE_WARPS) k_norm_reduce(const NormReduce q) {
  __shared__ float sums[REDUCE_WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, which = blockIdx.y;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float* const out = which || q.dw == nullptr ? q.db : q.dw;
  float s = 0.f;
  if (c < q.d) {
    const float* p = q.part + (long long)which * q.d + c;
#pragma unroll 8
    for (int g = warp; g < q.ctas; g += REDUCE_WARPS) s += p[(long long)g * q.wanted * q.d];
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

// Warps a row and groups a CTA for `per` elements a thread.
NormShape norm_shape(long long rows, int d, int per, long long rows_per_group, bool backward) {
  NormShape s;
  s.warps = (d + 32 * per - 1) / (32 * per);
  s.groups_per_cta = NORM_GROUP_THREADS / (32 * s.warps);
  if (s.groups_per_cta < 1) s.groups_per_cta = 1;
  const long long want = (rows + rows_per_group - 1) / rows_per_group;       // groups
  if (backward && want <= s.groups_per_cta) {
    s.groups_per_cta = (int)want;            // one CTA, which needs no second kernel (8 x 1024 bf16: 5.2 and 4.4 us, the call 15.0 and 13.2)
  } else {
    while (s.groups_per_cta > 1 && (want + s.groups_per_cta - 1) / s.groups_per_cta < sm_count()) --s.groups_per_cta;
  }
  s.ctas = 0;
  return s;
}
// And CTAs: as many as the rows ask for, or the GPU holds at one time.
void set_ctas(NormShape& s, long long rows, long long rows_per_group, int per_sm) {
  const long long want = (rows + rows_per_group - 1) / rows_per_group, need = (want + s.groups_per_cta - 1) / s.groups_per_cta;
  const long long most = (long long)sm_count() * (per_sm > 1 ? per_sm : 1);
  s.ctas = (int)(need < most ? need : most);
}

template <typename T, int W, int E, bool BIAS, bool RING, bool LOOSE, int THREADS, int ROWS = 1>
cudaError_t forward_as(const NormArgs& a, cudaStream_t st) {
  constexpr int N = E / W, STAGES = NORM_STAGES<N, THREADS, E>;
  constexpr auto KERN = k_norm_forward<T, W, N, BIAS, RING, LOOSE, THREADS, ROWS>;
  NormArgs q = a;
  NormShape s = norm_shape(q.rows, q.d, E, 1, false);
  q.warps = s.warps;
  const int threads = 32 * s.warps * s.groups_per_cta;
  int smem = 0;
  if constexpr (RING) {
    constexpr int MOST = STAGES * 2 * N * 16 * THREADS;
    static_assert(MOST <= 226 * 1024, "shared memory of an SM");
    const cudaError_t e = allow_smem<KERN, MOST>();
    if (e != cudaSuccess) return e;
    smem = STAGES * (q.r != nullptr ? 2 : 1) * N * threads * 16;
  }
  set_ctas(s, q.rows, 1, ctas_per_sm<KERN>(threads, smem));
  KERN<<<s.ctas, threads, smem, st>>>(q);
  return cudaGetLastError();
}
// Elements a thread: 8 where there are few rows (a row's loads and sums spread over most threads), where rows are short, and where
// they are read by elements (the next row then fits the registers of 1024 threads); 16 in rings, and of loose rows up to where the next
// row fits the registers of 512 threads; 32 where 1024 threads have to hold a longer row.
template <typename T, int W, bool LOOSE, bool BIAS>
cudaError_t forward_by(const NormArgs& q, cudaStream_t st) {
  constexpr bool RING = W * sizeof(T) == 16 && !LOOSE;
  if (q.d <= 256 || (q.d <= 8192 && ((!RING && !LOOSE) || q.rows <= 2 * sm_count()))) return forward_as<T, W, 8, BIAS, false, LOOSE, 1024>(q, st);
  if constexpr (RING) {
    if (q.d <= 8192) return q.rms ? forward_as<T, W, 16, BIAS, true, false, 512>(q, st) : forward_as<T, W, 16, BIAS, true, false, 512, 2>(q, st);
  } else if constexpr (LOOSE) {
    if (q.d <= 8192) return forward_as<T, W, 16, BIAS, false, true, 512>(q, st);
  }
  if (q.d <= 16384) return forward_as<T, W, 16, BIAS, RING, LOOSE, 1024>(q, st);
  return forward_as<T, W, 32, BIAS, false, LOOSE, 1024>(q, st);
}

// The backward pass: threads an SM is given (of 64 or 128 registers), and rows a group takes at least: a group's shares cost the second
// kernel as much as a few of its rows do here, more where rows are not read by 16 bytes.
constexpr int backward_threads(int per) { return per <= 8 ? 1024 : 512; }
int backward_rows(bool vec) { return vec ? 2 * BACKWARD_ROWS : BACKWARD_ROWS; }

// *ctas: how many shares there are to add up; none where one CTA wrote the gradients of the weights itself.
template <typename T, int W, int E, bool BIAS, bool LOOSE, int THREADS>
cudaError_t backward_as(const NormArgs& a, size_t room, bool* fits, int* ctas, cudaStream_t st) {
  constexpr int N = E / W, STAGES = NORM_STAGES<N, THREADS, E>;
  constexpr bool VEC = W * sizeof(T) == 16, LONG = THREADS > 512 && E >= 16;
  // fp32 rows off 16-byte boundaries are copied by words (24630 x 1192 with d_sum and bias: 205 us without the ring, 124 with it; short rows
  // lose by it: 30000 x 128 20 and 29 us)
  constexpr bool RING = VEC && (!LOOSE || (sizeof(T) == 4 && E == 16)) && (!LONG || (E == 16 && sizeof(T) == 2));
  constexpr auto KERN = k_norm_backward<T, W, N, BIAS, RING, LOOSE, THREADS>;
  NormArgs q = a;
  NormShape s = norm_shape(q.rows, q.d, E, backward_rows(VEC), true);
  const int threads = 32 * s.warps * s.groups_per_cta;
  set_ctas(s, q.rows, backward_rows(VEC), backward_threads(E) / threads);
  q.warps = s.warps;
  *ctas = s.ctas;
  if (s.ctas > 1 || ((reinterpret_cast<uintptr_t>(q.dw) | reinterpret_cast<uintptr_t>(q.db)) & 15)) q.dw = q.db = nullptr;
  if (q.dw != nullptr || q.db != nullptr) *ctas = 0;
  *fits = (size_t)s.ctas * (q.want_w + q.want_b) * q.d * 4 <= room;
  if (!*fits) return cudaSuccess;
  constexpr int ACC = LONG ? 4 * (BIAS ? 2 : 1) : 0;                    // bytes a column
  constexpr int MOST = (RING ? STAGES * 3 * N * 16 * THREADS : 0) + ACC * (E * THREADS < NORM_MAX_D ? E * THREADS : BIAS ? NORM_BOTH_D : NORM_MAX_D);
  static_assert(MOST <= 226 * 1024, "shared memory of an SM");
  // the groups' shares of a CTA take the ring's room, which is larger
  const int shares = s.groups_per_cta > 1 && !RING ? 4 * (q.want_w + q.want_b) * q.d : 0;
  static_assert(RING || LONG || 2 * 4 * (NORM_GROUP_THREADS / 2) * E <= 48 * 1024, "what a kernel may use without asking");
  const int smem = shares + (RING ? STAGES * (q.r != nullptr ? 3 : 2) * N * threads * 16 : 0) + (q.d <= NORM_BOTH_D ? ACC : ACC > 0 ? 4 : 0) * E * threads;
  if constexpr (MOST > 0) {
    const cudaError_t e = allow_smem<KERN, MOST>();
    if (e != cudaSuccess) return e;
  }
  return launch_chained(KERN, q, s.ctas, 1, 1, threads, smem, false, st);
}
template <typename T, int W, bool LOOSE, bool BIAS>
cudaError_t backward_by(const NormArgs& q, size_t room, bool* fits, int* ctas, cudaStream_t st) {
  constexpr bool VEC = W * sizeof(T) == 16;
  if constexpr (VEC) {
    if (q.d <= 256) return backward_as<T, W, 8, BIAS, LOOSE, 256>(q, room, fits, ctas, st);
    if (q.d <= 8192) return backward_as<T, W, 16, BIAS, LOOSE, 512>(q, room, fits, ctas, st);
  } else {
    if (q.d <= 128) return backward_as<T, W, 4, BIAS, LOOSE, 1024>(q, room, fits, ctas, st);
    if (q.d <= 8192) return backward_as<T, W, 8, BIAS, LOOSE, 1024>(q, room, fits, ctas, st);
  }
  if (q.d <= 16384) return backward_as<T, W, 16, BIAS, LOOSE, 1024>(q, room, fits, ctas, st);
  return backward_as<T, W, 32, BIAS, LOOSE, 1024>(q, room, fits, ctas, st);
}

// Shares of any alignment, and no fewer bytes for more rows, so that a workspace serves every smaller call: no more CTAs than groups,
// and those are what the rows ask for, rounded up to whole CTAs, or as many as the GPU holds at one time.
size_t norm_part_bound(int64_t rows, int d) {
  // of 8 elements a thread, or of 16
  const int short_sm = backward_threads(8) / 32 / ((d + 255) / 256), long_sm = backward_threads(16) / 32 / ((d + 511) / 512);
  const int most_sm = short_sm > long_sm ? short_sm : long_sm;
  const int64_t want = (rows + BACKWARD_ROWS - 1) / BACKWARD_ROWS + NORM_GROUP_THREADS / 32, most = (int64_t)sm_count() * (most_sm > 1 ? most_sm : 1);
  return (size_t)(want < most ? want : most) * 2 * d * 4;
}

// How the matrices of a call can be accessed; p and ld of each (p null: none), and the weights.  BY_LOOSE: what is written is on 16-byte
// boundaries, what is read is not; a thread then still takes 16 bytes in a row, read one by one (rows on odd elements, bf16: layer norm
// of 1354 x 7872 48 us by single elements, 24 so; backward with d_sum and bias, 1259 x 8768, 378 and 73).
constexpr int BY_LOOSE = BY_ONE + 1;
struct Rows { const void* p; long long ld; };
template <int K, int L>
int access_of(const Rows (&in)[K], const Rows (&out)[L], int d, int size, const void* w, const void* b, int w_size) {
  auto all = [&](const auto& m, int unit) {
    bool on = true;
    for (const Rows& r : m) on = on && rows_on(r.p, r.ld, size, unit);
    return on;
  };
  if ((d * size) % 16 == 0 && all(out, 16)) return all(in, 16) && rows_on(w, 0, 1, 16) && rows_on(b, 0, 1, 16) ? BY_16 : BY_LOOSE;
  return d % 2 == 0 && all(in, 2 * size) && all(out, 2 * size) && rows_on(w, 0, 1, 2 * w_size) && rows_on(b, 0, 1, 2 * w_size) ? BY_TWO : BY_ONE;
}

template <typename T, bool BIAS>
cudaError_t forward_any(const NormArgs& q, int access, cudaStream_t st) {
  return access == BY_16    ? forward_by<T, 16 / (int)sizeof(T), false, BIAS>(q, st)
       : access == BY_LOOSE ? forward_by<T, 16 / (int)sizeof(T), true, BIAS>(q, st)
       : access == BY_TWO   ? forward_by<T, 2, false, BIAS>(q, st)
                            : forward_by<T, 1, false, BIAS>(q, st);
}
template <typename T, bool BIAS>
cudaError_t backward_any(const NormArgs& q, int access, size_t room, bool* fits, int* ctas, cudaStream_t st) {
  return access == BY_16    ? backward_by<T, 16 / (int)sizeof(T), false, BIAS>(q, room, fits, ctas, st)
       : access == BY_LOOSE ? backward_by<T, 16 / (int)sizeof(T), true, BIAS>(q, room, fits, ctas, st)
       : access == BY_TWO   ? backward_by<T, 2, false, BIAS>(q, room, fits, ctas, st)
                            : backward_by<T, 1, false, BIAS>(q, room, fits, ctas, st);
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
  const int access = access_of({Rows{q.x, q.x_ld}, Rows{q.r, q.r_ld}}, {Rows{q.sum, q.sum_ld}, Rows{q.y, q.y_ld}}, q.d, size, q.w, q.b, q.w_f32 ? 4 : 2);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (size == 2) NORM_CK(q.b != nullptr ? forward_any<__nv_bfloat16, true>(q, access, st) : forward_any<__nv_bfloat16, false>(q, access, st));
  else NORM_CK(q.b != nullptr ? forward_any<float, true>(q, access, st) : forward_any<float, false>(q, access, st));
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
  q.part = static_cast<float*>(workspace); q.want_w = d_weight != nullptr; q.want_b = d_bias != nullptr; q.dw = d_weight; q.db = d_bias;
  const int size = n->dtype == CAMERA_BF16 ? 2 : 4;
  const int access = access_of({Rows{q.x, q.x_ld}, Rows{q.r, q.r_ld}, Rows{q.dy, q.dy_ld}}, {Rows{q.y, q.y_ld}}, q.d, size, q.w, nullptr, q.w_f32 ? 4 : 2);
  if (want_w && (workspace == nullptr || (reinterpret_cast<uintptr_t>(workspace) & 255))) return CAMERA_ERR_WORKSPACE;
  bool fits = false;
  int ctas = 0;
  if (size == 2)
    NORM_CK(q.want_b ? backward_any<__nv_bfloat16, true>(q, access, workspace_bytes, &fits, &ctas, st)
                     : backward_any<__nv_bfloat16, false>(q, access, workspace_bytes, &fits, &ctas, st));
  else
    NORM_CK(q.want_b ? backward_any<float, true>(q, access, workspace_bytes, &fits, &ctas, st)
                     : backward_any<float, false>(q, access, workspace_bytes, &fits, &ctas, st));
  if (!fits) return CAMERA_ERR_WORKSPACE;
  if (want_w && ctas > 0) {
    const NormReduce r = {q.part, ctas, q.d, q.want_w + q.want_b, d_weight, d_bias};
    NORM_CK(launch_chained(k_norm_reduce, r, (q.d + 31) / 32, r.wanted, 1, 32 * REDUCE_WARPS, 0, true, st));
  }
  return CAMERA_OK;
}
