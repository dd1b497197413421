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
  float* part;                             // backward: [groups][2][d] partial sums of dw and db
  bool want_w;
};

template <int W>
__device__ __forceinline__ void load_weight(const void* p, bool f32, int c, float absent, float* out) {
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
    const Pack<__nv_bfloat16, W> t = *reinterpret_cast<const Pack<__nv_bfloat16, W>*>(static_cast<const __nv_bfloat16*>(p) + c);
#pragma unroll
    for (int i = 0; i < W; ++i) out[i] = __bfloat162float(t.v[i]);
  }
}

// W elements a load (16 bytes, or 1 element where rows or the width are not aligned for that), N loads a thread.
template <typename T, int W, int N, bool RES>
__global__ void __launch_bounds__(1024, 1) k_norm_forward(const NormArgs q) {
  using P = Pack<T, W>;
  constexpr bool AHEAD = N * W * (int)sizeof(T) <= 32;     // the next row in registers too
  const int threads = 32 * q.warps, group = threadIdx.x / threads, t = threadIdx.x - group * threads;
  const int groups = blockDim.x / threads;
  const long long step = (long long)gridDim.x * groups;
  const T* const x = static_cast<const T*>(q.x);
  const T* const r = static_cast<const T*>(q.r);
  int buf = 0;
  P nx[N], nr[RES ? N : 1];
  auto load = [&](long long row) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = (j * threads + t) * W;
      if (c < q.d) {
        nx[j] = *reinterpret_cast<const P*>(x + row * q.x_ld + c);
        if (RES) nr[j] = *reinterpret_cast<const P*>(r + row * q.r_ld + c);
      }
    }
  };
  long long row = (long long)blockIdx.x * groups + group;
  if (AHEAD && row < q.rows) load(row);
  for (; row < q.rows; row += step) {
    if (!AHEAD) load(row);
    float z[N * W], s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = (j * threads + t) * W;
      if (c < q.d) {
        P keep;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          float v = to_f32(nx[j].v[i]);
          if (RES) {
            keep.v[i] = from_f32<T>(v + to_f32(nr[j].v[i]));
            v = to_f32(keep.v[i]);
          }
          z[j * W + i] = v;
          s[0] += v;
        }
        if (RES) *reinterpret_cast<P*>(static_cast<T*>(q.sum) + row * q.sum_ld + c) = keep;
      }
    }
    if (AHEAD && row + step < q.rows) load(row + step);
    float mu = 0.f;
    if (!q.rms) {
      group_sum(s, q.warps, group, buf);
      mu = s[0] / (float)q.d;
    }
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if ((j * threads + t) * W < q.d) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
          z[j * W + i] -= mu;
          s[0] = fmaf(z[j * W + i], z[j * W + i], s[0]);
        }
      }
    group_sum(s, q.warps, group, buf);
    const float rstd = 1.f / sqrtf(s[0] / (float)q.d + q.eps);
    if (t == 0) {
      if (q.mean != nullptr) q.mean[row] = mu;
      if (q.rstd != nullptr) q.rstd[row] = rstd;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = (j * threads + t) * W;
      if (c < q.d) {
        float w[W], b[W];
        load_weight<W>(q.w, q.w_f32, c, 1.f, w);
        load_weight<W>(q.b, q.w_f32, c, 0.f, b);
        P out;
#pragma unroll
        for (int i = 0; i < W; ++i) out.v[i] = from_f32<T>(fmaf(z[j * W + i] * rstd, w[i], b[i]));
        *reinterpret_cast<P*>(static_cast<T*>(q.y) + row * q.y_ld + c) = out;
      }
    }
  }
}

// A thread keeps the columns it owns for all rows of its group, so their shares of dw and db stay in its registers; the
// groups' shares are added up by k_norm_reduce in a fixed order.
template <typename T, int W, int N>
__global__ void __launch_bounds__(N * W <= 16 ? 512 : 1024, 1) k_norm_backward(const NormArgs q) {
  using P = Pack<T, W>;
  constexpr bool AHEAD = N * W <= 16;
  const int threads = 32 * q.warps, group = threadIdx.x / threads, t = threadIdx.x - group * threads;
  const int groups = blockDim.x / threads;
  const long long step = (long long)gridDim.x * groups;
  const T* const x = static_cast<const T*>(q.x);
  const T* const r = static_cast<const T*>(q.r);
  const T* const dy = static_cast<const T*>(q.dy);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int buf = 0;
  P nx[N], ny[N], nr[N];
  float dw[N * W], db[N * W];
#pragma unroll
  for (int i = 0; i < N * W; ++i) dw[i] = db[i] = 0.f;
  auto load = [&](long long row) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = (j * threads + t) * W;
      if (c < q.d) {
        nx[j] = *reinterpret_cast<const P*>(x + row * q.x_ld + c);
        ny[j] = *reinterpret_cast<const P*>(dy + row * q.dy_ld + c);
        if (r != nullptr) nr[j] = *reinterpret_cast<const P*>(r + row * q.r_ld + c);
      }
    }
  };
  const long long first = (long long)blockIdx.x * groups + group;
  if (AHEAD && first < q.rows) load(first);
  for (long long row = first; row < q.rows; row += step) {
    if (!AHEAD) load(row);
    P cx[N], cy[N], cr[N];
#pragma unroll
    for (int j = 0; j < N; ++j) { cx[j] = nx[j]; cy[j] = ny[j]; cr[j] = nr[j]; }
    if (AHEAD && row + step < q.rows) load(row + step);
    const float mu = q.rms ? 0.f : q.mean[row], rstd = q.rstd[row];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = (j * threads + t) * W;
      if (c < q.d) {
        float w[W];
        load_weight<W>(q.w, q.w_f32, c, 1.f, w);
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float h = (to_f32(cx[j].v[i]) - mu) * rstd, d = to_f32(cy[j].v[i]), g = d * w[i];
          s[0] += g;
          s[1] = fmaf(g, h, s[1]);
          dw[j * W + i] = fmaf(d, h, dw[j * W + i]);
          db[j * W + i] += d;
        }
      }
    }
    if (q.y == nullptr) continue;
    group_sum(s, q.warps, group, buf);
    const float m1 = q.rms ? 0.f : s[0] / (float)q.d, m2 = s[1] / (float)q.d;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int c = (j * threads + t) * W;
      if (c < q.d) {
        float w[W];
        load_weight<W>(q.w, q.w_f32, c, 1.f, w);
        P out;
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float h = (to_f32(cx[j].v[i]) - mu) * rstd, g = to_f32(cy[j].v[i]) * w[i];
          float v = (g - m1 - h * m2) * rstd;
          if (r != nullptr) v += to_f32(cr[j].v[i]);
          out.v[i] = from_f32<T>(v);
        }
        *reinterpret_cast<P*>(static_cast<T*>(q.y) + row * q.y_ld + c) = out;
      }
    }
  }
  if (!q.want_w) return;
  float* const part = q.part + first * 2 * q.d;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int c = (j * threads + t) * W;
    if (c < q.d) {
      constexpr int V = W >= 4 ? 4 : 1;
#pragma unroll
      for (int k = 0; k < W; k += V) {
        Pack<float, V> a, b;
#pragma unroll
        for (int i = 0; i < V; ++i) { a.v[i] = dw[j * W + k + i]; b.v[i] = db[j * W + k + i]; }
        *reinterpret_cast<Pack<float, V>*>(part + c + k) = a;
        *reinterpret_cast<Pack<float, V>*>(part + q.d + c + k) = b;
      }
    }
  }
}

constexpr int REDUCE_WARPS = 16;
struct NormReduce { const float* part; int groups, d; float *dw, *db; };
// Columns of the groups' shares added up: a lane takes a column, the warps take every 16th group.
__global__ void __launch_bounds__(32 * REDUCE_WARPS) k_norm_reduce(const NormReduce q) {
  __shared__ float sums[REDUCE_WARPS][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane, which = blockIdx.y;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  float* const out = which ? q.db : q.dw;
  if (out == nullptr) return;
  float s = 0.f;
  if (c < q.d) {
    const float* p = q.part + (long long)which * q.d + c;
#pragma unroll 8
    for (int g = warp; g < q.groups; g += REDUCE_WARPS) s += p[(long long)g * 2 * q.d];
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
NormShape backward_shape(long long rows, int d) { return norm_shape(rows, d, backward_per(d), 512, BACKWARD_ROWS); }

template <typename T, int W, int N>
cudaError_t forward_as(const NormArgs& a, cudaStream_t st) {
  NormArgs q = a;
  const NormShape s = norm_shape(q.rows, q.d, N * W, 1024, 1);
  q.warps = s.warps;
  const int threads = 32 * s.warps * s.groups_per_cta;
  if (q.r != nullptr) k_norm_forward<T, W, N, true><<<s.ctas, threads, 0, st>>>(q);
  else k_norm_forward<T, W, N, false><<<s.ctas, threads, 0, st>>>(q);
  return cudaGetLastError();
}
template <typename T>
cudaError_t forward_typed(const NormArgs& q, bool vec, cudaStream_t st) {
  constexpr int W = 16 / (int)sizeof(T);
  if (!vec) return q.d <= 8 * 1024 ? forward_as<T, 1, 8>(q, st) : forward_as<T, 1, 32>(q, st);
  // Few rows: one load a thread, so that a row's loads and sums are spread over most threads.
  if (q.rows <= 2 * sm_count() && q.d <= W * 1024) return forward_as<T, W, 1>(q, st);
  if (q.d <= 2 * W * 1024) return forward_as<T, W, 2>(q, st);
  return forward_as<T, W, 32 / W>(q, st);
}

template <typename T, int W, int N>
cudaError_t backward_as(const NormArgs& a, const NormShape& s, cudaStream_t st) {
  NormArgs q = a;
  q.warps = s.warps;
  return launch_chained(k_norm_backward<T, W, N>, q, s.ctas, 1, 1, 32 * s.warps * s.groups_per_cta, 0, false, st);
}
template <typename T>
cudaError_t backward_typed(const NormArgs& q, const NormShape& s, bool vec, cudaStream_t st) {
  constexpr int W = 16 / (int)sizeof(T);
  const bool small = backward_per(q.d) == 16;
  if (!vec) return small ? backward_as<T, 1, 16>(q, s, st) : backward_as<T, 1, 32>(q, s, st);
  return small ? backward_as<T, W, 16 / W>(q, s, st) : backward_as<T, W, 32 / W>(q, s, st);
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

size_t norm_part_bytes(int64_t rows, int d) {
  const NormShape s = backward_shape(rows, d);
  return (size_t)s.ctas * s.groups_per_cta * 2 * d * 4;
}
// At least that, and no less for more rows, so that a workspace serves every smaller call: groups are what the rows ask for,
// rounded up to whole CTAs, or as many as the GPU holds at one time.
size_t norm_part_bound(int64_t rows, int d) {
  const int warps = (d + 32 * backward_per(d) - 1) / (32 * backward_per(d));
  const int64_t want = (rows + BACKWARD_ROWS - 1) / BACKWARD_ROWS + NORM_GROUP_THREADS / 32, most = (int64_t)sm_count() * (16 / warps > 1 ? 16 / warps : 1);
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
  NORM_CK(size == 2 ? forward_typed<__nv_bfloat16>(q, vec, st) : forward_typed<float>(q, vec, st));
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
  if (want_w && (workspace == nullptr || workspace_bytes < norm_part_bytes(n->n_rows, n->d) || (reinterpret_cast<uintptr_t>(workspace) & 255)))
    return CAMERA_ERR_WORKSPACE;
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
  q.part = static_cast<float*>(workspace); q.want_w = want_w;
  const int size = n->dtype == CAMERA_BF16 ? 2 : 4;
  const bool vec = (n->d * size) % 16 == 0 && vec_ok(q.x, q.x_ld, size) && vec_ok(q.r, q.r_ld, size) && vec_ok(q.dy, q.dy_ld, size) &&
                   vec_ok(q.y, q.y_ld, size) && vec_ok(q.w, 0, 1);
  const NormShape s = backward_shape(q.rows, q.d);
  NORM_CK(size == 2 ? backward_typed<__nv_bfloat16>(q, s, vec, st) : backward_typed<float>(q, s, vec, st));
  if (want_w) {
    const NormReduce r = {q.part, s.ctas * s.groups_per_cta, q.d, d_weight, d_bias};
    NORM_CK(launch_chained(k_norm_reduce, r, (q.d + 31) / 32, 2, 1, 32 * REDUCE_WARPS, 0, true, st));
  }
  return CAMERA_OK;
}
