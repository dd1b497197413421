// Tokens sorted by expert and back, with the gradients of both.
//   rows[t, j]  place of the pair (token t, slot j) when all pairs are sorted by expert (within one by t, then j)
//   dispatch           xs[rows[t, j]] = x[t]
//   combine            y[t] = add[t] + sum_j w[t, j] ys[rows[t, j]]
//   combine, backward  dys[rows[t, j]] = w[t, j] dy[t],  dw[t, j] = <dy[t], ys[rows[t, j]]>
//   dispatch, backward dx[t] = add[t] + sum_j dxs[rows[t, j]]  (a combine without weights)
// All of it is moving rows, bound by HBM.  16384 tokens to 8 of 64 experts, 3584 bf16: dispatch 200 us (1058 MB, 940 of them written:
// 5.3 TB/s; a plain fill of the 940 MB takes 240 us, and hints on the stores, other runs of tokens per CTA and more rows in flight changed
// nothing), combine 180 us (1175 MB, 6.5
// TB/s), its backward pass 320 us (1998 MB, 6.2 TB/s).  Where there are few tokens it is latency: dispatch of 64 tokens 6 us, of which
// counting and ranking take half.
#include "common.cuh"
#include "launch.cuh"
#include "rowgroup.cuh"

namespace camera {

namespace {

constexpr int MOE_MAX_EXPERTS = 1024, MOE_MAX_D = 1 << 20;
constexpr int MOE_THREADS = 256, MOE_WARPS = MOE_THREADS / 32;
// Up to so many pairs every CTA counts all of them for itself; beyond, a kernel before counts them chunk by chunk.
constexpr long long MOE_SMALL = 16384;

struct Dispatch {
  const void* x;
  void* xs;
  long long x_ld, xs_ld;
  const int32_t* idx;
  int32_t *rows, *offsets;
  int32_t* hist;                 // [experts][chunks] pairs per expert and chunk, then those of the chunks before; or null
  int32_t* totals;               // [experts]
  int tokens, k, experts, d;
  int chunk, chunks;             // tokens a CTA handles, CTAs
};

__device__ __forceinline__ bool usable(int e, int experts) { return (unsigned)e < (unsigned)experts; }

__global__ void __launch_bounds__(MOE_THREADS) k_moe_count(const Dispatch q) {
  extern __shared__ int32_t count[];
  for (int e = threadIdx.x; e < q.experts; e += MOE_THREADS) count[e] = 0;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __syncthreads();
  const long long p0 = (long long)blockIdx.x * q.chunk * q.k, p1 = min(p0 + (long long)q.chunk * q.k, (long long)q.tokens * q.k);
  for (long long p = p0 + threadIdx.x; p < p1; p += MOE_THREADS) {
    const int e = q.idx[p];
    if (usable(e, q.experts)) atomicAdd(&count[e], 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < q.experts; e += MOE_THREADS) q.hist[(long long)e * gridDim.x + blockIdx.x] = count[e];
}

// A warp per expert: exclusive sums over the chunks.  The kernel after it is let in when this one ends, not before: CTAs that
// come while those of k_moe_count still run spread unevenly over the SMs (16384 tokens to 8 of 64 experts: 206 -> 245 us).
constexpr int SCAN_WARPS = 4;
__global__ void __launch_bounds__(32 * SCAN_WARPS) k_moe_scan(const Dispatch q) {
  const int e = blockIdx.x * SCAN_WARPS + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (e >= q.experts) return;
  int32_t* const hist = q.hist + (long long)e * q.chunks;
  constexpr int R = 10;              // chunks a lane holds at a time: 2 * 148 chunks are one pass
  int before = 0;
  for (int c0 = 0; c0 < q.chunks; c0 += 32 * R) {
    int v[R];
#pragma unroll
    for (int i = 0; i < R; ++i) v[i] = c0 + 32 * i + lane < q.chunks ? hist[c0 + 32 * i + lane] : 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      int sum = v[i];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += up;
      }
      if (c0 + 32 * i + lane < q.chunks) hist[c0 + 32 * i + lane] = before + sum - v[i];
      before += __shfl_sync(0xffffffffu, sum, 31);
    }
  }
  if (lane == 0) q.totals[e] = before;
}

// A CTA takes a run of consecutive tokens: it finds where each expert's rows begin and how many pairs lie before its own,
// ranks its pairs (a warp takes a run of them, 32 at a time), and copies its tokens, read once, to their k rows.
template <typename T, int W>
__global__ void __launch_bounds__(MOE_THREADS) k_moe_dispatch(const Dispatch q) {
  using P = Pack<T, W>;
  extern __shared__ int32_t sh[];
  int32_t* const total = sh;                       // [experts]
  int32_t* const before = sh + q.experts;          // [experts] pairs of the CTAs before this one
  int32_t* const next = sh + 2 * q.experts;        // [warps][experts] pairs of the warp, then where its next one goes
  __shared__ int32_t warp_sum[MOE_WARPS];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, E = q.experts;
  for (int i = tid; i < (2 + MOE_WARPS) * E; i += MOE_THREADS) sh[i] = 0;
  __syncthreads();
  const long long pairs = (long long)q.tokens * q.k;
  const long long p0 = (long long)blockIdx.x * q.chunk * q.k, p1 = min(p0 + (long long)q.chunk * q.k, pairs);
  const long long seg = ((p1 - p0 + MOE_WARPS - 1) / MOE_WARPS + 31) & ~31ll;      // pairs a warp ranks
  const long long w0 = min(p0 + warp * seg, p1), w1 = min(w0 + seg, p1);
  for (long long p = w0 + lane; p < w1; p += 32) {
    const int e = q.idx[p];
    if (usable(e, E)) atomicAdd(&next[warp * E + e], 1);
  }
  if (q.hist == nullptr) {
    for (long long p = tid; p < pairs; p += MOE_THREADS) {
      const int e = q.idx[p];
      if (usable(e, E)) {
        atomicAdd(&total[e], 1);
        if (p < p0) atomicAdd(&before[e], 1);
      }
    }
  } else {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int e = tid; e < E; e += MOE_THREADS) {
      total[e] = q.totals[e];
      before[e] = q.hist[(long long)e * q.chunks + blockIdx.x];
    }
  }
  __syncthreads();
  // exclusive scan over the experts: a thread takes `per` consecutive ones
  const int per = (E + MOE_THREADS - 1) / MOE_THREADS;
  int sum = 0;
  for (int i = 0; i < per; ++i) {
    const int e = tid * per + i;
    if (e < E) sum += total[e];
  }
  int scan = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += v;
  }
  if (lane == 31) warp_sum[warp] = scan;
  __syncthreads();
  int at = scan - sum;
  for (int i = 0; i < warp; ++i) at += warp_sum[i];
  for (int i = 0; i < per; ++i) {
    const int e = tid * per + i;
    if (e >= E) break;
    const int n = total[e];
    if (blockIdx.x == 0) q.offsets[e] = at;
    int go = at + before[e];
    for (int w = 0; w < MOE_WARPS; ++w) {
      const int v = next[w * E + e];
      next[w * E + e] = go;
      go += v;
    }
    at += n;
    if (blockIdx.x == 0 && e == E - 1) q.offsets[E] = at;
  }
  __syncthreads();
  for (long long p = w0; p < w1; p += 32) {
    const bool here = p + lane < w1;
    const int e = here ? q.idx[p + lane] : -1;
    const bool ok = usable(e, E);
    const unsigned same = __match_any_sync(0xffffffffu, ok ? e : -1 - lane);
    int row = -1;
    if (ok) row = next[warp * E + e] + __popc(same & ((1u << lane) - 1u));
    __syncwarp();
    if (ok && lane == 31 - __clz(same)) next[warp * E + e] = row + 1;
    __syncwarp();
    if (here) q.rows[p + lane] = row;
  }
  __syncthreads();
  const T* const x = static_cast<const T*>(q.x);
  T* const xs = static_cast<T*>(q.xs);
  constexpr int U = 4;
  const long long first = (long long)blockIdx.x * q.chunk, t1 = min(first + q.chunk, (long long)q.tokens);
  if (q.d <= 32 * W) {                  // short rows: a token's in one load, U tokens at a time
    for (long long t0 = first + warp; t0 < t1; t0 += U * MOE_WARPS) {
      const int c = lane * W;
      P v[U];
      int mine[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long t = t0 + u * MOE_WARPS;
        if (t < t1 && c < q.d) v[u] = *reinterpret_cast<const P*>(x + t * q.x_ld + c);
        mine[u] = t < t1 && lane < q.k ? q.rows[t * q.k + lane] : -1;
      }
      for (int j = 0; j < q.k; ++j)
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int row = __shfl_sync(0xffffffffu, mine[u], j);
          if (row >= 0 && c < q.d) *reinterpret_cast<P*>(xs + row * q.xs_ld + c) = v[u];
        }
    }
    return;
  }
  for (long long t = first + warp; t < t1; t += MOE_WARPS) {
    const int mine = lane < q.k ? q.rows[t * q.k + lane] : -1;
    for (int c0 = 0; c0 < q.d; c0 += U * 32 * W) {
      P v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int c = c0 + (32 * u + lane) * W;
        if (c < q.d) v[u] = *reinterpret_cast<const P*>(x + t * q.x_ld + c);
      }
      for (int j = 0; j < q.k; ++j) {
        const int row = __shfl_sync(0xffffffffu, mine, j);
        if (row < 0) continue;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int c = c0 + (32 * u + lane) * W;
          if (c < q.d) *reinterpret_cast<P*>(xs + row * q.xs_ld + c) = v[u];
        }
      }
    }
  }
}

struct Combine {
  const void *ys, *add, *dy;
  void *y, *dys;
  long long ys_ld, add_ld, y_ld, dy_ld, dys_ld;
  long long n_rows;              // rows of ys: an entry of `rows` outside is no row
  const int32_t* rows;
  const float* w;                // or null: ones
  float* dw;
  int tokens, k, d;
  int warps;                     // backward: warps that share a token
};

// A thread takes U packs of one token, its k rows S at a time (S x U loads in flight), added in the order of the slots.  fp32 sums,
// rounded once.  With the weights read among the loads, each load waited for the one before (16384 tokens: 329 us instead of 180).
template <typename T, int W, int S, int U>
__global__ void __launch_bounds__(256, U == 1 ? 4 : U == 2 ? 3 : 2) k_moe_combine(const Combine q) {
  using P = Pack<T, W>;
  const long long t = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  const int c0 = (blockIdx.y * U * blockDim.x + threadIdx.x) * W, step = blockDim.x * W;
  if (t >= q.tokens) return;
  const T* const ys = static_cast<const T*>(q.ys) + c0;
  P extra[U];
  if (q.add != nullptr) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (c0 + u * step < q.d) extra[u] = *reinterpret_cast<const P*>(static_cast<const T*>(q.add) + t * q.add_ld + c0 + u * step);
  }
  float sum[U][W];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < W; ++i) sum[u][i] = 0.f;
  for (int j0 = 0; j0 < q.k; j0 += S) {
    // Row numbers first, then all loads, weights when they are needed: registers decide how many threads an SM holds, and with them
    // the loads in flight.
    int row[S];
    P v[S][U];
#pragma unroll
    for (int j = 0; j < S; ++j) {
      row[j] = j0 + j < q.k ? q.rows[t * q.k + j0 + j] : -1;
      if (row[j] >= q.n_rows) row[j] = -1;
    }
#pragma unroll
    for (int j = 0; j < S; ++j)
      if (row[j] >= 0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (c0 + u * step < q.d) v[j][u] = *reinterpret_cast<const P*>(ys + row[j] * q.ys_ld + u * step);
      }
#pragma unroll
    for (int j = 0; j < S; ++j)
      if (row[j] >= 0) {
        const float w = q.w != nullptr ? q.w[t * q.k + j0 + j] : 1.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float f[W];
          v[j][u].get(f);
#pragma unroll
          for (int i = 0; i < W; ++i) sum[u][i] = fmaf(w, f[i], sum[u][i]);
        }
      }
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (c0 + u * step < q.d) {
      if (q.add != nullptr) {
        float f[W];
        extra[u].get(f);
#pragma unroll
        for (int i = 0; i < W; ++i) sum[u][i] += f[i];
      }
      P out;
      out.set(sum[u]);
      *reinterpret_cast<P*>(static_cast<T*>(q.y) + t * q.y_ld + c0 + u * step) = out;
    }
}

// A group of warps takes a token: its row of dy goes, times each weight, to its k rows, and meets the k rows of ys in dot products that
// stay in registers until the row's end (fp32; a product is rounded once, where it is stored).  S slots at a time, so that dy is read
// from L2 again only beyond eight.  DOTS: with the gradient of the weights; without it nothing is read but dy.
template <typename T, int W, int S, int U, bool DOTS>
__global__ void __launch_bounds__(512, 1) k_moe_combine_backward(const Combine q) {
  using P = Pack<T, W>;
  const int threads = 32 * q.warps, group = threadIdx.x / threads, i0 = threadIdx.x - group * threads;
  const long long t = (long long)blockIdx.x * (blockDim.x / threads) + group;
  if (t >= q.tokens) return;
  const T* const dy = static_cast<const T*>(q.dy) + t * q.dy_ld;
  const T* const ys = static_cast<const T*>(q.ys);
  T* const dys = static_cast<T*>(q.dys);
  int buf = 0;
  for (int j0 = 0; j0 < q.k; j0 += S) {
    int row[S];
    float w[S], dot[S];
#pragma unroll
    for (int j = 0; j < S; ++j) {
      row[j] = j0 + j < q.k ? q.rows[t * q.k + j0 + j] : -1;
      if (row[j] >= q.n_rows) row[j] = -1;
      w[j] = row[j] >= 0 && q.w != nullptr ? q.w[t * q.k + j0 + j] : 1.f;
      dot[j] = 0.f;
    }
    const int step = threads * W;
    for (int c0 = i0 * W; c0 < q.d; c0 += U * step) {
      P g[U], v[DOTS ? S : 1][U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (c0 + u * step < q.d) g[u] = *reinterpret_cast<const P*>(dy + c0 + u * step);
      if constexpr (DOTS) {
#pragma unroll
        for (int j = 0; j < S; ++j)
          if (row[j] >= 0) {
#pragma unroll
            for (int u = 0; u < U; ++u)
              if (c0 + u * step < q.d) v[j][u] = *reinterpret_cast<const P*>(ys + row[j] * q.ys_ld + c0 + u * step);
          }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (c0 + u * step >= q.d) break;
        float d[W];
        g[u].get(d);
#pragma unroll
        for (int j = 0; j < S; ++j)
          if (row[j] >= 0) {
            P out;
            float f[W];
            if constexpr (DOTS) {
              v[j][u].get(f);
#pragma unroll
              for (int i = 0; i < W; ++i) dot[j] = fmaf(d[i], f[i], dot[j]);
            }
#pragma unroll
            for (int i = 0; i < W; ++i) f[i] = w[j] * d[i];
            out.set(f);
            if (q.dys != nullptr) *reinterpret_cast<P*>(dys + row[j] * q.dys_ld + c0 + u * step) = out;
          }
      }
    }
    if constexpr (!DOTS) continue;
    group_sum(dot, q.warps, group, buf);
    if (i0 == 0) {
#pragma unroll
      for (int j = 0; j < S; ++j)
        if (j0 + j < q.k) q.dw[t * q.k + j0 + j] = dot[j];
    }
  }
}

// ------------------------------------------------------------------------------------------------ host side
int moe_ctas(int64_t tokens) {
  const int64_t most = 2 * (int64_t)sm_count();
  return (int)(tokens < most ? tokens : most);
}
size_t moe_hist_bytes(int64_t tokens, int k, int experts) {
  return tokens * k <= MOE_SMALL ? 0 : (size_t)4 * (moe_ctas(tokens) + 1) * experts;
}

bool sizes_ok(int64_t tokens, int k, int d, int32_t dtype) {
  return tokens >= 0 && k >= 1 && d >= 1 && (dtype == CAMERA_BF16 || dtype == CAMERA_F32);
}
bool sizes_fit(int64_t tokens, int k, int d) { return k <= MAX_TOPK && tokens < (1ll << 31) && tokens * k < (1ll << 31) && d <= MOE_MAX_D; }
bool rows_fit(const void* p, int64_t ld, int d, int size) {
  return p != nullptr && ld >= d && (reinterpret_cast<uintptr_t>(p) & (size - 1)) == 0;
}
bool words_ok(const void* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

#define MOE_CK(...)             \
  do {                          \
    if ((__VA_ARGS__) != cudaSuccess) { \
      cudaGetLastError();       \
      return CAMERA_ERR_CUDA;   \
    }                           \
  } while (0)

template <typename T>
cudaError_t launch_dispatch(const Dispatch& q, int access, int ctas, cudaStream_t st) {
  const int smem = 4 * q.experts * (2 + MOE_WARPS);
  return launch_chained(access == BY_16 ? k_moe_dispatch<T, 16 / (int)sizeof(T)> : access == BY_TWO ? k_moe_dispatch<T, 2> : k_moe_dispatch<T, 1>, q, ctas, 1, 1,
                        MOE_THREADS, smem, q.hist != nullptr, st);
}
// Slots S and packs U a thread: as many loads in flight whatever k is (8 vectors or 16 elements), but one pack a thread where one
// wave of threads takes all of them.
template <typename T, int W, int S, int U>
cudaError_t combine_as(const Combine& q, cudaStream_t st) {
  const int packs = (q.d + W - 1) / W, slices = (packs + 256 * U - 1) / (256 * U);
  const int bx = ((packs + slices * U - 1) / (slices * U) + 31) & ~31, ty = 256 / bx;
  k_moe_combine<T, W, S, U><<<dim3((unsigned)(((long long)q.tokens + ty - 1) / ty), (unsigned)slices), dim3((unsigned)bx, (unsigned)ty), 0, st>>>(q);
  return cudaGetLastError();
}
template <typename T, int W>
cudaError_t launch_combine_as(const Combine& q, cudaStream_t st) {
  constexpr bool VEC = W * sizeof(T) == 16;
  constexpr int F = VEC ? 8 : 16;
  const bool one = (long long)q.tokens * ((q.d + W - 1) / W) <= 1024ll * sm_count();
  if (q.k == 1) return one ? combine_as<T, W, 1, 1>(q, st) : combine_as<T, W, 1, F / 2>(q, st);
  if (q.k == 2) return one ? combine_as<T, W, 2, 1>(q, st) : combine_as<T, W, 2, F / 2>(q, st);
  if (q.k <= 4) return one ? combine_as<T, W, 4, 1>(q, st) : combine_as<T, W, 4, F / 4>(q, st);
  if constexpr (VEC) return combine_as<T, W, 8, 1>(q, st);
  else return one ? combine_as<T, W, 8, 1>(q, st) : combine_as<T, W, 8, F / 8>(q, st);
}
template <typename T, int W, int S, int U, bool DOTS = true>
cudaError_t combine_backward_as(const Combine& a, int each, cudaStream_t st) {
  Combine q = a;
  const int packs = (q.d + W - 1) / W;
  q.warps = (packs + 32 * each - 1) / (32 * each);
  if (q.warps > 16) q.warps = 16;
  const int groups = q.warps >= 4 ? 1 : 4 / q.warps;
  k_moe_combine_backward<T, W, S, U, DOTS><<<(unsigned)(((long long)q.tokens + groups - 1) / groups), 32 * q.warps * groups, 0, st>>>(q);
  return cudaGetLastError();
}
template <typename T, int W>
cudaError_t launch_combine_backward_as(const Combine& q, cudaStream_t st) {
  // packs a thread: four or more; one where there are fewer tokens than CTAs the GPU holds
  const bool few = q.tokens < 2 * sm_count();
  if (q.dw == nullptr) {
    // only dy is in flight then: four packs a thread whatever k is, eight where k is 1 (12729 tokens of 2624 bf16 to 6 slots, 30 % of them
    // left out: 110 us with one pack, 58 with four)
    if (q.k == 1) return few ? combine_backward_as<T, W, 1, 1, false>(q, 1, st) : combine_backward_as<T, W, 1, 8, false>(q, 8, st);
    return few ? combine_backward_as<T, W, 8, 1, false>(q, 1, st) : combine_backward_as<T, W, 8, 4, false>(q, 4, st);
  }
  if (q.k == 1) return few ? combine_backward_as<T, W, 1, 1>(q, 1, st) : combine_backward_as<T, W, 1, 8>(q, 8, st);
  if (q.k == 2) return few ? combine_backward_as<T, W, 2, 1>(q, 1, st) : combine_backward_as<T, W, 2, 4>(q, 4, st);
  if (q.k <= 4) return few ? combine_backward_as<T, W, 4, 1>(q, 1, st) : combine_backward_as<T, W, 4, 2>(q, 4, st);
  return combine_backward_as<T, W, 8, 1>(q, few ? 1 : 4, st);
}

// How all matrices of a call can be accessed; p and ld of each (p null: none).
struct Rows { const void* p; long long ld; };
template <int K>
int access_of(const Rows (&m)[K], int d, int size) {
  bool by16 = (d * size) % 16 == 0, by2 = d % 2 == 0;
  for (const Rows& r : m) {
    by16 = by16 && rows_on(r.p, r.ld, size, 16);
    by2 = by2 && rows_on(r.p, r.ld, size, 2 * size);
  }
  return by16 ? BY_16 : by2 ? BY_TWO : BY_ONE;
}
template <typename T>
cudaError_t launch_combine(const Combine& q, int access, cudaStream_t st) {
  return access == BY_16 ? launch_combine_as<T, 16 / (int)sizeof(T)>(q, st) : access == BY_TWO ? launch_combine_as<T, 2>(q, st) : launch_combine_as<T, 1>(q, st);
}
template <typename T>
cudaError_t launch_combine_backward(const Combine& q, int access, cudaStream_t st) {
  return access == BY_16 ? launch_combine_backward_as<T, 16 / (int)sizeof(T)>(q, st)
       : access == BY_TWO ? launch_combine_backward_as<T, 2>(q, st)
                          : launch_combine_backward_as<T, 1>(q, st);
}

int combine(const void* ys, int32_t dtype, int64_t ys_ld, int64_t n_rows, const int32_t* rows, const float* w, int64_t tokens, int32_t k,
            int32_t d, const void* add, int64_t add_ld, void* y, int64_t y_ld, void* cuda_stream) {
  if (!sizes_ok(tokens, k, d, dtype) || n_rows < 0) return CAMERA_ERR_INVALID_ARG;
  if (!sizes_fit(tokens, k, d)) return CAMERA_ERR_UNSUPPORTED_SHAPE;
  const int size = dtype == CAMERA_BF16 ? 2 : 4;
  if (tokens == 0) return CAMERA_OK;
  if (!words_ok(rows) || (w != nullptr && !words_ok(w)) || !rows_fit(y, y_ld, d, size) || (n_rows > 0 && !rows_fit(ys, ys_ld, d, size)) ||
      (add != nullptr && !rows_fit(add, add_ld, d, size)))
    return CAMERA_ERR_INVALID_ARG;
  Combine q = {};
  q.ys = ys; q.add = add; q.y = y; q.ys_ld = ys_ld; q.add_ld = add_ld; q.y_ld = y_ld; q.n_rows = n_rows;
  q.rows = rows; q.w = w; q.tokens = (int)tokens; q.k = k; q.d = d;
  const int access = access_of({Rows{ys, ys_ld}, Rows{add, add_ld}, Rows{y, y_ld}}, d, size);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  MOE_CK(size == 2 ? launch_combine<__nv_bfloat16>(q, access, st) : launch_combine<float>(q, access, st));
  return CAMERA_OK;
}

}  // namespace
}  // namespace camera

extern "C" size_t camera_moe_dispatch_workspace_bytes(int64_t n_tokens, int32_t top_k, int32_t n_experts) {
  using namespace camera;
  if (n_tokens < 0 || top_k < 1 || n_experts < 1 || n_experts > MOE_MAX_EXPERTS || !sizes_fit(n_tokens, top_k, 1)) return 0;
  return 256 + moe_hist_bytes(n_tokens, top_k, n_experts);
}

extern "C" int camera_moe_dispatch(const void* x, int32_t dtype, int64_t ld, int64_t n_tokens, int32_t d_model,
                                   const int32_t* topk_idx, int32_t top_k, int32_t n_experts, void* x_sorted, int64_t sorted_ld,
                                   int32_t* rows, int32_t* offsets, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  using namespace camera;
  if (!sizes_ok(n_tokens, top_k, d_model, dtype) || n_experts < 1) return CAMERA_ERR_INVALID_ARG;
  if (!sizes_fit(n_tokens, top_k, d_model) || n_experts > MOE_MAX_EXPERTS) return CAMERA_ERR_UNSUPPORTED_SHAPE;
  if (!words_ok(offsets)) return CAMERA_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (n_tokens == 0) {
    MOE_CK(cudaMemsetAsync(offsets, 0, (size_t)4 * (n_experts + 1), st));
    return CAMERA_OK;
  }
  const int size = dtype == CAMERA_BF16 ? 2 : 4;
  if (!words_ok(topk_idx) || !words_ok(rows) || !rows_fit(x, ld, d_model, size) || !rows_fit(x_sorted, sorted_ld, d_model, size))
    return CAMERA_ERR_INVALID_ARG;
  const size_t hist = moe_hist_bytes(n_tokens, top_k, n_experts);
  if (hist > 0 && (workspace == nullptr || workspace_bytes < hist || (reinterpret_cast<uintptr_t>(workspace) & 255))) return CAMERA_ERR_WORKSPACE;
  Dispatch q = {};
  q.x = x; q.xs = x_sorted; q.x_ld = ld; q.xs_ld = sorted_ld;
  q.idx = topk_idx; q.rows = rows; q.offsets = offsets;
  q.tokens = (int)n_tokens; q.k = top_k; q.experts = n_experts; q.d = d_model;
  int ctas = moe_ctas(n_tokens);
  q.chunk = (int)((n_tokens + ctas - 1) / ctas);
  ctas = (int)((n_tokens + q.chunk - 1) / q.chunk);
  q.chunks = ctas;
  if (hist > 0) {
    q.totals = static_cast<int32_t*>(workspace);
    q.hist = q.totals + n_experts;
    MOE_CK(launch_chained(k_moe_count, q, ctas, 1, 1, MOE_THREADS, 4 * n_experts, false, st));
    MOE_CK(launch_chained(k_moe_scan, q, (n_experts + SCAN_WARPS - 1) / SCAN_WARPS, 1, 1, 32 * SCAN_WARPS, 0, true, st));
  }
  const int access = access_of({Rows{x, ld}, Rows{x_sorted, sorted_ld}}, d_model, size);
  MOE_CK(size == 2 ? launch_dispatch<__nv_bfloat16>(q, access, ctas, st) : launch_dispatch<float>(q, access, ctas, st));
  return CAMERA_OK;
}

extern "C" int camera_moe_combine(const void* y_sorted, int32_t dtype, int64_t sorted_ld, int64_t n_rows, const int32_t* rows,
                                  const float* topk_w, int64_t n_tokens, int32_t top_k, int32_t d_model, const void* add,
                                  int64_t add_ld, void* y, int64_t ld, void* cuda_stream) {
  return camera::combine(y_sorted, dtype, sorted_ld, n_rows, rows, topk_w, n_tokens, top_k, d_model, add, add_ld, y, ld, cuda_stream);
}

extern "C" int camera_moe_dispatch_backward(const void* dx_sorted, int32_t dtype, int64_t sorted_ld, int64_t n_rows, const int32_t* rows,
                                            int64_t n_tokens, int32_t top_k, int32_t d_model, const void* add, int64_t add_ld,
                                            void* dx, int64_t ld, void* cuda_stream) {
  return camera::combine(dx_sorted, dtype, sorted_ld, n_rows, rows, nullptr, n_tokens, top_k, d_model, add, add_ld, dx, ld, cuda_stream);
}

extern "C" int camera_moe_combine_backward(const void* dy, int32_t dtype, int64_t ld, int64_t n_tokens, int32_t d_model,
                                           const int32_t* rows, const float* topk_w, int32_t top_k, const void* y_sorted,
                                           int64_t sorted_ld, int64_t n_rows, void* dy_sorted, int64_t dy_sorted_ld,
                                           float* d_topk_w, void* cuda_stream) {
  using namespace camera;
  if (!sizes_ok(n_tokens, top_k, d_model, dtype) || n_rows < 0) return CAMERA_ERR_INVALID_ARG;
  if (!sizes_fit(n_tokens, top_k, d_model)) return CAMERA_ERR_UNSUPPORTED_SHAPE;
  if (n_tokens == 0) return CAMERA_OK;
  if (dy_sorted == nullptr && d_topk_w == nullptr && n_rows > 0) return CAMERA_ERR_INVALID_ARG;
  const int size = dtype == CAMERA_BF16 ? 2 : 4;
  if (!words_ok(rows) || (topk_w != nullptr && !words_ok(topk_w)) || (d_topk_w != nullptr && !words_ok(d_topk_w)) ||
      !rows_fit(dy, ld, d_model, size) || (dy_sorted != nullptr && n_rows > 0 && !rows_fit(dy_sorted, dy_sorted_ld, d_model, size)) ||
      (d_topk_w != nullptr && n_rows > 0 && !rows_fit(y_sorted, sorted_ld, d_model, size)))
    return CAMERA_ERR_INVALID_ARG;
  Combine q = {};
  q.ys = y_sorted; q.dy = dy; q.dys = dy_sorted; q.dw = d_topk_w;
  q.ys_ld = sorted_ld; q.dy_ld = ld; q.dys_ld = dy_sorted_ld; q.n_rows = n_rows;
  q.rows = rows; q.w = topk_w; q.tokens = (int)n_tokens; q.k = top_k; q.d = d_model;
  const int access = access_of({Rows{dy, ld}, Rows{dy_sorted, dy_sorted_ld}, Rows{d_topk_w != nullptr ? y_sorted : nullptr, sorted_ld}}, d_model, size);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  MOE_CK(size == 2 ? launch_combine_backward<__nv_bfloat16>(q, access, st) : launch_combine_backward<float>(q, access, st));
  return CAMERA_OK;
}
