// Orthogonalised updates: an odd polynomial applied to the singular values of a matrix, a few times over, by products alone
// (Newton-Schulz products).
//   X = U / (|U|_F + eps);   each step:  A = X X^T,  B = a I + b A + c A A,  X <- B X
// X is the matrix with its shorter side as rows (m), its longer as columns (n).  A and B are symmetric: only tiles on and
// above the diagonal are computed, each stored twice.  A step is m^2 n + m^3 + 2 m^2 n operations.  Bounds: where matrices are large,
// what is computed beyond that (rows are padded to 256, blocks on the diagonal computed whole: 999 GFLOP for the 766 that 16 matrices of
// 1408 .. 853 x 2048 need in five steps), and then bringing the operands of the products from L2 to the SMs, to which an epilogue adds
// its reads and writes (the same: 1000 us, 1.0 PFLOP/s of what is computed; a second tile of a unit some k blocks behind the first, so that
// no epilogue is waited for, changed nothing); where they are small, the chain of products, 6 us each, of which 3 to 4 are its way through
// global memory: first operand, stores, report and polling (5 matrices of 241 x 56: 99 us for fifteen).
//
// The operands of the products are fp16 with a power of two as factor, the sums fp32.  With h a bound of the singular values
// of X, no element of X is larger than h, none of A than h^2, none of B than the polynomial's largest value over [0, h^2]: the
// host follows these bounds from step to step (1 before the first) and picks the largest factors under which nothing can
// overflow.  fp16 has 3 bits more than bf16.  The diagonals of A and B hold most of what they are, and in a matrix whose singular
// values are alike all of it rounds the same way; so what their rounding leaves is kept in fp32 and enters the next product's
// epilogue (a row of it for B X, a row and a column for A A).
//
// X itself is held as two fp16 numbers, X + L: 22 bits, down to 2^-39 of the norm.  Its rounding reaches directions in which the matrix
// has nothing (a gradient made from few tokens), and there every step left multiplies it by a: 485 times in five steps, where what the
// matrix does have grows to 1.  There B is a I, so B L is a L, which an epilogue adds by element; no product needs L.  In the directions the
// matrix has, the rounding does not grow, and B L is nearer to the diagonal of B times L.  The factor lies between the two, nearer to a the
// more the steps left can make of it (f_low).  The rest of B L is left out.  1000 x 2048, fp32, made from 1, 8, 64, 256 and 2048 tokens: 1.7, 1.7,
// 1.9, 1.9 and 1.7e-3 off 64 bits (root mean square, relative), of which the result's rounding to bf16 alone makes 1.7e-3; with X in one fp16 it
// was 0.15, 4.2e-2, 2.1e-2, 7.7e-3 and 1.9e-3.  It costs a product's epilogue its reads and writes: sixteen matrices 940 -> 1000 us, three 225 ->
// 243.
// The first X is the matrix itself times a power of two, so bf16 inputs enter exactly; 1 / (|U| + eps) goes into the factors of the
// first step.
//
// Matrices of one call lie one below the other in the workspace, padded with zeros to whole tiles of 256 rows and whole
// 64 columns, so one tensor map serves them all and one launch walks the tiles of them all.
#include <cuda.h>
#include <cuda_fp16.h>
#include <math.h>
#include <string.h>

#include <atomic>

#include "common.cuh"
#include "launch.cuh"
#include "rowgroup.cuh"
#include "umma.cuh"
#include "umma_pair.cuh"

namespace camera {

namespace {

constexpr int O_EPI_WARPS = 8;               // epilogue: two warps per 32 rows, each with half of the columns
constexpr int O_PRODUCER = O_EPI_WARPS, O_ISSUER = O_EPI_WARPS + 1;
constexpr int O_THREADS = 32 * (O_EPI_WARPS + 2);
constexpr int O_TILE_M = 256;                // rows of the output a pair computes: 128 per CTA
constexpr int O_A_BYTES = 128 * 128;         // this CTA's 128 rows x 64 k
constexpr int O_MAX_STAGES = 8;
constexpr int O_RING_BYTES = 144 * 1024;
constexpr int O_CHUNK = 32;                   // columns an epilogue warp handles at a time,
constexpr int O_BUFS = 4;                    // and the chunks of 32 rows x 64 bytes it has in shared memory
constexpr int O_AHEAD = 2;                   // boxes on their way before they are needed
constexpr int O_BUF_BYTES = 32 * O_CHUNK * 2;
constexpr int O_EPI_BYTES = O_EPI_WARPS * O_BUFS * O_BUF_BYTES;
constexpr int O_REST_BYTES = O_EPI_WARPS * 256 * 4;      // POLY: the rests of the columns each epilogue warp works on
constexpr int O_SMEM_BYTES = O_RING_BYTES + O_EPI_BYTES + O_REST_BYTES + 512 + 1024;
constexpr int O_GROUP_M = 16;                // row tiles that are walked together
constexpr int O_TMEM_COLS = 512;
constexpr int O_MAX_MATS = 64;               // matrices of one round of launches
constexpr long long O_MAX_ELEMS = 1ll << 27; // and the elements of X that close a round
constexpr int O_MAX_SIDE = 1 << 17;
constexpr int O_MAX_STEPS = 64;

enum { ORTHO_GRAM = 0, ORTHO_POLY = 1, ORTHO_APPLY = 2 };

struct OrthoMat {
  const void* in;
  void* out;
  long long in_ld, out_ld;
  int m, n;                 // shorter and longer side
  int row0;                 // first row in the packed buffers
  int turned;               // in and out are [n, m]
};

struct OrthoBatch {
  int n_mats;
  OrthoMat mat[O_MAX_MATS];
};

// Factors of one step (see the top of the file): of the sums of GRAM, POLY and APPLY, of A and on the diagonal in POLY; and what the
// steps so far can have made of a small matrix (see scale_of), before and after this one.
struct OrthoStep {
  float f_gram, f_poly, f_aux, f_diag, f_apply, f_low;      // f_low: share of B's diagonal (over that of a) in the factor of X's low half
  int small_in, small_out;
};

// A packed buffer's tensor maps: as an operand in boxes of 64 columns x 128 or 64 rows, and in the epilogue's boxes.
struct OrthoMaps { CUtensorMap rows128, rows64, box; };
enum { BUF_X0 = 0, BUF_X1 = 1, BUF_A = 2, BUF_B = 3 };

struct OrthoRun {
  OrthoMaps maps[4];
  OrthoBatch batch;
  int unit0[3][O_MAX_MATS + 1];          // per product: first unit of each matrix
  int per_step, n_units, n_steps;        // units of one step; of all steps
  int bn, nb, kps, n_stages, n_acc;      // columns per B tile, B tiles per unit, k blocks per stage, ring depth, accumulators
  OrthoStep step[O_MAX_STEPS];
  __half* out[2];                        // A and B
  long long out_ld;
  float* rest[2];                        // [rows] what the rounding of the diagonals of A and B left
  float* low_f;                          // [rows] factor of a row of X's low half
  uint4* low;                            // the low half of X, in place through all steps (see low_at)
  int low_ld;                            // and the columns its rows have
  int low_first;                         // whether the first X has one
  const float* first;                    // factor of each matrix's first X
  const int* small;                      // exponents by which matrices are smaller than the bounds
  int* done;                             // [mats] warps that have finished with a unit of this matrix
  PlanTotals* totals;
  unsigned long long wait_limit_ns;
};

static_assert(sizeof(OrthoRun) <= 16384, "kernel arguments");

__host__ __device__ __forceinline__ int pad_rows(int m) { return (m + O_TILE_M - 1) / O_TILE_M * O_TILE_M; }
__host__ __device__ __forceinline__ int pad_cols(int n) { return (n + UMMA_BK - 1) / UMMA_BK * UMMA_BK; }

// A matrix whose norm is far below eps starts with singular values of 2^-small at most, where small = log2((|U| + eps) / |U|), and
// would be lost in fp16 at the others' factors.  A step makes them larger by no more than the largest value of its polynomial, so
// X keeps 2^(small - what the steps so far can have added) as a further factor, as long as that is above 1.
__device__ __forceinline__ int scale_of(int small, int used) { return max(0, small - used); }

// Where eight elements of X's low half lie, from column c on (a multiple of 8): rows in groups of 32, so that the lanes of an epilogue
// warp, each with its row, read and write 512 bytes in a row.
__host__ __device__ __forceinline__ long long low_at(int row, int c, int ld) { return ((long long)(row >> 5) * (ld >> 3) + (c >> 3)) * 32 + (row & 31); }

// need: how many warps must have finished with this matrix before the unit's operands are there.
struct OrthoUnit { int step, mode, e, m0, n0, two, kb, limit, need; };

// All steps' units in one row: step by step, in a step GRAM, POLY and APPLY, in each matrix by matrix.  A unit needs what the
// products before its own have made of its matrix, all of which lies before it in the row; so as long as CTAs take their units in
// order (and run at one time), somebody can always go on.
__device__ __forceinline__ OrthoUnit ortho_unit(const OrthoRun& q, int unit) {
  OrthoUnit r;
  const int mats = q.batch.n_mats;
  r.step = unit / q.per_step;
  int rem = unit - r.step * q.per_step;
  r.mode = ORTHO_GRAM;
  while (r.mode < ORTHO_APPLY && rem >= q.unit0[r.mode][mats]) rem -= q.unit0[r.mode++][mats];
  r.e = upper_segment(q.unit0[r.mode], mats, rem);
  rem -= q.unit0[r.mode][r.e];
  int before = 0, whole = 0;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int u = q.unit0[k][r.e + 1] - q.unit0[k][r.e];
    whole += u;
    before += k < r.mode ? u : 0;
  }
  r.need = (r.step * whole + before) * 2 * O_EPI_WARPS;
  const int m = q.batch.mat[r.e].m, n = q.batch.mat[r.e].n, w = q.nb * q.bn;
  const int rt = pad_rows(m) / O_TILE_M;
  if (r.mode == ORTHO_APPLY) {
    // row tiles in groups of O_GROUP_M, the row tile fastest: what runs at one time shares few column tiles and rows of B
    const int ct = (n + w - 1) / w, per_group = O_GROUP_M * ct, grp = rem / per_group;
    rem -= grp * per_group;
    const int in_group = min(O_GROUP_M, rt - grp * O_GROUP_M);
    r.m0 = (grp * O_GROUP_M + rem % in_group) * O_TILE_M;
    r.n0 = (rem / in_group) * w;
    r.limit = pad_cols(n);
    r.kb = pad_cols(m) / UMMA_BK;
  } else {
    int i = 0;
    for (;; ++i) {
      const int c = ((rt - i) * O_TILE_M + w - 1) / w;
      if (rem < c) break;
      rem -= c;
    }
    r.m0 = i * O_TILE_M;
    r.n0 = r.m0 + rem * w;
    r.limit = rt * O_TILE_M;
    r.kb = pad_cols(r.mode == ORTHO_GRAM ? n : m) / UMMA_BK;
  }
  r.two = q.nb == 2 && r.n0 + q.bn < r.limit;
  return r;
}

// Waits (one lane) until `need` warps have finished with a matrix, then lets the asynchronous proxy see what they wrote.
__device__ __forceinline__ bool wait_done(const int* done, int need, volatile int* abort_flag) {
  unsigned long long t0 = 0;
  for (unsigned spins = 0;; ++spins) {
    int v;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(done) : "memory");
    if (v >= need) break;
    if (spins == 0) t0 = globaltimer_ns();
    if ((spins & 15u) == 15u) {
      if (*abort_flag) return false;
      if (globaltimer_ns() - t0 > wait_limit_ns(abort_flag)) { *abort_flag = 1; return false; }
    }
    __nanosleep(64);
  }
  asm volatile("fence.proxy.async;" ::: "memory");
  return true;
}

// The same within a CTA: until its producer has seen the operands of its k-th unit.  A poller per CTA instead of nine lets the
// reports through sooner (7 matrices of 1487 x 245: 174 -> 165 us; polling more often than every 64 ns made it slower).
__device__ __forceinline__ bool wait_seen(uint32_t seen, int k, volatile int* abort_flag) {
  unsigned long long t0 = 0;
  for (unsigned spins = 0;; ++spins) {
    int v;
    asm volatile("ld.acquire.cta.shared.s32 %0, [%1];" : "=r"(v) : "r"(seen) : "memory");
    if (v > k) break;
    if (spins == 0) t0 = globaltimer_ns();
    if ((spins & 15u) == 15u) {
      if (*abort_flag) return false;
      if (globaltimer_ns() - t0 > wait_limit_ns(abort_flag)) { *abort_flag = 1; return false; }
    }
    __nanosleep(32);
  }
  asm volatile("fence.proxy.async;" ::: "memory");
  return true;
}

// What other CTAs have written during this launch: read from L2, and not before the waits that stand above in the program.
__device__ __forceinline__ float load_written(const float* p) {
  float v;
  asm volatile("ld.global.cg.f32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ float4 load_written(const float4* p) {
  float4 v;
  asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint4 load_written(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.cg.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// What the rounding of a and b to the halves in p leaves.
__device__ __forceinline__ uint32_t pack_low(float a, float b, uint32_t p) {
  const float2 high = __half22float2(*reinterpret_cast<const __half2*>(&p));
  return pack_half(a - high.x, b - high.y);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// The transpose of 16 columns of a warp's 32 rows: p[j] holds columns 2j and 2j + 1 of this lane's row.  Two lanes exchange
// halves, so that each stores two neighbouring rows of a column in one word.  at: where column 0 of this warp's first row
// goes; columns are ld elements apart, rows follow one another.
__device__ __forceinline__ void store_turned(uint16_t* at, long long ld, const uint32_t* p, int lane, int rows, int cols, bool words) {
  if (words && rows >= 32) {
    const bool odd = lane & 1;
    uint32_t* const dst = reinterpret_cast<uint32_t*>(at + (odd ? ld : 0) + (lane & ~1));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t other = __shfl_xor_sync(0xffffffffu, p[j], 1);
      const uint32_t v = odd ? __byte_perm(other, p[j], 0x7632) : __byte_perm(p[j], other, 0x5410);
      if (2 * j + odd < cols) *reinterpret_cast<uint32_t*>(reinterpret_cast<uint16_t*>(dst) + 2 * j * ld) = v;
    }
  } else if (lane < rows) {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (j < cols) at[j * ld + lane] = (uint16_t)(j & 1 ? p[j >> 1] >> 16 : p[j >> 1] & 0xffffu);
  }
}

// A box of 32 x 32 elements in shared memory (64-byte swizzle) to rows of `to` that are ld elements apart, V's size at a time, so that
// the lanes store whole runs of a row.
template <typename V>
__device__ __forceinline__ void box_out(uint16_t* to, long long ld, uint32_t box, int lane, int rows, int cols) {
  constexpr int E = sizeof(V) / 2, LANES = O_CHUNK / E;          // elements a lane stores, lanes a row
  const int c = lane % LANES * E;
  if (c >= cols) return;
#pragma unroll
  for (int r = lane / LANES; r < 32; r += 32 / LANES) {
    if (r >= rows) break;
    const uint32_t at = box + r * (2 * O_CHUNK) + (((c >> 3) ^ (r >> 1 & 3)) << 4) + 2 * (c & 7);
    V v;
    if constexpr (E == 8) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    else if constexpr (E == 2) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at));
    else asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(at));
    *reinterpret_cast<V*>(to + r * ld + c) = v;
  }
}

template <int M> struct Mode { static constexpr int value = M; };

// All products of all steps in one launch: CTAs stay, and a unit starts when the units it depends on have been reported finished (a
// counter per matrix).  With a launch per product (15 of them) 7 matrices of 53 x 62 took 96 us and 94 us of the host's time.
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(O_THREADS, 1) k_ortho(const __grid_constant__ OrthoRun q) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bars = base + O_RING_BYTES + O_EPI_BYTES + O_REST_BYTES;
  auto full_bar = [&](int s) { return bars + 8u * s; };                                 // first CTA
  auto empty_bar = [&](int s) { return bars + 8u * (O_MAX_STAGES + s); };               // each CTA
  auto tfull_bar = [&](int a) { return bars + 8u * (2 * O_MAX_STAGES + a); };           // each CTA
  auto tempty_bar = [&](int a) { return bars + 8u * (2 * O_MAX_STAGES + 2 + a); };      // first CTA, the pair's epilogue threads
  auto aux_bar = [&](int i) { return bars + 8u * (2 * O_MAX_STAGES + 4 + i); };         // per epilogue warp and buffer
  uint8_t* const tail = base_ptr + O_RING_BYTES + O_EPI_BYTES + O_REST_BYTES + 8 * (2 * O_MAX_STAGES + 4 + O_EPI_WARPS * O_BUFS);
  volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(tail);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tail + 8);

  volatile int* const seen = reinterpret_cast<volatile int*>(tail + 32);                    // units whose operands are there

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t rank = cluster_ctarank();
  const int n_pairs = gridDim.x >> 1, pair = blockIdx.x >> 1;
  const int half = q.bn >> 1;                               // columns of a B tile this CTA supplies
  const int b_bytes = half * 128;
  const int block_bytes = O_A_BYTES + q.nb * b_bytes;       // operands of one k block
  const int stage_bytes = q.kps * block_bytes;

  if (tid == 0) {
    for (int s = 0; s < q.n_stages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 2 * 32 * O_EPI_WARPS); }
    for (int i = 0; i < O_EPI_WARPS * O_BUFS; ++i) mbar_init(aux_bar(i), 1);
    wait_state_init(abort_flag, q.wait_limit_ns);
    *seen = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == O_ISSUER) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)),
                 "r"(O_TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();     // the other CTA's barriers are initialised before anything arrives on them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;

  if (warp == O_PRODUCER) {
    // ------------------------------------------------------------------ TMA producer (each CTA loads its own share)
    const uint32_t lead = lane == 0;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int unit = pair, k = 0; ok && unit < q.n_units; unit += n_pairs) {
      const OrthoUnit u = ortho_unit(q, unit);
      const int row0 = q.batch.mat[u.e].row0;
      const int am = row0 + u.m0 + 128 * (int)rank, bn0 = u.n0 + half * (int)rank;
      const bool B_MN = u.mode == ORTHO_APPLY;
      const OrthoMaps& from = q.maps[u.mode == ORTHO_GRAM ? u.step & 1 : u.mode == ORTHO_POLY ? BUF_A : BUF_B];
      const CUtensorMap* const map_a = &from.rows128;
      const CUtensorMap* const map_b = B_MN ? &q.maps[u.step & 1].rows64 : half > 64 ? &from.rows128 : &from.rows64;
      ok = __all_sync(0xffffffffu, lane != 0 || wait_done(q.done + u.e, u.need, abort_flag));
      if (ok && lane == 0) asm volatile("st.release.cta.shared.s32 [%0], %1;" ::"r"(smem_u32((const void*)seen)), "r"(++k) : "memory");
      for (int kb = 0, blocks; ok && kb < u.kb; kb += blocks) {
        blocks = min(q.kps, u.kb - kb);
        ok = warp_wait(empty_bar(stage), phase ^ 1u, abort_flag);
        if (!ok) break;
        const uint32_t full0 = map_to_cta(full_bar(stage), 0);
        if (rank == 0 && lane == 0) mbar_expect_tx(full_bar(stage), 2 * blocks * (O_A_BYTES + (u.two ? 2 : 1) * b_bytes));
        __syncwarp();
        uint32_t dst = base + stage * stage_bytes;
        for (int k0 = kb * UMMA_BK; k0 < (kb + blocks) * UMMA_BK; k0 += UMMA_BK, dst += block_bytes) {
          tma_load_lead(lead, dst, map_a, full0, k0, am);
          const uint32_t dst_b = dst + O_A_BYTES;
          if (B_MN) {
            tma_load_lead(lead, dst_b, map_b, full0, bn0, row0 + k0);
            if (half > 64) tma_load_lead(lead, dst_b + 8192, map_b, full0, bn0 + 64, row0 + k0);
            if (u.two) {
              tma_load_lead(lead, dst_b + b_bytes, map_b, full0, bn0 + q.bn, row0 + k0);
              if (half > 64) tma_load_lead(lead, dst_b + b_bytes + 8192, map_b, full0, bn0 + q.bn + 64, row0 + k0);
            }
          } else {
            tma_load_lead(lead, dst_b, map_b, full0, k0, row0 + bn0);
            if (u.two) tma_load_lead(lead, dst_b + b_bytes, map_b, full0, k0, row0 + bn0 + q.bn);
          }
        }
        if (++stage == q.n_stages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok) {               // copies in flight land before the CTA's shared memory is given up
      const unsigned long long t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
  } else if (warp == O_ISSUER) {
    // ------------------------------------------------------------------ MMA issuer (first CTA of the pair only)
    if (rank == 0) {
      const uint32_t lead = lane == 0;
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true, ready = false;       // ready: the next stage has been seen full
      constexpr int A_STEP = 32 >> 4;                                          // 16 k further
      const unsigned long long a_first = make_smem_desc(base);
      const unsigned long long b2_off = (unsigned long long)(b_bytes >> 4);
      for (int unit = pair; ok && unit < q.n_units; unit += n_pairs) {
        const OrthoUnit u = ortho_unit(q, unit);
        const bool B_MN = u.mode == ORTHO_APPLY;
        const uint32_t idesc = make_idesc_pair_f16(q.bn) | (B_MN ? 1u << 16 : 0u);
        const unsigned long long b_first = B_MN ? make_smem_desc_mn(base + O_A_BYTES) : make_smem_desc(base + O_A_BYTES);
        ok = __all_sync(0xffffffffu, mbar_wait_cluster(tempty_bar(acc), acc_phase ^ 1u, abort_flag));
        if (!ok) break;
        tc_fence_after();
        const uint32_t d0 = tmem_base + (uint32_t)(acc * q.nb * q.bn), d1 = d0 + (uint32_t)q.bn;
        uint32_t accumulate = 0;
        for (int kb = 0, blocks; kb < u.kb; kb += blocks) {
          blocks = min(q.kps, u.kb - kb);
          if (!ready) {
            ok = warp_wait(full_bar(stage), phase, abort_flag);
            if (!ok) break;
          }
          tc_fence_after();
          unsigned long long at = (unsigned long long)((uint32_t)(stage * stage_bytes) >> 4);
          const uint32_t done = empty_bar(stage);
          if (++stage == q.n_stages) { stage = 0; phase ^= 1u; }
          for (int block = blocks; block > 0; --block, at += (unsigned long long)(block_bytes >> 4)) {
            const unsigned long long a_desc = a_first + at, b_desc = b_first + at;
            if (u.two) {
              const unsigned long long b2_desc = b_desc + b2_off;
              const int b_step = B_MN ? 2048 >> 4 : 32 >> 4;
#pragma unroll
              for (int k = 0; k < UMMA_BK / 16; ++k) {
                umma_lead(lead, d0, a_desc + A_STEP * k, b_desc + b_step * k, idesc, accumulate | (uint32_t)k);
                umma_lead(lead, d1, a_desc + A_STEP * k, b2_desc + b_step * k, idesc, accumulate | (uint32_t)k);
              }
            } else if (B_MN) {
              umma_block<A_STEP, (2048 >> 4)>(lead, d0, a_desc, b_desc, idesc, accumulate);
            } else {
              umma_block<A_STEP, (32 >> 4)>(lead, d0, a_desc, b_desc, idesc, accumulate);
            }
            accumulate = 1;
          }
          ready = __all_sync(0xffffffffu, mbar_test(full_bar(stage), phase));
          umma_commit_lead(lead, done);
        }
        if (!ok) break;
        umma_commit_lead(lead, tfull_bar(acc));
        if (++acc == q.n_acc) { acc = 0; acc_phase ^= 1u; }
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue: a thread owns a row of the output
    // What it reads beside the accumulators (this tile of A or X) and what it writes travel as boxes of 32 rows x 32 columns
    // through the warp's buffers in shared memory, by TMA both ways: a lane's loads and stores of 32 bytes of its own row
    // each take a request per lane (16 matrices of up to 1408 x 2048: POLY 62 us, APPLY 122 us; without their reads 46 and
    // 91 us).  The result takes the place of what was read; two boxes are in flight ahead.
    int acc = 0;
    uint32_t acc_phase = 0, n = 0, loads = 0;                // boxes so far, in buffer n % O_BUFS; those of them that were loaded
    bool ok = true;
    const int c_half = q.nb * q.bn / 2, c_first = c_half * (warp >> 2);
    uint8_t* const bufs = base_ptr + O_RING_BYTES + warp * O_BUFS * O_BUF_BYTES;
    [[maybe_unused]] float* const rests = reinterpret_cast<float*>(base_ptr + O_RING_BYTES + O_EPI_BYTES) + 256 * warp;
    const uint32_t buf0 = smem_u32(bufs), swz = (uint32_t)(lane >> 1) & 3u;       // 64-byte swizzle: 16-byte piece i of a row at i ^ swz
    auto unit_done = [&](auto mode, const OrthoUnit& u, int k) {    // the k-th of this CTA; false: a wait ran out
      constexpr int MODE = decltype(mode)::value;
      const OrthoStep& st = q.step[u.step];
      const bool to_caller = MODE == ORTHO_APPLY && u.step + 1 == q.n_steps;
      const OrthoMat& mat = q.batch.mat[u.e];
      const int warp_row = u.m0 + 128 * (int)rank + (warp & 3) * 32, row = warp_row + lane;      // in the matrix, < pad_rows(m)
      const int cols = min(u.limit - u.n0, c_first + c_half);       // where this warp's columns end, a multiple of O_CHUNK
      const CUtensorMap* const aux_map = &q.maps[MODE == ORTHO_POLY ? BUF_A : u.step & 1].box;
      const CUtensorMap* const out_map = &q.maps[MODE == ORTHO_GRAM ? BUF_A : MODE == ORTHO_POLY ? BUF_B : (u.step + 1) & 1].box;
      __half* const out_rows = q.out[MODE == ORTHO_POLY];
      // read while the products run: an argument's first use takes a while (POLY's epilogue of one tile: 3.5 and 2.9 us)
      float f_aux = MODE == ORTHO_POLY ? st.f_aux : 0.f, f_diag = MODE == ORTHO_POLY ? st.f_diag : 0.f;
      const float* rest_in = q.rest[MODE == ORTHO_APPLY] + mat.row0;
      float* rest_out = q.rest[MODE == ORTHO_POLY] + mat.row0;
      asm volatile("" : "+f"(f_aux), "+f"(f_diag), "+l"(rest_in), "+l"(rest_out));
      uint16_t* const out = static_cast<uint16_t*>(mat.out);
      float f = MODE == ORTHO_GRAM ? st.f_gram : MODE == ORTHO_POLY ? st.f_poly : st.f_apply;
      if (MODE != ORTHO_POLY) {
        const int small = q.small[u.e];
        const float s = u.step == 0 ? q.first[u.e] : scalbnf(1.f, scale_of(small, st.small_in));
        f = MODE == ORTHO_GRAM ? f / s / s : scalbnf(f / s, to_caller ? 0 : scale_of(small, st.small_out));
      }
      if (MODE != ORTHO_GRAM && !__all_sync(0xffffffffu, lane != 0 || wait_seen(smem_u32((const void*)seen), k, abort_flag))) return false;
      __syncwarp();                                                // a vote orders no memory: what lane 0 acquired is there for all lanes
      const float rest = MODE == ORTHO_GRAM ? 0.f : load_written(rest_in + row);
      const float low_f = MODE == ORTHO_APPLY ? load_written(q.low_f + mat.row0 + row) : 0.f;
      const bool has_low = MODE == ORTHO_APPLY && (u.step > 0 || q.low_first);
      uint4* const low_row = q.low + low_at(mat.row0 + row, u.n0, q.low_ld);
      uint4 low[4], low_next[4];                                   // this lane's of the chunk at work and of the next
      auto fetch_low = [&](int c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) low_next[i] = has_low && c < cols ? load_written(low_row + 4 * c + 32 * i) : make_uint4(0, 0, 0, 0);
      };
      if (MODE == ORTHO_APPLY) fetch_low(c_first);
      auto fetch = [&](int c, uint32_t k) {                        // lane 0: the k-th box from here, at column c, on its way
        if (MODE != ORTHO_GRAM && c < cols) {
          const uint32_t bar = aux_bar(warp * O_BUFS + (loads + k) % O_BUFS);
          mbar_expect_tx(bar, O_BUF_BYTES);
          tma_load_2d(buf0 + (n + k) % O_BUFS * O_BUF_BYTES, aux_map, bar, u.n0 + c, mat.row0 + warp_row);
        }
      };
      if (lane == 0) {
#pragma unroll
        for (int k = 0; k < O_AHEAD; ++k) fetch(c_first + O_CHUNK * k, k);
      }
      if (MODE == ORTHO_POLY) {
        __syncwarp();
        for (int i = 4 * lane; c_first + i < cols; i += 128)
          *reinterpret_cast<float4*>(rests + i) = load_written(reinterpret_cast<const float4*>(rest_in + u.n0 + c_first + i));
      }
      __syncwarp();
      if (!__all_sync(0xffffffffu, mbar_wait(tfull_bar(acc), acc_phase, abort_flag))) return false;
      tc_fence_after();
      const uint32_t t0 = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(acc * q.nb * q.bn);
      uint8_t* box_row = bufs;                                      // this lane's row of the box at work
      auto put = [&](const uint32_t* raw, int k, int c) {
        uint32_t p[8];
        float v[16];
        uint4* const piece0 = reinterpret_cast<uint4*>(box_row + (((2 * k) ^ swz) << 4));
        uint4* const piece1 = reinterpret_cast<uint4*>(box_row + (((2 * k + 1) ^ swz) << 4));
        const F2 f_2 = f2(f, f);
        if (MODE == ORTHO_GRAM) {
#pragma unroll
          for (int j = 0; j < 16; j += 2) split(mul2(f2(__uint_as_float(raw[j]), __uint_as_float(raw[j + 1])), f_2), v[j], v[j + 1]);
        } else {
          uint32_t a[8];
          *reinterpret_cast<uint4*>(a) = *piece0;
          *reinterpret_cast<uint4*>(a + 4) = *piece1;
#pragma unroll
          for (int j = 0; j < 16; j += 2) {
            const float2 old = __half22float2(*reinterpret_cast<const __half2*>(&a[j >> 1]));
            const F2 old2 = f2(old.x, old.y), sum = f2(__uint_as_float(raw[j]), __uint_as_float(raw[j + 1]));
            if (MODE == ORTHO_APPLY) {                  // (B + rest) X, and of its low half what matters of B
              const uint4& piece = low[2 * k + (j >> 3)];
              const uint32_t word = (j >> 1 & 3) == 0 ? piece.x : (j >> 1 & 3) == 1 ? piece.y : (j >> 1 & 3) == 2 ? piece.z : piece.w;
              const float2 lo = __half22float2(*reinterpret_cast<const __half2*>(&word));
              split(mul2(fma2(f2(low_f, low_f), f2(lo.x, lo.y), fma2(f2(rest, rest), old2, sum)), f_2), v[j], v[j + 1]);
            } else {                                    // (A + rest)^2 up to the square of the rest, and b A (b rest: below)
              const float2 down = *reinterpret_cast<const float2*>(rests + c - c_first + j);
              split(fma2(old2, f2(f_aux, f_aux), mul2(fma2(add2(f2(rest, rest), f2(down.x, down.y)), old2, sum), f_2)), v[j], v[j + 1]);
            }
          }
        }
        if (to_caller) {
          // the result, in the caller's layout
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] = pack_bf16(v[2 * j], v[2 * j + 1]);
          if (mat.turned) {
            store_turned(out + (long long)(u.n0 + c) * mat.out_ld + warp_row, mat.out_ld, p, lane, mat.m - warp_row, mat.n - u.n0 - c,
                         ((reinterpret_cast<uintptr_t>(out) & 3) | (mat.out_ld & 1)) == 0);
          } else {
            *piece0 = make_uint4(p[0], p[1], p[2], p[3]);
            *piece1 = make_uint4(p[4], p[5], p[6], p[7]);
          }
          return;
        }
        if (MODE != ORTHO_APPLY && u.n0 + c < warp_row + 32 && u.n0 + c + 16 > warp_row) {
          // on the diagonal: what its rounding leaves is kept (by selections: 16 branches that one lane each takes cost 0.7 us)
          const int own = row - u.n0 - c;
          float mine = 0.f;
#pragma unroll
          for (int j = 0; j < 16; ++j) mine = j == own ? v[j] : mine;
          if (MODE == ORTHO_POLY) mine += fmaf(rest, f_aux, f_diag);
#pragma unroll
          for (int j = 0; j < 16; ++j) v[j] = j == own ? mine : v[j];
          if (own >= 0 && own < 16) {
            rest_out[row] = mine - __half2float(__float2half_rn(mine));
            // (one row: B is its diagonal)
            if (MODE == ORTHO_POLY) q.low_f[mat.row0 + row] = mat.m == 1 ? mine : fmaf(st.f_low, mine - f_diag, f_diag);
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = pack_half(v[2 * j], v[2 * j + 1]);
        if (MODE == ORTHO_APPLY) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            low_row[4 * c + 32 * i] = make_uint4(pack_low(v[8 * i], v[8 * i + 1], p[4 * i]), pack_low(v[8 * i + 2], v[8 * i + 3], p[4 * i + 1]),
                                                 pack_low(v[8 * i + 4], v[8 * i + 5], p[4 * i + 2]), pack_low(v[8 * i + 6], v[8 * i + 7], p[4 * i + 3]));
        }
        *piece0 = make_uint4(p[0], p[1], p[2], p[3]);
        *piece1 = make_uint4(p[4], p[5], p[6], p[7]);
        if (MODE != ORTHO_APPLY && u.n0 + c >= u.m0 + O_TILE_M)      // off the diagonal's block: the other half of the result
          store_turned(reinterpret_cast<uint16_t*>(out_rows) + (long long)(mat.row0 + u.n0 + c) * q.out_ld + warp_row, q.out_ld, p, lane, 32, 16,
                       true);
      };
      uint32_t v0[16], v1[16];
      if (c_first < cols) tmem_ld16(t0 + c_first, v0);
      for (int c = c_first; c < cols; c += O_CHUNK, ++n, loads += MODE != ORTHO_GRAM) {
        const uint32_t box = n % O_BUFS;
        box_row = bufs + box * O_BUF_BYTES + lane * (2 * O_CHUNK);
        if (MODE == ORTHO_APPLY) {
#pragma unroll
          for (int i = 0; i < 4; ++i) low[i] = low_next[i];
          fetch_low(c + O_CHUNK);
        }
        if (MODE != ORTHO_GRAM) {
          if (!warp_wait(aux_bar(warp * O_BUFS + loads % O_BUFS), loads / O_BUFS & 1u, abort_flag)) return false;
        }
        tmem_ld_wait(v0);
        tmem_ld16(t0 + c + 16, v1);
        put(v0, 0, c);
        tmem_ld_wait(v1);
        if (c + O_CHUNK < cols) tmem_ld16(t0 + c + O_CHUNK, v0);
        put(v1, 1, c + 16);
        // before a box leaves by TMA, and before one (the result's too) takes the room of what lanes wrote or read
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (to_caller && !mat.turned) {
          // the box's rows as they lie in memory: by 16 bytes, by two elements or by one
          uint16_t* const to = out + warp_row * mat.out_ld + u.n0 + c;
          const uint32_t from = buf0 + box * O_BUF_BYTES;
          const int rows = mat.m - warp_row, left = mat.n - u.n0 - c;
          const unsigned on = (unsigned)reinterpret_cast<uintptr_t>(out) | 2u * (unsigned)mat.out_ld | 2u * (unsigned)mat.n;
          if ((on & 15u) == 0) box_out<uint4>(to, mat.out_ld, from, lane, rows, left);
          else if ((on & 3u) == 0) box_out<uint32_t>(to, mat.out_ld, from, lane, rows, left);
          else box_out<uint16_t>(to, mat.out_ld, from, lane, rows, left);
        }
        if (lane == 0) {
          if (!to_caller) {
            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(out_map),
                         "r"(buf0 + box * O_BUF_BYTES), "r"(u.n0 + c), "r"(mat.row0 + warp_row)
                         : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            // the next box to fetch, or (GRAM) to write, takes the room of one whose store has read it by now
            asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(MODE == ORTHO_GRAM ? O_BUFS - 1 : O_BUFS - O_AHEAD) : "memory");
          }
          fetch(c + O_AHEAD * O_CHUNK, O_AHEAD);
        }
        __syncwarp();
      }
      tc_fence_before();
      mbar_arrive_cluster(map_to_cta(tempty_bar(acc), 0));
      if (++acc == q.n_acc) { acc = 0; acc_phase ^= 1u; }
      // While the next unit's products run: what this warp wrote (boxes, mirrored words, rests) is there for everybody.
      if (!to_caller) {
        __syncwarp();
        if (lane == 0) {
          asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
          asm volatile("fence.proxy.async;" ::: "memory");
          asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(q.done + u.e) : "memory");
        }
      }
      return true;
    };
    for (int unit = pair, k = 0; ok && unit < q.n_units; unit += n_pairs, ++k) {
      const OrthoUnit u = ortho_unit(q, unit);
      ok = u.mode == ORTHO_GRAM   ? unit_done(Mode<ORTHO_GRAM>(), u, k)
           : u.mode == ORTHO_POLY ? unit_done(Mode<ORTHO_POLY>(), u, k)
                                  : unit_done(Mode<ORTHO_APPLY>(), u, k);
    }
    if (!ok) {               // boxes on their way land before the CTA's shared memory is given up
      const unsigned long long t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag && tid == 0) atomicExch(&q.totals->status, (int)CAMERA_ERR_DEVICE_TIMEOUT);
  cluster_sync_all();     // neither CTA leaves while the other may still read its shared or tensor memory
  if (warp == O_ISSUER) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(O_TMEM_COLS) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------ the first X
struct OrthoLoad {
  OrthoBatch batch;
  double* part;             // [mats][parts] sums of squares
  int parts;
  float* first;             // [mats] factor between X as stored and X
  int* small;               // [mats]
  int* done;                // [mats], cleared here
  float eps;
  __half* x;
  long long x_ld;
  uint4* low;               // fp32: the low half of X
  PlanTotals* totals;
  int clear_status;
};
constexpr int LOAD_THREADS = 256;

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double sums[LOAD_THREADS / 32];
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < LOAD_THREADS / 32; ++i) v += sums[i];
  return v;
}

// Whether the matrix's rows all start on 16-byte boundaries.
template <typename T>
__device__ __forceinline__ bool rows_aligned(const OrthoMat& mat) {
  return ((reinterpret_cast<uintptr_t>(mat.in) | (uintptr_t)(mat.in_ld * (long long)sizeof(T))) & 15) == 0;
}
// Eight squares, in fp32 (added up in double) or in double where fp32 might overflow or lose them.
__device__ __forceinline__ double squares(const float (&v)[8]) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) s = fmaf(v[i], v[i], s);
  if (s > 1e-20f && s < 1e30f) return (double)s;
  double d = 0.0;
#pragma unroll
  for (int i = 0; i < 8; ++i) d = fma((double)v[i], (double)v[i], d);
  return d;
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {          // 16-byte aligned
  constexpr int N = Vec16<T>::N;
#pragma unroll
  for (int i = 0; i < 8; i += N) Vec16<T>::load(p + i, v + i);
}

// Sums of squares of the rows each warp takes.
template <typename T>
__global__ void __launch_bounds__(LOAD_THREADS, 6) k_ortho_norm(const __grid_constant__ OrthoLoad q) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (q.clear_status && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) q.totals->status = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) q.done[blockIdx.y] = 0;
  const OrthoMat& mat = q.batch.mat[blockIdx.y];
  const int rows = mat.turned ? mat.n : mat.m, cols = mat.turned ? mat.m : mat.n, lane = threadIdx.x & 31;
  const T* const in = static_cast<const T*>(mat.in);
  const bool vec = rows_aligned<T>(mat);
  double sum = 0.0;
  for (int r = blockIdx.x * (LOAD_THREADS / 32) + (threadIdx.x >> 5); r < rows; r += gridDim.x * (LOAD_THREADS / 32)) {
    const T* const p = in + r * mat.in_ld;
    int done = 0;
    if (vec) {
      done = cols & ~7;
      for (int c = 8 * lane; c < done; c += 1024) {
        float v[4][8];
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (c + 256 * k < done) {
            load8(p + c + 256 * k, v[k]);
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[k][i] = 0.f;
          }
#pragma unroll
        for (int k = 0; k < 4; ++k) sum += squares(v[k]);
      }
    }
    for (int c = done + lane; c < cols; c += 256) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c + 32 * i < cols ? to_f32(p[c + 32 * i]) : 0.f;
      sum += squares(v);
    }
  }
  const double s = block_sum(sum);
  if (threadIdx.x == 0) q.part[blockIdx.y * q.parts + blockIdx.x] = s;
}

// X = U 2^p in fp16 (of fp32 matrices a second fp16 holds what the rounding leaves), shorter side as rows, zeros around it.  p puts
// 2^p |U| into [2^14, 2^15): nothing overflows, and what is below 2^-39 of the norm is lost.  A CTA turns tiles of 64 x 64 in shared
// memory.
template <typename T>
__global__ void __launch_bounds__(LOAD_THREADS, 6) k_ortho_load(const __grid_constant__ OrthoLoad q) {
  constexpr bool LOW = sizeof(T) == 4;
  __shared__ __align__(16) __half tile[LOW ? 2 : 1][64][72];
  __shared__ int power;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const OrthoMat& mat = q.batch.mat[blockIdx.y];
  double s = 0.0;
  for (int i = threadIdx.x; i < q.parts; i += LOAD_THREADS) s += q.part[blockIdx.y * q.parts + i];
  s = block_sum(s);
  if (threadIdx.x == 0) {
    const double norm = sqrt(s);
    int p = 0;
    if (norm > 0.0 && norm < 1e300) {
      int e;
      frexp(norm, &e);                    // norm in [2^(e-1), 2^e)
      p = 15 - e;
    }
    power = p;
    if (blockIdx.x == 0) {
      const double all = norm + (double)q.eps;
      q.first[blockIdx.y] = norm == 0.0 ? 1.f : norm < 1e300 ? (float)fmin(ldexp(all, p), 1e38) : __int_as_float(0x7fffffff);
      int e = 1;
      if (norm > 0.0 && norm < 1e300) frexp(all / norm, &e);       // all / norm in [2^(e-1), 2^e)
      q.small[blockIdx.y] = min(e - 1, 100);
    }
  }
  __syncthreads();
  const int p = power;
  const float up = scalbnf(1.f, p / 2), up2 = scalbnf(1.f, p - p / 2);
  const int rt = pad_rows(mat.m) / 64, ct = pad_cols(mat.n) / 64;
  const T* const in = static_cast<const T*>(mat.in);
  const bool vec = rows_aligned<T>(mat);
  for (int t = blockIdx.x; t < rt * ct; t += gridDim.x) {
    const int r0 = t / ct * 64, c0 = t % ct * 64;
    const int a0 = mat.turned ? c0 : r0, b0 = mat.turned ? r0 : c0;         // in the caller's rows and columns
    const int a_end = mat.turned ? mat.n : mat.m, b_end = mat.turned ? mat.m : mat.n;
    // two runs of 8 elements a thread
    float v[2][8];
    const int b = (threadIdx.x & 7) * 8;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int a = (threadIdx.x >> 3) + 32 * k;
      const T* const from = in + (a0 + a) * mat.in_ld + b0 + b;
      if (vec && a0 + a < a_end && b0 + b + 8 <= b_end) {
        load8(from, v[k]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] = a0 + a < a_end && b0 + b + i < b_end ? to_f32(from[i]) : 0.f;
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int a = (threadIdx.x >> 3) + 32 * k;
      uint32_t w[LOW ? 2 : 1][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float a0 = v[k][2 * i] * up * up2, a1 = v[k][2 * i + 1] * up * up2;
        w[0][i] = pack_half(a0, a1);
        if constexpr (LOW) w[1][i] = pack_low(a0, a1, w[0][i]);
      }
#pragma unroll
      for (int h = 0; h < (LOW ? 2 : 1); ++h)
        if (mat.turned) {
#pragma unroll
          for (int i = 0; i < 8; ++i) tile[h][b + i][a] = __ushort_as_half((unsigned short)(i & 1 ? w[h][i >> 1] >> 16 : w[h][i >> 1] & 0xffffu));
        } else {
          *reinterpret_cast<uint4*>(&tile[h][a][b]) = make_uint4(w[h][0], w[h][1], w[h][2], w[h][3]);
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = (threadIdx.x >> 3) + 32 * k;
      *reinterpret_cast<uint4*>(q.x + (long long)(mat.row0 + r0 + r) * q.x_ld + c0 + b) = *reinterpret_cast<const uint4*>(&tile[0][r][b]);
      if constexpr (LOW) q.low[low_at(mat.row0 + r0 + r, c0 + b, (int)q.x_ld)] = *reinterpret_cast<const uint4*>(&tile[1][r][b]);
    }
  }
}

// ------------------------------------------------------------------------------------------------ host side
size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

// One round of launches: matrices [begin, end) of the call, those without elements left out.
struct OrthoRound {
  int begin, end;
  long long rows;           // of the packed buffers
  int x_ld, a_ld;
};
OrthoRound ortho_round(const camera_matrix_t* mats, int n, int begin) {
  OrthoRound r = {begin, begin, 0, 0, 0};
  int count = 0;
  for (; r.end < n && count < O_MAX_MATS; ++r.end) {
    const camera_matrix_t& t = mats[r.end];
    if (t.rows == 0 || t.cols == 0) continue;
    const int m = t.rows < t.cols ? t.rows : t.cols, w = t.rows < t.cols ? t.cols : t.rows;
    const long long rows = r.rows + pad_rows(m);
    const int x_ld = pad_cols(w) > r.x_ld ? pad_cols(w) : r.x_ld, a_ld = pad_rows(m) > r.a_ld ? pad_rows(m) : r.a_ld;
    if (count > 0 && rows * x_ld > O_MAX_ELEMS) break;
    r.rows = rows; r.x_ld = x_ld; r.a_ld = a_ld;
    ++count;
  }
  return r;
}
constexpr int MAX_PARTS = 296;
struct OrthoLayout { size_t part, first, rest_a, rest_b, low_f, x0, x1, low, a, b, total; };
OrthoLayout ortho_layout(const OrthoRound& r) {
  OrthoLayout l;
  l.part = up256(sizeof(PlanTotals));
  l.first = l.part + up256((size_t)8 * O_MAX_MATS * MAX_PARTS);
  l.rest_a = l.first + up256(12 * O_MAX_MATS);
  l.rest_b = l.rest_a + up256((size_t)4 * r.rows);
  l.low_f = l.rest_b + up256((size_t)4 * r.rows);
  l.x0 = l.low_f + up256((size_t)4 * r.rows);
  const size_t x = up256((size_t)2 * r.rows * r.x_ld), a = up256((size_t)2 * r.rows * r.a_ld);
  l.x1 = l.x0 + x;
  l.low = l.x1 + x;
  l.a = l.low + x;
  l.b = l.a + a;
  l.total = l.b + a;
  return l;
}

int check_matrices(const camera_matrix_t* mats, int32_t n, int32_t dtype, bool pointers) {
  if (n < 0 || (n > 0 && mats == nullptr) || (dtype != CAMERA_BF16 && dtype != CAMERA_F32)) return CAMERA_ERR_INVALID_ARG;
  const uintptr_t mask = dtype == CAMERA_BF16 ? 1 : 3;
  for (int i = 0; i < n; ++i) {
    const camera_matrix_t& t = mats[i];
    if (t.rows < 0 || t.cols < 0) return CAMERA_ERR_INVALID_ARG;
    if (t.rows > O_MAX_SIDE || t.cols > O_MAX_SIDE || (t.rows > O_MAX_SIDE / 4 && t.cols > O_MAX_SIDE / 4)) return CAMERA_ERR_UNSUPPORTED_SHAPE;
    if (!pointers || t.rows == 0 || t.cols == 0) continue;
    if (t.in == nullptr || t.out == nullptr || t.in_ld < t.cols || t.out_ld < t.cols || (reinterpret_cast<uintptr_t>(t.in) & mask) ||
        (reinterpret_cast<uintptr_t>(t.out) & 1))
      return CAMERA_ERR_INVALID_ARG;
  }
  return CAMERA_OK;
}

// Bounds of what a step makes of singular values in [0, h]: of |a + b t + c t^2| over t in [0, h^2] (no element of B is
// larger) and of s |a + b s^2 + c s^4| over [0, h] (the singular values after the step).
struct StepBound { double b, h; };
StepBound step_bound(const float* k, double h) {
  const double a = k[0], b = k[1], c = k[2], t1 = h * h;
  double ts[4] = {0.0, t1, t1, t1};
  auto poly = [&](double t) { return fabs(a + t * (b + t * c)); };
  StepBound r = {0.0, 0.0};
  if (c != 0.0 && -b / (2 * c) > 0.0 && -b / (2 * c) < t1) ts[2] = -b / (2 * c);
  for (double t : ts) r.b = fmax(r.b, poly(t));
  ts[2] = ts[3] = t1;
  const double disc = 9 * b * b - 20 * a * c;        // a + 3 b t + 5 c t^2 = 0
  if (c != 0.0 && disc >= 0.0) {
    const double s = sqrt(disc), u = (-3 * b + s) / (10 * c), v = (-3 * b - s) / (10 * c);
    if (u > 0.0 && u < t1) ts[2] = u;
    if (v > 0.0 && v < t1) ts[3] = v;
  } else if (c == 0.0 && b != 0.0 && -a / (3 * b) > 0.0 && -a / (3 * b) < t1) {
    ts[2] = -a / (3 * b);
  }
  for (double t : ts) r.h = fmax(r.h, sqrt(t) * poly(t));
  return r;
}
constexpr double MARGIN = 1.02;         // for the roundings, which the bounds leave out (some 1e-3 a step)
constexpr double MOST = 1e3;            // singular values beyond this: the polynomial is not one that converges
double factor_for(double bound) { return ldexp(1.0, (int)floor(log2(65504.0 / fmax(bound * MARGIN, 1e-3)))); }

// Units of one matrix: symmetric products take, per row tile of 256, the column tiles from the diagonal on; APPLY all.
int units_of(int mode, const OrthoMat& t, int w) {
  const int rt = pad_rows(t.m) / O_TILE_M;
  if (mode == ORTHO_APPLY) return rt * ((t.n + w - 1) / w);
  int units = 0;
  for (int i = 0; i < rt; ++i) units += ((rt - i) * O_TILE_M + w - 1) / w;
  return units;
}

// Tiles: the choice with the least estimated time of a step.  A k block takes 0.60 us for 512 columns, 0.43 for 256, 0.32 for 128:
// all three are what bringing its operands from L2 takes (77 GB/s an SM), of which wide tiles need least.  A unit of 512 columns
// adds its epilogue; smaller ones have two accumulators and overlap it.  A product's units spread over the pairs, those of a later
// product of another matrix fill what they leave (but not where there is one matrix); and no product is over before its longest unit.
struct OrthoTile { int bn, nb; };
OrthoTile choose_tile(const OrthoBatch& b, int n_pairs) {
  static constexpr OrthoTile kinds[3] = {{256, 2}, {256, 1}, {128, 1}};
  static constexpr double k_block[3] = {0.60, 0.43, 0.32}, epilogue[3] = {7.0, 1.0, 0.7};
  OrthoTile best = kinds[0];
  double best_cost = 1e300;
  for (int i = 0; i < 3; ++i) {
    double cost = 0.0;
    for (int mode = 0; mode < 3; ++mode) {
      double sum = 0.0, longest = 0.0;
      for (int e = 0; e < b.n_mats; ++e) {
        const int u = units_of(mode, b.mat[e], kinds[i].bn * kinds[i].nb);
        const double one = pad_cols(mode == ORTHO_GRAM ? b.mat[e].n : b.mat[e].m) / UMMA_BK * k_block[i] + epilogue[i];
        sum += b.n_mats > 1 ? u * one / n_pairs : (double)((u + n_pairs - 1) / n_pairs) * one;
        longest = fmax(longest, one);
      }
      cost += fmax(sum, longest);
    }
    if (cost < best_cost * 0.99) { best = kinds[i]; best_cost = cost; }
  }
  return best;
}

// (fp16 and bf16 differ in nothing a copy without arithmetic sees.)
bool encode(OrthoMaps* m, const void* p, long long rows, long long cols) {
  return encode_bf16_2d_pitch(&m->rows128, p, (uint64_t)rows, (uint64_t)cols, (uint64_t)cols, 128) &&
         encode_bf16_2d_pitch(&m->rows64, p, (uint64_t)rows, (uint64_t)cols, (uint64_t)cols, 64) &&
         encode_bf16_2d_narrow(&m->box, p, (uint64_t)rows, (uint64_t)cols, (uint64_t)cols, 32);
}

// Pairs of CTAs that run at one time, asked of the driver once per device.
int pairs_at_once() {
  static std::atomic<int> known[KNOWN_DEVICES];
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 1; }
  if (dev < KNOWN_DEVICES && (n = known[dev].load(std::memory_order_relaxed)) != 0) return n;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(sm_count() & ~1));
  cfg.blockDim = dim3(O_THREADS);
  cfg.dynamicSmemBytes = O_SMEM_BYTES;
  if (cudaOccupancyMaxActiveClusters(&n, k_ortho, &cfg) != cudaSuccess || n < 1) { cudaGetLastError(); return 1; }
  if (dev < KNOWN_DEVICES) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

#define ORTHO_CK(...)             \
  do {                            \
    if ((__VA_ARGS__) != cudaSuccess) { \
      cudaGetLastError();         \
      return CAMERA_ERR_CUDA;     \
    }                             \
  } while (0)

int run_round(const camera_matrix_t* mats, const OrthoRound& r, int32_t dtype, const float* coefficients, int32_t steps, float eps, char* ws,
              bool first_round, cudaStream_t st) {
  const OrthoLayout l = ortho_layout(r);
  OrthoRun q;
  memset(&q, 0, sizeof(q));
  long long row0 = 0, tiles = 0;
  for (int i = r.begin; i < r.end; ++i) {
    const camera_matrix_t& t = mats[i];
    if (t.rows == 0 || t.cols == 0) continue;
    OrthoMat& o = q.batch.mat[q.batch.n_mats++];
    o.turned = t.rows > t.cols;
    o.m = o.turned ? t.cols : t.rows;
    o.n = o.turned ? t.rows : t.cols;
    o.in = t.in; o.out = t.out; o.in_ld = t.in_ld; o.out_ld = t.out_ld;
    o.row0 = (int)row0;
    row0 += pad_rows(o.m);
    const long long here = (long long)(pad_rows(o.m) / 64) * (pad_cols(o.n) / 64);
    if (here > tiles) tiles = here;
  }
  if (q.batch.n_mats == 0) return CAMERA_OK;
  const int sms = sm_count();
  OrthoLoad ld;
  ld.batch = q.batch;
  ld.part = reinterpret_cast<double*>(ws + l.part);
  ld.first = reinterpret_cast<float*>(ws + l.first);
  ld.small = reinterpret_cast<int*>(ld.first + O_MAX_MATS);
  ld.done = ld.small + O_MAX_MATS;
  ld.eps = eps; ld.x = reinterpret_cast<__half*>(ws + l.x0); ld.x_ld = r.x_ld;
  ld.low = reinterpret_cast<uint4*>(ws + l.low);
  ld.totals = reinterpret_cast<PlanTotals*>(ws);
  ld.clear_status = first_round;
  ld.parts = 8 * sms / q.batch.n_mats;
  if (ld.parts > MAX_PARTS) ld.parts = MAX_PARTS;
  if (ld.parts < 8) ld.parts = 8;
  long long load_ctas = 8ll * sms / q.batch.n_mats + 1;
  if (load_ctas > tiles) load_ctas = tiles;
  if (dtype == CAMERA_BF16) {
    ORTHO_CK(launch_chained(k_ortho_norm<__nv_bfloat16>, ld, ld.parts, q.batch.n_mats, 1, LOAD_THREADS, 0, false, st));
    ORTHO_CK(launch_chained(k_ortho_load<__nv_bfloat16>, ld, (int)load_ctas, q.batch.n_mats, 1, LOAD_THREADS, 0, true, st));
  } else {
    ORTHO_CK(launch_chained(k_ortho_norm<float>, ld, ld.parts, q.batch.n_mats, 1, LOAD_THREADS, 0, false, st));
    ORTHO_CK(launch_chained(k_ortho_load<float>, ld, (int)load_ctas, q.batch.n_mats, 1, LOAD_THREADS, 0, true, st));
  }
  if (!encode(&q.maps[BUF_X0], ws + l.x0, r.rows, r.x_ld) || !encode(&q.maps[BUF_X1], ws + l.x1, r.rows, r.x_ld) ||
      !encode(&q.maps[BUF_A], ws + l.a, r.rows, r.a_ld) || !encode(&q.maps[BUF_B], ws + l.b, r.rows, r.a_ld))
    return CAMERA_ERR_CUDA;
  q.out[0] = reinterpret_cast<__half*>(ws + l.a);
  q.out[1] = reinterpret_cast<__half*>(ws + l.b);
  q.out_ld = r.a_ld;
  q.rest[0] = reinterpret_cast<float*>(ws + l.rest_a);
  q.rest[1] = reinterpret_cast<float*>(ws + l.rest_b);
  q.low_f = reinterpret_cast<float*>(ws + l.low_f);
  q.low = ld.low; q.low_ld = r.x_ld; q.low_first = dtype == CAMERA_F32;
  q.first = ld.first; q.small = ld.small; q.done = ld.done; q.totals = ld.totals;
  q.wait_limit_ns = current_wait_limit_ns();
  double h = 1.0, sx = 1.0;             // the first X's factor is known on the device only
  double grown = 1.0;                   // what the steps so far can have made of a small singular value
  for (int s = 0; s < steps; ++s) {
    const float* const k = coefficients + 3 * s;
    const StepBound bound = step_bound(k, h * MARGIN);
    const double sa = factor_for(h * h), sb = factor_for(bound.b), sn = factor_for(bound.h);
    OrthoStep& o = q.step[s];
    o.f_gram = (float)(sa / (sx * sx));
    o.f_poly = (float)(sb * k[2] / (sa * sa)); o.f_aux = (float)(sb * k[1] / sa); o.f_diag = (float)(sb * k[0]);
    o.f_apply = (float)((s + 1 == steps ? 1.0 : sn) / (sb * sx));
    o.small_in = (int)ceil(log2(fmax(grown / h, 1.0)));
    grown *= bound.b * MARGIN;
    o.small_out = (int)ceil(log2(fmax(grown / bound.h, 1.0)));
    h = bound.h;
    sx = sn;
    double growth = 1.0;
    for (int later = s + 1; later < steps; ++later) growth = fmin(growth * fmax(fabs((double)coefficients[3 * later]), 1.0), 1e30);
    o.f_low = (float)(1.0 / (1.0 + (growth / 8) * (growth / 8)));
  }
  ORTHO_CK(allow_smem<k_ortho, O_SMEM_BYTES>());
  int pairs = pairs_at_once();
  const OrthoTile t = choose_tile(q.batch, pairs);
  q.bn = t.bn; q.nb = t.nb;
  q.n_acc = t.nb * t.bn <= 256 ? 2 : 1;
  q.kps = t.nb * t.bn <= 128 ? 2 : 1;        // two small k blocks a stage: a stage costs the issuing thread as much as one takes
  const int stage = q.kps * (O_A_BYTES + t.nb * t.bn * 64);
  q.n_stages = O_RING_BYTES / stage < O_MAX_STAGES ? O_RING_BYTES / stage : O_MAX_STAGES;
  int most = 0;
  for (int mode = 0; mode < 3; ++mode) {
    int units = 0;
    for (int e = 0; e < q.batch.n_mats; ++e) {
      q.unit0[mode][e] = units;
      units += units_of(mode, q.batch.mat[e], t.nb * t.bn);
    }
    q.unit0[mode][q.batch.n_mats] = units;
    q.per_step += units;
    if (units > most) most = units;
  }
  q.n_steps = steps;
  q.n_units = steps * q.per_step;
  // with one matrix a product's units are all there is to do at one time
  if (q.batch.n_mats == 1 && most < pairs) pairs = most;
  if (q.per_step < pairs) pairs = q.per_step;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(2 * pairs));
  cfg.blockDim = dim3(O_THREADS);
  cfg.dynamicSmemBytes = O_SMEM_BYTES;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeCooperative;        // units wait for those of other CTAs, so all run at one time
  at[0].val.cooperative = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, k_ortho, q) != cudaSuccess) {
    cudaGetLastError();                             // a context without cooperative launches: one pair, which waits for nobody else
    cfg.gridDim = dim3(2);
    cfg.numAttrs = 0;
    ORTHO_CK(cudaLaunchKernelEx(&cfg, k_ortho, q));
  }
  return CAMERA_OK;
}

}  // namespace
}  // namespace camera

extern "C" size_t camera_orthogonalize_workspace_bytes(const camera_matrix_t* mats, int32_t n_mats) {
  using namespace camera;
  if (check_matrices(mats, n_mats, CAMERA_BF16, false) != CAMERA_OK) return 0;
  size_t most = ortho_layout(OrthoRound{0, 0, 0, 0, 0}).total;
  for (int at = 0; at < n_mats;) {
    const OrthoRound r = ortho_round(mats, n_mats, at);
    const size_t need = ortho_layout(r).total;
    if (need > most) most = need;
    at = r.end;
  }
  return most;
}

extern "C" int camera_orthogonalize(const camera_matrix_t* mats, int32_t n_mats, int32_t dtype, const float* coefficients, int32_t steps,
                                    float eps, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  using namespace camera;
  const int rc = check_matrices(mats, n_mats, dtype, true);
  if (rc != CAMERA_OK) return rc;
  if (steps < 1 || steps > O_MAX_STEPS || coefficients == nullptr || !(eps >= 0.f) || !(eps < 3.0e38f)) return CAMERA_ERR_INVALID_ARG;
  double h = 1.0;
  for (int s = 0; s < steps; ++s) {
    for (int i = 0; i < 3; ++i)
      if (!isfinite(coefficients[3 * s + i])) return CAMERA_ERR_INVALID_ARG;
    const StepBound b = step_bound(coefficients + 3 * s, h * MARGIN);
    if (!(b.h <= MOST) || !(b.b <= MOST)) return CAMERA_ERR_INVALID_ARG;
    h = b.h;
  }
  if (workspace == nullptr || workspace_bytes < camera_orthogonalize_workspace_bytes(mats, n_mats) ||
      (reinterpret_cast<uintptr_t>(workspace) & 255))
    return CAMERA_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* const ws = static_cast<char*>(workspace);
  bool first = true;
  for (int at = 0; at < n_mats;) {
    const OrthoRound r = ortho_round(mats, n_mats, at);
    const int e = run_round(mats, r, dtype, coefficients, steps, eps, ws, first, st);
    if (e != CAMERA_OK) return e;
    if (r.rows > 0) first = false;
    at = r.end;
  }
  if (first) ORTHO_CK(cudaMemsetAsync(ws, 0, sizeof(PlanTotals), st));
  return CAMERA_OK;
}
