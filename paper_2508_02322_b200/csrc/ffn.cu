// The gated feed-forward block of one expert, forward and backward (Eq. 1-2 without the router):
//   G = X Wg^T, U = X Wu^T, H = SiLU(G) * U, Y = H Wd^T
//   dH = dY Wd,  dU = dH * SiLU(G),  dG = dH * U * s (1 + G (1 - s)) with s = sigmoid(G)
//   dX = dG Wg + dU Wu,  dWg = dG^T X,  dWu = dU^T X,  dWd = dY^T H
//
// Five GEMM shapes, one kernel (k_ffn_gemm) on CTA pairs (tcgen05 cta_group::2), which differ in the orientation of
// their operands in memory and in the epilogue:
//   GATE_UP  A = X, B = Wg and Wu, both with K (d_model) contiguous; epilogue writes H and, for a backward pass, G and U
//   DOWN     A = H, B = Wd, K (d_ff) contiguous; epilogue writes Y
//   DH       A = dY (K = d_model contiguous), B = Wd with N (d_ff) contiguous; epilogue reads G, U and writes dG, dU, H
//   DX       A = dG then dU (K = d_ff contiguous), B = Wg then Wu with N (d_model) contiguous: one accumulator for both
//   DW       three problems in one launch: A = dG / dU / dY, B = X / X / H, both with K (tokens) as the slow dimension
// H, dG and dU are rounded to bf16, being operands of the next product on the tensor cores (camera_layer_forward rounds its h
// likewise): results are 2.3e-3 to 2.5e-3 off 64 bits (root mean square, relative), products kept in 32 bits and rounded
// once at the end 1.7e-3.
// An operand whose M or N index is the contiguous one is loaded as boxes of 64 of those x 64 k and described to the MMA
// as MN-major; nothing is transposed in memory.
#include <cuda.h>
#include <string.h>

#include "common.cuh"
#include "launch.cuh"
#include "umma.cuh"
#include "umma_pair.cuh"

namespace camera {

namespace {

constexpr int G_EPI_WARPS = 8;               // epilogue: two warps per 32 rows, each with half of the columns
constexpr int G_PRODUCER = G_EPI_WARPS, G_ISSUER = G_EPI_WARPS + 1;
constexpr int G_THREADS = 32 * (G_EPI_WARPS + 2);
constexpr int G_TILE_M = 256;                // rows of the output a pair computes: 128 per CTA
constexpr int G_A_BYTES = 128 * 128;         // this CTA's 128 rows x 64 k
constexpr int G_MAX_STAGES = 8;
constexpr int G_RING_BYTES = 192 * 1024;
constexpr int G_SMEM_BYTES = G_RING_BYTES + 256 + 1024;
constexpr int G_GROUP_M = 16;                // row tiles that are walked together (see decode)
constexpr int G_TMEM_COLS = 512;

enum { FFN_GATE_UP = 0, FFN_DOWN = 1, FFN_DH = 2, FFN_DX = 3, FFN_DW = 4 };

struct FfnProblem {
  int m, n;                 // rows and columns of the output
  int n_tiles, unit0;       // column tiles; first work unit of this problem
  __nv_bfloat16* out;
  long long ld;             // of out
};

struct FfnGemm {
  CUtensorMap a[3], b[3];   // per problem (DW) or per k segment (DX); GATE_UP: b[0] gate, b[1] up
  FfnProblem prob[3];
  int n_prob, n_units;
  int n_kb;                 // k blocks per segment
  int splits, tiles;        // DOWN, DX: parts of the sum over k, each a work unit per tile; tiles of one part
  float* part;              // splits > 1: where the parts' sums go, [splits][m][n] fp32
  int kps;                  // k blocks per stage of the ring (1 or 2)
  int bn, nb;               // columns per B tile; B tiles per work unit (GATE_UP: 2, one of each matrix)
  int n_stages, n_acc;      // ring depth; accumulator sets in tensor memory
  uint16_t *g, *u;          // GATE_UP: where to keep the upper halves of G and U (or null); DH: inputs
  long long lo_off;         // the lower byte of the element at g + i is at (uint8_t*)g + lo_off + i
  __nv_bfloat16 *dg, *du, *h;   // DH outputs; GATE_UP: h
  long long act_ld, h_ld;   // pitch of g and u, dg and du; of h
  PlanTotals* totals;
  int clear_status;         // first kernel of the call
  unsigned long long wait_limit_ns;
};

struct FfnUnit { int p, m0, n0, two, k0, k1, split; };

// Units of a problem are numbered group by group of G_GROUP_M row tiles, inside a group column tile by column tile and
// the row tile fastest: the pairs at work at one time share a few column tiles of B and a block of rows of A, both of
// which stay in L2.
template <int MODE>
__device__ __forceinline__ FfnUnit decode(const FfnGemm& q, int unit) {
  constexpr bool dual = MODE == FFN_GATE_UP, SPLIT = MODE == FFN_DOWN || MODE == FFN_DX;
  FfnUnit r;
  r.p = 0;
  r.split = 0;
  r.k0 = 0;
  r.k1 = MODE == FFN_DX ? 2 * q.n_kb : q.n_kb;
  if (SPLIT && q.splits > 1) {
    r.split = unit / q.tiles;
    unit -= r.split * q.tiles;
    const int all = r.k1;
    r.k0 = all * r.split / q.splits;
    r.k1 = all * (r.split + 1) / q.splits;
  }
  while (r.p + 1 < q.n_prob && unit >= q.prob[r.p + 1].unit0) ++r.p;
  const FfnProblem& pr = q.prob[r.p];
  const int m_tiles = (pr.m + G_TILE_M - 1) / G_TILE_M;
  int rem = unit - pr.unit0;
  const int per_group = G_GROUP_M * pr.n_tiles;
  const int grp = rem / per_group;
  rem -= grp * per_group;
  const int in_group = min(G_GROUP_M, m_tiles - grp * G_GROUP_M);
  r.m0 = (grp * G_GROUP_M + rem % in_group) * G_TILE_M;
  r.n0 = (rem / in_group) * (dual ? q.bn : q.nb * q.bn);
  r.two = dual || (q.nb == 2 && r.n0 + q.bn < pr.n);
  return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// G and U are kept for the backward pass with 24 of their 32 bits (15 of mantissa): rounding them to bf16 would add as
// much error to the gradients as everything else together (relative error of the weight gradients against 64 bits
// 3.5e-3 with bf16, 2.4e-3 with 24 bits, of which 1.7e-3 is the rounding of the result).  The cut is a
// truncation, so that NaN and infinity survive it.
__device__ __forceinline__ void keep24(uint16_t* hi, uint8_t* lo, const uint32_t* v) {
  uint32_t h[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) h[j] = __byte_perm(v[2 * j], v[2 * j + 1], 0x7632);
  st_global_v8(hi, h);
  uint32_t l[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    l[j] = __byte_perm(__byte_perm(v[4 * j], v[4 * j + 1], 0x0051), __byte_perm(v[4 * j + 2], v[4 * j + 3], 0x0051), 0x5410);
  *reinterpret_cast<uint4*>(lo) = make_uint4(l[0], l[1], l[2], l[3]);
}
// Element j (0 .. 15) of a chunk of 16: h its 8 words of upper halves, l its 4 words of lower bytes.
__device__ __forceinline__ float kept24(const uint32_t* h, const uint32_t* l, int j) {
  const uint32_t top = j & 1 ? h[j >> 1] & 0xffff0000u : h[j >> 1] << 16;
  return __uint_as_float(top | (((l[j >> 2] >> (8 * (j & 3))) & 0xffu) << 8));
}
// 16 kept elements of G and U on their way from memory.
struct Kept {
  uint4 g[2], u[2], g_lo, u_lo;
  __device__ __forceinline__ void load(const FfnGemm& q, long long at) {
    const long long u_off = q.u - q.g;
    const uint8_t* const lo = reinterpret_cast<const uint8_t*>(q.g) + q.lo_off;
    const uint4* const gp = reinterpret_cast<const uint4*>(q.g + at);
    const uint4* const up = reinterpret_cast<const uint4*>(q.g + at + u_off);
    g[0] = gp[0]; g[1] = gp[1];
    u[0] = up[0]; u[1] = up[1];
    g_lo = *reinterpret_cast<const uint4*>(lo + at);
    u_lo = *reinterpret_cast<const uint4*>(lo + at + u_off);
  }
  __device__ __forceinline__ float gate(int j) const {
    return kept24(reinterpret_cast<const uint32_t*>(g), reinterpret_cast<const uint32_t*>(&g_lo), j);
  }
  __device__ __forceinline__ float up(int j) const {
    return kept24(reinterpret_cast<const uint32_t*>(u), reinterpret_cast<const uint32_t*>(&u_lo), j);
  }
};
__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }

// Bound by the tensor pipe once tiles fill the 74 pairs, and by the power cap: 4096 tokens, d_model 3584, d_ff 20480
// forward 1220 us after a pause and 1370 to 1410 us call after call (1104 us at cuBLAS's burst rate, 1306 us at its
// rate under the cap), a training pass over 8192 tokens at d_ff 2560 1063 and 1190 to 1245 us (828 and 980 us).  Smaller
// problems by the k blocks in a row, 0.32 to 0.39 us each.
template <int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(G_THREADS, 1) k_ffn_gemm(const __grid_constant__ FfnGemm q) {
  constexpr bool A_MN = MODE == FFN_DW;
  constexpr bool B_MN = MODE == FFN_DH || MODE == FFN_DX || MODE == FFN_DW;
  constexpr bool DUAL = MODE == FFN_GATE_UP;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t bars = base + G_RING_BYTES;
  auto full_bar = [&](int s) { return bars + 8u * s; };                                 // first CTA
  auto empty_bar = [&](int s) { return bars + 8u * (G_MAX_STAGES + s); };               // each CTA
  auto tfull_bar = [&](int a) { return bars + 8u * (2 * G_MAX_STAGES + a); };           // each CTA
  auto tempty_bar = [&](int a) { return bars + 8u * (2 * G_MAX_STAGES + 2 + a); };      // first CTA, the pair's epilogue threads
  uint8_t* const tail = base_ptr + G_RING_BYTES + 8 * (2 * G_MAX_STAGES + 4);
  volatile uint32_t* const tmem_slot = reinterpret_cast<volatile uint32_t*>(tail);
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(tail + 8);

  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  const uint32_t rank = cluster_ctarank();
  const int n_pairs = gridDim.x >> 1, pair = blockIdx.x >> 1;
  const int half = q.bn >> 1;                               // columns of a B tile this CTA supplies
  const int b_bytes = half * 128;
  const int block_bytes = G_A_BYTES + q.nb * b_bytes;      // operands of one k block
  const int stage_bytes = q.kps * block_bytes;

  if (tid == 0) {
    for (int s = 0; s < q.n_stages; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 2 * 32 * G_EPI_WARPS); }
    wait_state_init(abort_flag, q.wait_limit_ns);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == G_ISSUER) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)),
                 "r"(G_TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();     // the other CTA's barriers are initialised before anything arrives on them
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  // The next kernel of the call may take SMs as they fall free and set itself up; what it reads or writes beyond that
  // waits for the kernels before it (here) to end.
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // The call's first kernel clears its status word.  A CTA that gives up records that at its end, 2 ms after the wait that
  // ran out at the earliest, when every CTA of the grid (one per SM) has long started.
  if (q.clear_status && blockIdx.x == 0 && tid == 0) atomicExch(&q.totals->status, 0);

  if (warp == G_PRODUCER) {
    // ------------------------------------------------------------------ TMA producer (each CTA loads its own share)
    const uint32_t lead = lane == 0;
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int unit = pair; ok && unit < q.n_units; unit += n_pairs) {
      const FfnUnit u = decode<MODE>(q, unit);
      const int am = u.m0 + 128 * (int)rank, bn0 = u.n0 + half * (int)rank;
      for (int t = u.k0, blocks; t < u.k1; t += blocks) {
        const int seg = MODE == FFN_DX && t >= q.n_kb, kb = t - seg * q.n_kb;
        const CUtensorMap* const map_a = &q.a[MODE == FFN_DX ? seg : u.p];
        const CUtensorMap* const map_b = &q.b[MODE == FFN_DX ? seg : u.p];
        const CUtensorMap* const map_b2 = DUAL ? &q.b[1] : map_b;
        const int bn1 = DUAL ? bn0 : bn0 + q.bn;
        blocks = min(q.kps, min(q.n_kb - kb, u.k1 - t));
        ok = warp_wait(empty_bar(stage), phase ^ 1u, abort_flag);
        if (!ok) break;
        const uint32_t full0 = map_to_cta(full_bar(stage), 0);
        if (rank == 0 && lane == 0) mbar_expect_tx(full_bar(stage), 2 * blocks * (G_A_BYTES + (u.two ? 2 : 1) * b_bytes));
        __syncwarp();
        uint32_t dst = base + stage * stage_bytes;
        for (int k0 = kb * UMMA_BK; k0 < (kb + blocks) * UMMA_BK; k0 += UMMA_BK, dst += block_bytes) {
          // whatever lies past a matrix's last row or column arrives as zeros
          if (A_MN) {
            tma_load_lead(lead, dst, map_a, full0, am, k0);
            tma_load_lead(lead, dst + 8192, map_a, full0, am + 64, k0);
          } else {
            tma_load_lead(lead, dst, map_a, full0, k0, am);
          }
          const uint32_t dst_b = dst + G_A_BYTES;
          if (B_MN) {
            tma_load_lead(lead, dst_b, map_b, full0, bn0, k0);
            if (half > 64) tma_load_lead(lead, dst_b + 8192, map_b, full0, bn0 + 64, k0);
            if (u.two) {
              tma_load_lead(lead, dst_b + b_bytes, map_b2, full0, bn1, k0);
              if (half > 64) tma_load_lead(lead, dst_b + b_bytes + 8192, map_b2, full0, bn1 + 64, k0);
            }
          } else {
            tma_load_lead(lead, dst_b, map_b, full0, k0, bn0);
            if (u.two) tma_load_lead(lead, dst_b + b_bytes, map_b2, full0, k0, bn1);
          }
        }
        if (++stage == q.n_stages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok) {               // copies in flight land before the CTA's shared memory is given up
      const unsigned long long t0 = globaltimer_ns();
      while (globaltimer_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
  } else if (warp == G_ISSUER) {
    // ------------------------------------------------------------------ MMA issuer (first CTA of the pair only)
    if (rank == 0) {
      const uint32_t lead = lane == 0;
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true, ready = false;       // ready: the next stage has been seen full
      const uint32_t idesc = make_idesc_pair(q.bn) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u);
      constexpr int A_STEP = A_MN ? 2048 >> 4 : 32 >> 4, B_STEP = B_MN ? 2048 >> 4 : 32 >> 4;     // 16 k further
      const unsigned long long a_first = A_MN ? make_smem_desc_mn(base) : make_smem_desc(base);
      const unsigned long long b_first = B_MN ? make_smem_desc_mn(base + G_A_BYTES) : make_smem_desc(base + G_A_BYTES);
      const unsigned long long b2_off = (unsigned long long)(b_bytes >> 4);
      for (int unit = pair; ok && unit < q.n_units; unit += n_pairs) {
        const FfnUnit u = decode<MODE>(q, unit);
        ok = __all_sync(0xffffffffu, mbar_wait_cluster(tempty_bar(acc), acc_phase ^ 1u, abort_flag));
        if (!ok) break;
        tc_fence_after();
        const uint32_t d0 = tmem_base + (uint32_t)(acc * q.nb * q.bn), d1 = d0 + (uint32_t)q.bn;
        uint32_t accumulate = 0;
        for (int t = u.k0, blocks; t < u.k1; t += blocks) {
          blocks = min(q.kps, u.k1 - t);
          if (MODE == FFN_DX && t < q.n_kb) blocks = min(blocks, q.n_kb - t);      // a stage holds one segment's blocks
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
#pragma unroll
              for (int k = 0; k < UMMA_BK / 16; ++k) {
                umma_lead(lead, d0, a_desc + A_STEP * k, b_desc + B_STEP * k, idesc, accumulate | (uint32_t)k);
                umma_lead(lead, d1, a_desc + A_STEP * k, b2_desc + B_STEP * k, idesc, accumulate | (uint32_t)k);
              }
            } else {
              umma_block<A_STEP, B_STEP>(lead, d0, a_desc, b_desc, idesc, accumulate);
            }
            accumulate = 1;
          }
          // The tensor pipe holds only a few MMAs: a look at the next stage's barrier while they run.
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
    // Loads of the next chunk (tensor memory, and for DH the kept products from global memory) fly while one is worked on.
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    const int c_half = (DUAL ? q.bn : q.nb * q.bn) / 2, c_first = c_half * (warp >> 2);
    constexpr int c_step = 16;
    for (int unit = pair; ok && unit < q.n_units; unit += n_pairs) {
      const FfnUnit u = decode<MODE>(q, unit);
      const FfnProblem& pr = q.prob[u.p];
      const long long row = (long long)u.m0 + 128 * (int)rank + (warp & 3) * 32 + lane;
      const bool live = row < pr.m;
      const int cols = min(pr.n - u.n0, c_first + c_half);     // where this warp's columns end
      [[maybe_unused]] Kept next;
      if constexpr (MODE == FFN_DH) {
        if (live && c_first < cols) next.load(q, row * q.act_ld + u.n0 + c_first);
      }
      ok = __all_sync(0xffffffffu, mbar_wait(tfull_bar(acc), acc_phase, abort_flag));
      if (!ok) break;
      tc_fence_after();
      const uint32_t t0 = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(acc * q.nb * q.bn);
      if constexpr (MODE == FFN_GATE_UP) {
        __nv_bfloat16* const h = q.h + row * q.h_ld + u.n0;
        const bool keep = q.g != nullptr;
        const long long g_at = row * q.act_ld + u.n0, u_at = g_at + (q.u - q.g);
        uint8_t* const lo = reinterpret_cast<uint8_t*>(q.g) + q.lo_off;
        auto put = [&](const uint32_t* vg, const uint32_t* vu, int c) {
          if (!live) return;
          uint32_t p[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float g0 = __uint_as_float(vg[2 * j]), g1 = __uint_as_float(vg[2 * j + 1]);
            p[j] = pack_bf16(g0 * sigmoid(g0) * __uint_as_float(vu[2 * j]), g1 * sigmoid(g1) * __uint_as_float(vu[2 * j + 1]));
          }
          st_global_v8(h + c, p);                      // the pitches of h, g, u are multiples of 64: whole chunks fit
          if (keep) {
            keep24(q.g + g_at + c, lo + g_at + c, vg);
            keep24(q.g + u_at + c, lo + u_at + c, vu);
          }
        };
        uint32_t g0[16], u0[16], g1[16], u1[16];
        int c = c_first;
        if (c < cols) { tmem_ld16(t0 + c, g0); tmem_ld16(t0 + q.bn + c, u0); }
        for (; c < cols; c += 2 * c_step) {
          const int c1 = c + c_step, c2 = c1 + c_step;
          tmem_ld_wait(g0, u0);
          if (c1 < cols) { tmem_ld16(t0 + c1, g1); tmem_ld16(t0 + q.bn + c1, u1); }
          put(g0, u0, c);
          if (c1 >= cols) break;
          tmem_ld_wait(g1, u1);
          if (c2 < cols) { tmem_ld16(t0 + c2, g0); tmem_ld16(t0 + q.bn + c2, u0); }
          put(g1, u1, c1);
        }
      } else if constexpr (MODE == FFN_DH) {
        const long long at = row * q.act_ld + u.n0;
        for (int c = c_first; c < cols; c += c_step) {
          uint32_t v[16], pg[8], pu[8], ph[8];
          tmem_ld16(t0 + c, v);
          const Kept kept = next;
          if (live && c + c_step < cols) next.load(q, at + c + c_step);
          tmem_ld_wait(v);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float dg[2], du[2], h[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float g = kept.gate(2 * j + e), up = kept.up(2 * j + e);
              const float dh = __uint_as_float(v[2 * j + e]), s = sigmoid(g), act = g * s;
              h[e] = act * up;
              du[e] = dh * act;
              dg[e] = dh * up * fmaf(act, 1.f - s, s);
            }
            pg[j] = pack_bf16(dg[0], dg[1]);
            pu[j] = pack_bf16(du[0], du[1]);
            ph[j] = pack_bf16(h[0], h[1]);
          }
          if (live) {
            st_global_v8(q.dg + at + c, pg);
            st_global_v8(q.du + at + c, pu);
            st_global_v8(q.h + row * q.h_ld + u.n0 + c, ph);
          }
        }
      } else {
        __nv_bfloat16* const out = pr.out + row * pr.ld + u.n0;
        const bool whole = q.splits <= 1;
        // Rows of an odd multiple of 16 bytes start off a 32-byte sector every other time: such a row is stored half a
        // chunk later, so that whole sectors are written all the same (dW of 40 tokens, 3000 x 15000: 155 -> 115 us).
        const bool sectors = (reinterpret_cast<uintptr_t>(out + c_first) & 31) == 0;
        uint32_t carry[4] = {0u, 0u, 0u, 0u};
        float* const part = q.part + ((long long)u.split * pr.m + row) * pr.n + u.n0;
        auto put = [&](const uint32_t* v, int c) {
          if (!live) return;
          if (!whole) {                    // n is a multiple of 8 here (d_model)
            st_global_v8(part + c, v);
            if (c + 16 <= cols) st_global_v8(part + c + 8, v + 8);
            return;
          }
          uint32_t p[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) p[j] = pack_bf16(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1]));
          if (sectors && c + 16 <= cols) {
            st_global_v8(out + c, p);
            return;
          }
          if (!sectors) {
            if (c > c_first) {             // the chunk before left its second half
              if (c + 8 <= cols) {
                const uint32_t w[8] = {carry[0], carry[1], carry[2], carry[3], p[0], p[1], p[2], p[3]};
                st_global_v8(out + c - 8, w);
              } else {
                *reinterpret_cast<uint4*>(out + c - 8) = make_uint4(carry[0], carry[1], carry[2], carry[3]);
              }
            } else if (c + 8 <= cols) {
              *reinterpret_cast<uint4*>(out + c) = make_uint4(p[0], p[1], p[2], p[3]);
            }
            if (c + 16 < cols) {
#pragma unroll
              for (int j = 0; j < 4; ++j) carry[j] = p[4 + j];
              return;
            }
            if (c + 16 == cols) {
              *reinterpret_cast<uint4*>(out + c + 8) = make_uint4(p[4], p[5], p[6], p[7]);
              return;
            }
          }
          // the last, ragged chunk, without the half that has been stored
          const int from = !sectors && c + 8 <= cols ? 8 : 0;
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j >= from && c + j < cols)
              out[c + j] = __ushort_as_bfloat16((unsigned short)(j & 1 ? p[j >> 1] >> 16 : p[j >> 1] & 0xffffu));
        };
        uint32_t v0[16], v1[16];
        int c = c_first;
        if (c < cols) tmem_ld16(t0 + c, v0);
        for (; c < cols; c += 2 * c_step) {
          const int c1 = c + c_step, c2 = c1 + c_step;
          tmem_ld_wait(v0);
          if (c1 < cols) tmem_ld16(t0 + c1, v1);
          put(v0, c);
          if (c1 >= cols) break;
          tmem_ld_wait(v1);
          if (c2 < cols) tmem_ld16(t0 + c2, v0);
          put(v1, c1);
        }
      }
      tc_fence_before();
      mbar_arrive_cluster(map_to_cta(tempty_bar(acc), 0));
      if (++acc == q.n_acc) { acc = 0; acc_phase ^= 1u; }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag && tid == 0) atomicExch(&q.totals->status, (int)CAMERA_ERR_DEVICE_TIMEOUT);
  cluster_sync_all();     // neither CTA leaves while the other may still read its shared or tensor memory
  if (warp == G_ISSUER) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(G_TMEM_COLS) : "memory");
  }
}

// Sums of the parts of a split k in order, rounded: 8 elements per thread.  Bound by its start and the parts' bytes, which
// are still in L2 (about 4 us); with it 100 tokens, 1024 x 9000 take 29 us forward, 60 us without a split.
__global__ void __launch_bounds__(256) k_ffn_join(const FfnGemm q) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const long long n = (long long)q.prob[0].m * q.prob[0].n, i = 8 * ((long long)blockIdx.x * 256 + threadIdx.x);
  if (i >= n) return;
  float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < q.splits; ++s) {
    const float4* const src = reinterpret_cast<const float4*>(q.part + s * n + i);
    const float4 a = src[0], b = src[1];
    sum[0] += a.x; sum[1] += a.y; sum[2] += a.z; sum[3] += a.w;
    sum[4] += b.x; sum[5] += b.y; sum[6] += b.z; sum[7] += b.w;
  }
  // the output's rows are as long as they are wide (y, dx)
  *reinterpret_cast<uint4*>(q.prob[0].out + i) = make_uint4(pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3]),
                                                            pack_bf16(sum[4], sum[5]), pack_bf16(sum[6], sum[7]));
}

// ------------------------------------------------------------------------------------------------ few tokens
// Up to 8 * NT tokens: the work is reading the weights once.  A tensor-core tile of 256 rows would be mostly padding and
// its column tiles too few to keep every SM's loads in flight, so these kernels stream the weights into the A fragments of
// mma.sync (m16n8k16).  A lane takes 16 bytes = 8 consecutive k of its row, which is its share of two MMAs once the k
// index is permuted the same way in both operands; it copies them itself (cp.async) into its own places of a ring in
// shared memory, so a warp waits for nothing but its own copies.  The tokens are the n index; their fragments come the
// same way from x or h, through L1.
// The 8 warps of a CTA lie WK along k and 8 / WK along the rows, a warp has R tiles of 16 rows: at a step the CTA reads
// 128 WK contiguous bytes of each of its 16 R 8 / WK rows (DRAM wants runs), and its warps read the tokens' fragments
// 8 / WK times.  GATE_UP tiles are 8 rows of Wg over the same 8 rows of Wu, so that a thread ends with gate and up of one
// element.  Where that gives too few CTAs to fill the GPU, k is split further over the CTAs of a cluster (up to 8).  The
// sums of the warps and CTAs along k meet through (distributed) shared memory in a fixed order.
// Bound by the weights' bytes: 24 tokens through 20480 micro-experts of d_model 3584 take 101 to 105 us (4.2 TB/s; with
// 128-byte runs a row 137 us), one token through 2560 of them 16.4 us a call (3.4 TB/s; 12.3 us where the weights of one
// call after the other are found in L2), two kernels' start and end among them.
constexpr int S_WARPS = 8;
constexpr int S_THREADS = 32 * S_WARPS;
constexpr int S_STEP_BYTES = S_THREADS * 64;       // a step of one tile per warp

struct FfnFew {
  const __nv_bfloat16 *w0, *w1;    // GATE_UP: Wg, Wu; DOWN: Wd in both
  const __nv_bfloat16* in;         // x or h
  long long w_ld, in_ld, out_ld;
  int rows, k, T;                  // weight rows (d_ff or d_model), length of the sums, tokens
  __nv_bfloat16* out;              // h or y
  uint16_t* g;                     // as in FfnGemm
  long long u_off, lo_off, act_ld;
  PlanTotals* totals;
};

__device__ __forceinline__ void mma16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The first n (< 8) of 8 bf16, the others zero: what lies behind the last column of a pitched matrix may be anything.
__device__ __forceinline__ uint4 first_n(uint4 v, int n) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] &= (2 * i < n ? 0xffffu : 0u) | (2 * i + 1 < n ? 0xffff0000u : 0u);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t cluster_addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr) : "memory");
  return v;
}
__device__ __forceinline__ void cluster_barrier() {
  __syncthreads();
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

// One element's results: gate and up of (token, micro-expert), or one (GATE_UP false: lo) or two rows of y.
template <bool GATE_UP>
__device__ __forceinline__ void few_store(const FfnFew& q, int row, int tok, float lo, float hi) {
  if (tok >= q.T) return;
  if (GATE_UP) {
    if (row >= q.rows) return;
    q.out[(size_t)tok * q.out_ld + row] = __float2bfloat16_rn(lo * sigmoid(lo) * hi);
    if (q.g != nullptr) {
      const size_t ga = (size_t)tok * q.act_ld + row, ua = ga + q.u_off;
      uint8_t* const low = reinterpret_cast<uint8_t*>(q.g) + q.lo_off;
      const uint32_t gb = __float_as_uint(lo), ub = __float_as_uint(hi);
      q.g[ga] = (uint16_t)(gb >> 16); low[ga] = (uint8_t)(gb >> 8);
      q.g[ua] = (uint16_t)(ub >> 16); low[ua] = (uint8_t)(ub >> 8);
    }
  } else {
    if (row < q.rows) q.out[(size_t)tok * q.out_ld + row] = __float2bfloat16_rn(lo);
    if (row + 8 < q.rows) q.out[(size_t)tok * q.out_ld + row + 8] = __float2bfloat16_rn(hi);
  }
}

// SLOTS: steps in the ring.  AHEAD: the tokens' fragments of a step are loaded during the step before.
template <bool GATE_UP, int WK, int R, int NT, int SLOTS, int CTAS>
__global__ void __launch_bounds__(S_THREADS, CTAS) k_ffn_few(const FfnFew q) {
  constexpr bool AHEAD = NT <= 4;
  extern __shared__ __align__(16) uint8_t few_ring[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, tg = lane & 3;
  const int splits = gridDim.y, split = blockIdx.y;
  constexpr int TILE = GATE_UP ? 8 : 16;                    // rows of the result per tile
  constexpr int TILES = S_WARPS / WK * R, KSTEP = 64 * WK;  // tiles of the CTA; k of a step
  const int warp_k = warp % WK, warp_r = warp / WK;
  const int row0 = (blockIdx.x * TILES + warp_r * R) * TILE;
  if (GATE_UP) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (blockIdx.x == 0 && split == 0 && tid == 0) q.totals->status = 0;       // nothing here can fail
  }
  const int steps = (q.k + KSTEP - 1) / KSTEP;
  const int s0 = steps * split / splits, s1 = steps * (split + 1) / splits;
  // this lane's two weight rows of each tile; a row past the last one, and k past the end, are filled with zeros
  const __nv_bfloat16* w[R][2];
  uint32_t has = 0;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = row0 + r * TILE + g + (GATE_UP ? 0 : 8 * e);
      if (row < q.rows) has |= 1u << (2 * r + e);
      w[r][e] = (e ? q.w1 : q.w0) + (row < q.rows ? (size_t)row * q.w_ld : 0) + tg * 8;
    }
  const uint32_t mine = smem_u32(few_ring) + tid * 16;
  auto issue = [&](int s) {
    if (s < s1) {
      const uint32_t dst = mine + (uint32_t)((s - s0) % SLOTS) * (R * S_STEP_BYTES);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int k = s * KSTEP + warp_k * 64 + j * 32, bytes = min(16, max(0, 2 * (q.k - k - tg * 8)));
        const int at = bytes > 0 ? k : 0;
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + (uint32_t)((2 * r + e) * 2 + j) * S_THREADS * 16),
                         "l"(w[r][e] + at), "r"((has >> (2 * r + e)) & 1u ? bytes : 0)
                         : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < SLOTS; ++i) issue(s0 + i);
  if (!GATE_UP) asm volatile("griddepcontrol.wait;" ::: "memory");     // the weights are on their way; h is the kernel before's

  const __nv_bfloat16* const in = q.in + (size_t)g * q.in_ld + warp_k * 64 + tg * 8;
  auto load_tokens = [&](int s, uint4 (*b)[2]) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int k = s * KSTEP + warp_k * 64 + j * 32 + tg * 8;
        b[n][j] = make_uint4(0, 0, 0, 0);
        if (s < s1 && 8 * n + g < q.T && k < q.k)
          b[n][j] = *reinterpret_cast<const uint4*>(in + (size_t)(8 * n) * q.in_ld + s * KSTEP + j * 32);
        if (!GATE_UP && k + 8 > q.k) b[n][j] = first_n(b[n][j], q.k - k);
      }
  };
  float acc[R][NT][4];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[r][n][i] = 0.f;
  uint4 b[NT][2], next[AHEAD ? NT : 1][2];
  if (AHEAD) load_tokens(s0, b);
  for (int s = s0; s < s1; ++s) {
    asm volatile("cp.async.wait_group %0;" ::"n"(SLOTS - 1) : "memory");
    const uint8_t* const at = few_ring + ((s - s0) % SLOTS) * (R * S_STEP_BYTES) + tid * 16;
    if constexpr (AHEAD) load_tokens(s + 1, next); else load_tokens(s, b);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      uint4 a[2][2];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int j = 0; j < 2; ++j) a[e][j] = *reinterpret_cast<const uint4*>(at + ((2 * r + e) * 2 + j) * S_THREADS * 16);
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma16816(acc[r][n], a[0][j].x, a[1][j].x, a[0][j].y, a[1][j].y, b[n][j].x, b[n][j].y);
          mma16816(acc[r][n], a[0][j].z, a[1][j].z, a[0][j].w, a[1][j].w, b[n][j].z, b[n][j].w);
        }
    }
    issue(s + SLOTS);
    if constexpr (AHEAD) {
#pragma unroll
      for (int n = 0; n < NT; ++n) { b[n][0] = next[n][0]; b[n][1] = next[n][1]; }
    }
  }
  // acc[r][n][i]: weight row g (i < 2) or g + 8 of the warp's tile r, token 8 n + 2 tg + i % 2
  // every warp leaves its sums in its CTA's shared memory (the ring is empty by now); the CTAs of a cluster share the
  // adding up
  __syncthreads();
  float* const part = reinterpret_cast<float*>(few_ring);
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[(((warp_k * TILES + warp_r * R + r) * NT + n) * 4 + i) * 32 + lane] = acc[r][n][i];
  if (splits > 1) cluster_barrier(); else __syncthreads();
  const int share = TILES * NT * 2 * 32 / splits;
  for (int p = split * share + tid; p < (split + 1) * share; p += S_THREADS) {
    const int l = p & 31, i = (p >> 5) & 1, n = (p >> 6) % NT, t = (p >> 6) / NT;
    const float* const src = part + ((t * NT + n) * 4 + i) * 32 + l;
    float lo = 0.f, hi = 0.f;
    for (int c = 0; c < splits; ++c) {
      const uint32_t from = map_to_cta(smem_u32(src), (uint32_t)c);
#pragma unroll
      for (int k = 0; k < WK; ++k) {
        const int off = k * TILES * NT * 4 * 32;
        lo += splits > 1 ? ld_cluster_f32(from + 4 * off) : src[off];
        hi += splits > 1 ? ld_cluster_f32(from + 4 * (off + 2 * 32)) : src[off + 2 * 32];
      }
    }
    few_store<GATE_UP>(q, (blockIdx.x * TILES + t) * TILE + (l >> 2), 8 * n + 2 * (l & 3) + i, lo, hi);
  }
  if (splits > 1) cluster_barrier();        // nobody leaves while its sums are read
}

// ------------------------------------------------------------------------------------------------ host side
size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

struct FfnShape {
  int64_t T;
  int D, F, ld;
  long long fp;             // pitch of h, g, u, dg, du: d_ff rounded up to whole 128-byte rows
};

int check_ffn(const camera_ffn_t* f, int64_t T, FfnShape* s) {
  if (f == nullptr || T < 0 || f->d_model < 1 || f->d_ff < 1 || f->down_ld < 0) return CAMERA_ERR_INVALID_ARG;
  s->T = T; s->D = f->d_model; s->F = f->d_ff; s->ld = f->down_ld ? f->down_ld : f->d_ff;
  if (s->ld < s->F) return CAMERA_ERR_INVALID_ARG;
  if (s->D % 8 != 0 || s->ld % 8 != 0 || T > (1ll << 30) || s->D > (1 << 20) || s->ld > (1 << 20))
    return CAMERA_ERR_UNSUPPORTED_SHAPE;
  if (f->w_gate == nullptr || f->w_up == nullptr || f->w_down == nullptr) return CAMERA_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(f->w_gate) | reinterpret_cast<uintptr_t>(f->w_up) | reinterpret_cast<uintptr_t>(f->w_down)) & 15)
    return CAMERA_ERR_INVALID_ARG;
  s->fp = (s->F + 63) & ~63;
  return CAMERA_OK;
}

// `saved`: upper halves of G and U, [T][2 fp] 16-bit (a row holds G, then U), then their lower bytes, [T][2 fp].
size_t saved_lo_offset(const FfnShape& s) { return up256((size_t)4 * s.T * s.fp + 1); }

constexpr int FEW_TOKENS = 64;     // up to here the streaming kernels

// Columns per B tile and B tiles per work unit: the choice with the least estimated time, rounds of units over the pairs
// times a unit's time.  Measured per k block (us): 0.60 for 512 columns, of which the products alone take 0.54 at
// 1.9 GHz; 0.43 for one tile of 256, 0.40 for two of 128; 0.39 for two and 0.32 for one tile of up to 128 columns, where
// the issue of the MMAs bounds it.  So 512 columns give the
// highest rate, and fewer give more units where 512 would leave pairs idle.  `epilogue` (us): what a unit of 512 columns,
// whose accumulators fill tensor memory, adds after its last k block; smaller units have two sets and overlap it.  (8192
// tokens, d_model 3584, d_ff 2560: dX with 512 columns 231 us, with 256 241 us; 4096 tokens, d_ff 20480: dH with 256
// columns 650 us, with 512 970 us, whose epilogue reads and writes 12 bytes an element.)
// max_splits > 1: the sum over k may also be cut into parts of their own units, whose fp32 sums a second kernel adds up
// (4 us and their bytes): with few tiles and a long k, pairs would idle through it.
struct Tile { int bn, nb, splits; };
Tile choose_tile(long long m_tiles, int n, bool dual, int min_bn, int n_kb, double epilogue, int max_splits, double part_bytes, int n_pairs) {
  Tile best{256, 2, 1};
  double best_cost = 1e300;
  for (int splits = 1; splits <= max_splits && 4 * splits <= n_kb + 3; ++splits)
    for (int bn = 256; bn >= min_bn; bn >>= 1)
      for (int nb = 2; nb >= (dual ? 2 : 1); --nb) {
        const int cols = nb * bn, per = dual ? bn : cols;
        const long long units = m_tiles * ((n + per - 1) / per) * splits;
        const double k_block = cols >= 512 ? 0.60 : bn >= 256 ? 0.43 : cols >= 256 ? 0.40 : nb == 2 ? 0.39 : 0.32;
        const double join = splits > 1 ? 4.0 + splits * 2.0 * part_bytes / 5.0e6 : 0.0;
        const double cost = (double)((units + n_pairs - 1) / n_pairs) * ((n_kb + splits - 1) / splits * k_block + (cols >= 512 ? epilogue : 1.0)) + join;
        if (cost < best_cost * 0.99) { best = Tile{bn, nb, splits}; best_cost = cost; }
      }
  return best;
}

// The tiles of y (one segment of k) and of dX (two).  room: bytes for the fp32 sums [T][d_model] of the parts of a split k.
constexpr int MAX_PARTS = 8;
Tile out_tile(const FfnShape& s, bool dx, int n_pairs, size_t room) {
  const int n_kb = (dx ? 2 : 1) * ((s.F + UMMA_BK - 1) / UMMA_BK);
  const size_t fit = room / ((size_t)4 * s.T * s.D);
  return choose_tile((s.T + G_TILE_M - 1) / G_TILE_M, s.D, false, dx ? 128 : 32, n_kb, 3.0, fit < MAX_PARTS ? (fit > 1 ? (int)fit : 1) : MAX_PARTS,
                     4.0 * s.T * s.D, n_pairs);
}

// What a call cannot do without grows with tokens and d_ff; the parts of a split k, which a smaller call may want more
// of, come last and take what room there is.  So a workspace of the query's size serves every smaller call.
struct FfnLayout { size_t h, dg, part, total; };     // dg: its rows hold dU behind dG; total: with all the parts wanted
FfnLayout ffn_layout(const FfnShape& s, bool backward) {
  FfnLayout l;
  const size_t act = up256((size_t)2 * s.T * s.fp);
  l.h = up256(sizeof(PlanTotals));
  l.dg = l.h + act;
  l.part = l.dg + (backward ? 2 * act : 0);
  const int n_pairs = sm_count() / 2;
  int parts = 0;
  if (s.T > FEW_TOKENS) parts = out_tile(s, false, n_pairs, ~(size_t)0).splits;
  if (backward && s.T > 0) {
    const int dx = out_tile(s, true, n_pairs, ~(size_t)0).splits;
    if (dx > parts) parts = dx;
  }
  l.total = l.part + (parts > 1 ? up256((size_t)4 * parts * s.T * s.D) : 0);
  return l;
}

bool enc(CUtensorMap* out, const void* p, long long rows, long long cols, long long pitch, int box_rows) {
  return encode_bf16_2d_pitch(out, p, (uint64_t)rows, (uint64_t)cols, (uint64_t)pitch, (uint32_t)box_rows);
}

template <int MODE>
cudaError_t launch_gemm(FfnGemm& q, Tile t, int n_pairs, bool first, cudaStream_t st) {
  q.bn = t.bn; q.nb = t.nb; q.splits = t.splits;
  q.clear_status = first;
  q.n_acc = t.nb * t.bn <= 256 ? 2 : 1;
  // A stage costs the issuing thread about 400 cycles beside the MMAs of its k blocks (wait, fence, commit), and a k block
  // of up to 256 columns 409 to 512 cycles of the tensor pipe, which holds too few MMAs to bridge that: such tiles get
  // two k blocks per stage (256 x 128 tile, K 4096, one unit per pair: 0.42 -> 0.31 us per k block).
  q.kps = t.nb * t.bn <= 256 ? 2 : 1;
  const int stage = q.kps * (G_A_BYTES + t.nb * t.bn * 64);
  q.n_stages = G_RING_BYTES / stage < G_MAX_STAGES ? G_RING_BYTES / stage : G_MAX_STAGES;
  int units = 0;
  for (int p = 0; p < q.n_prob; ++p) {
    const int per = MODE == FFN_GATE_UP ? t.bn : t.nb * t.bn;
    q.prob[p].n_tiles = (q.prob[p].n + per - 1) / per;
    q.prob[p].unit0 = units;
    units += ((q.prob[p].m + G_TILE_M - 1) / G_TILE_M) * q.prob[p].n_tiles;
  }
  q.tiles = units;
  units *= t.splits;
  q.n_units = units;
  cudaError_t e = allow_smem<k_ffn_gemm<MODE>, G_SMEM_BYTES>();
  if (e != cudaSuccess) return e;
  const int pairs = units < n_pairs ? units : n_pairs;
  e = launch_chained(k_ffn_gemm<MODE>, q, 2 * pairs, 1, 1, G_THREADS, G_SMEM_BYTES, !first, st);
  if (e != cudaSuccess || t.splits == 1) return e;
  const long long threads = ((long long)q.prob[0].m * q.prob[0].n + 7) / 8;
  return launch_chained(k_ffn_join, q, (int)((threads + 255) / 256), 1, 1, 256, 0, true, st);
}

template <bool GATE_UP, int WK, int R, int NT, int SLOTS, int CTAS>
cudaError_t launch_few_as(const FfnFew& q, cudaStream_t st) {
  constexpr int SMEM = SLOTS * R * S_STEP_BYTES, ROWS = (GATE_UP ? 8 : 16) * S_WARPS / WK * R;
  static_assert(SMEM >= S_WARPS * R * NT * 4 * 32 * 4, "the warps' sums take the ring's room");
  const cudaError_t e = allow_smem<k_ffn_few<GATE_UP, WK, R, NT, SLOTS, CTAS>, SMEM>();
  if (e != cudaSuccess) return e;
  const int row_ctas = (q.rows + ROWS - 1) / ROWS, steps = (q.k + 64 * WK - 1) / (64 * WK);
  // split k over a cluster until there is a CTA per SM or a CTA has fewer steps than its ring
  int splits = 1;
  while (splits < 8 && row_ctas * splits < sm_count() && steps >= splits * SLOTS) splits *= 2;
  return launch_chained(k_ffn_few<GATE_UP, WK, R, NT, SLOTS, CTAS>, q, row_ctas, splits, splits, S_THREADS, SMEM, !GATE_UP, st);
}
template <bool GATE_UP>
cudaError_t launch_few(const FfnFew& q, cudaStream_t st) {
  const int nt = (q.T + 7) / 8;
  if (nt <= 1) return launch_few_as<GATE_UP, 8, 1, 1, 4, 3>(q, st);
  if (nt <= 2) return launch_few_as<GATE_UP, 8, 2, 2, 3, 2>(q, st);
  if (nt <= 3) return launch_few_as<GATE_UP, 8, 2, 3, 3, 2>(q, st);
  if (nt <= 4) return launch_few_as<GATE_UP, 8, 2, 4, 3, 2>(q, st);
  if (nt <= 6) return launch_few_as<GATE_UP, 4, 1, 6, 6, 2>(q, st);
  return launch_few_as<GATE_UP, 4, 1, 8, 6, 2>(q, st);
}

#define FFN_CK(expr)                               \
  do {                                             \
    if ((expr) != cudaSuccess) {                   \
      cudaGetLastError();                          \
      return CAMERA_ERR_CUDA;                      \
    }                                              \
  } while (0)

}  // namespace
}  // namespace camera

extern "C" size_t camera_ffn_workspace_bytes(const camera_ffn_t* f, int64_t n_tokens, int32_t backward) {
  camera::FfnShape s;
  if (camera::check_ffn(f, n_tokens, &s) != CAMERA_OK) return 0;
  return camera::ffn_layout(s, backward != 0).total;
}

extern "C" size_t camera_ffn_saved_bytes(const camera_ffn_t* f, int64_t n_tokens) {
  camera::FfnShape s;
  if (camera::check_ffn(f, n_tokens, &s) != CAMERA_OK) return 0;
  return camera::saved_lo_offset(s) + camera::up256((size_t)2 * s.T * s.fp + 1);
}

extern "C" int camera_ffn_forward(const camera_ffn_t* f, const void* x, int64_t n_tokens, void* y, void* saved,
                                  void* workspace, size_t workspace_bytes, void* cuda_stream) {
  using namespace camera;
  FfnShape s;
  const int rc = check_ffn(f, n_tokens, &s);
  if (rc != CAMERA_OK) return rc;
  const FfnLayout l = ffn_layout(s, false);
  if (workspace == nullptr || workspace_bytes < l.part || (reinterpret_cast<uintptr_t>(workspace) & 255)) return CAMERA_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* const ws = static_cast<char*>(workspace);
  if (n_tokens > 0 && (x == nullptr || y == nullptr || ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y)) & 15) ||
                       (reinterpret_cast<uintptr_t>(saved) & 31)))
    return CAMERA_ERR_INVALID_ARG;
  if (n_tokens > 0 && n_tokens <= FEW_TOKENS) {
    FfnFew w;
    w.w0 = static_cast<const __nv_bfloat16*>(f->w_gate); w.w1 = static_cast<const __nv_bfloat16*>(f->w_up);
    w.in = static_cast<const __nv_bfloat16*>(x);
    w.w_ld = s.D; w.in_ld = s.D; w.out_ld = s.fp;
    w.rows = s.F; w.k = s.D; w.T = (int)s.T;
    w.out = reinterpret_cast<__nv_bfloat16*>(ws + l.h);
    w.g = static_cast<uint16_t*>(saved); w.u_off = s.fp; w.lo_off = (long long)saved_lo_offset(s); w.act_ld = 2 * s.fp;
    w.totals = reinterpret_cast<PlanTotals*>(ws);
    FFN_CK(launch_few<true>(w, st));
    w.w0 = w.w1 = static_cast<const __nv_bfloat16*>(f->w_down);
    w.in = w.out; w.out = static_cast<__nv_bfloat16*>(y);
    w.w_ld = s.ld; w.in_ld = s.fp; w.out_ld = s.D; w.rows = s.D; w.k = s.F;
    w.g = nullptr; w.totals = nullptr;
    FFN_CK(launch_few<false>(w, st));
    return CAMERA_OK;
  }
  if (n_tokens == 0) {
    FFN_CK(cudaMemsetAsync(ws, 0, sizeof(PlanTotals), st));
    return CAMERA_OK;
  }
  const int n_pairs = sm_count() / 2;
  const long long m_tiles = (s.T + G_TILE_M - 1) / G_TILE_M;
  FfnGemm q;
  memset(&q, 0, sizeof(q));
  q.totals = reinterpret_cast<PlanTotals*>(ws);
  q.wait_limit_ns = current_wait_limit_ns();
  q.h = reinterpret_cast<__nv_bfloat16*>(ws + l.h);
  q.h_ld = s.fp;
  q.part = reinterpret_cast<float*>(ws + l.part);
  q.act_ld = 2 * s.fp;
  q.g = static_cast<uint16_t*>(saved);
  q.u = saved ? q.g + s.fp : nullptr;
  q.lo_off = (long long)saved_lo_offset(s);
  q.n_prob = 1;
  q.prob[0] = FfnProblem{(int)s.T, s.F, 0, 0, nullptr, 0};
  q.n_kb = (s.D + UMMA_BK - 1) / UMMA_BK;
  Tile t = choose_tile(m_tiles, s.F, true, 32, q.n_kb, saved ? 6.0 : 3.0, 1, 0.0, n_pairs);
  if (!enc(&q.a[0], x, s.T, s.D, s.D, 128) || !enc(&q.b[0], f->w_gate, s.F, s.D, s.D, t.bn / 2) ||
      !enc(&q.b[1], f->w_up, s.F, s.D, s.D, t.bn / 2))
    return CAMERA_ERR_CUDA;
  FFN_CK(launch_gemm<FFN_GATE_UP>(q, t, n_pairs, true, st));
  q.prob[0] = FfnProblem{(int)s.T, s.D, 0, 0, static_cast<__nv_bfloat16*>(y), s.D};
  q.n_kb = (s.F + UMMA_BK - 1) / UMMA_BK;
  t = out_tile(s, false, n_pairs, workspace_bytes - l.part);
  if (!enc(&q.a[0], q.h, s.T, s.F, s.fp, 128) || !enc(&q.b[0], f->w_down, s.D, s.F, s.ld, t.bn / 2)) return CAMERA_ERR_CUDA;
  FFN_CK(launch_gemm<FFN_DOWN>(q, t, n_pairs, false, st));
  return CAMERA_OK;
}

extern "C" int camera_ffn_backward(const camera_ffn_t* f, const void* x, const void* dy, int64_t n_tokens, const void* saved,
                                   void* dx, void* dw_gate, void* dw_up, void* dw_down, void* workspace,
                                   size_t workspace_bytes, void* cuda_stream) {
  using namespace camera;
  FfnShape s;
  const int rc = check_ffn(f, n_tokens, &s);
  if (rc != CAMERA_OK) return rc;
  const FfnLayout l = ffn_layout(s, true);
  if (workspace == nullptr || workspace_bytes < l.part || (reinterpret_cast<uintptr_t>(workspace) & 255)) return CAMERA_ERR_WORKSPACE;
  const bool weights = dw_gate != nullptr;
  if ((dw_up != nullptr) != weights || (dw_down != nullptr) != weights || (!weights && dx == nullptr)) return CAMERA_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(dw_gate) | reinterpret_cast<uintptr_t>(dw_up) | reinterpret_cast<uintptr_t>(dw_down)) & 15)
    return CAMERA_ERR_INVALID_ARG;
  if (n_tokens > 0 && (x == nullptr || dy == nullptr || saved == nullptr || (reinterpret_cast<uintptr_t>(saved) & 31) ||
                       ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(dy) | reinterpret_cast<uintptr_t>(dx)) & 15)))
    return CAMERA_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* const ws = static_cast<char*>(workspace);
  if (n_tokens == 0) {                          // sums over no token
    FFN_CK(cudaMemsetAsync(ws, 0, sizeof(PlanTotals), st));
    if (weights) {
      FFN_CK(cudaMemsetAsync(dw_gate, 0, (size_t)2 * s.F * s.D, st));
      FFN_CK(cudaMemsetAsync(dw_up, 0, (size_t)2 * s.F * s.D, st));
      FFN_CK(cudaMemset2DAsync(dw_down, (size_t)2 * s.ld, 0, (size_t)2 * s.F, (size_t)s.D, st));
    }
    return CAMERA_OK;
  }
  const int n_pairs = sm_count() / 2;
  const long long m_tiles = (s.T + G_TILE_M - 1) / G_TILE_M;
  FfnGemm q;
  memset(&q, 0, sizeof(q));
  q.totals = reinterpret_cast<PlanTotals*>(ws);
  q.wait_limit_ns = current_wait_limit_ns();
  q.h = reinterpret_cast<__nv_bfloat16*>(ws + l.h);
  q.h_ld = s.fp;
  q.part = reinterpret_cast<float*>(ws + l.part);
  q.act_ld = 2 * s.fp;          // dg and du share rows in the workspace as G and U do in `saved`
  q.g = static_cast<uint16_t*>(const_cast<void*>(saved));
  q.u = q.g + s.fp;
  q.lo_off = (long long)saved_lo_offset(s);
  q.dg = reinterpret_cast<__nv_bfloat16*>(ws + l.dg);
  q.du = q.dg + s.fp;
  // dH and its element-wise part
  q.n_prob = 1;
  q.prob[0] = FfnProblem{(int)s.T, s.F, 0, 0, nullptr, 0};
  q.n_kb = (s.D + UMMA_BK - 1) / UMMA_BK;
  Tile t = choose_tile(m_tiles, s.F, false, 128, q.n_kb, 20.0, 1, 0.0, n_pairs);
  if (!enc(&q.a[0], dy, s.T, s.D, s.D, 128) || !enc(&q.b[0], f->w_down, s.D, s.F, s.ld, 64)) return CAMERA_ERR_CUDA;
  FFN_CK(launch_gemm<FFN_DH>(q, t, n_pairs, true, st));
  if (weights) {               // before dx, which may take the room of x or dy
    q.n_prob = 3;
    q.prob[0] = FfnProblem{s.F, s.D, 0, 0, static_cast<__nv_bfloat16*>(dw_gate), s.D};
    q.prob[1] = FfnProblem{s.F, s.D, 0, 0, static_cast<__nv_bfloat16*>(dw_up), s.D};
    q.prob[2] = FfnProblem{s.D, s.F, 0, 0, static_cast<__nv_bfloat16*>(dw_down), s.ld};
    q.n_kb = (int)((s.T + UMMA_BK - 1) / UMMA_BK);
    // the third problem has as many tiles as either of the others, up to their edges
    t = choose_tile(3ll * ((s.F + G_TILE_M - 1) / G_TILE_M), s.D, false, 128, q.n_kb, 3.0, 1, 0.0, n_pairs);
    if (!enc(&q.a[0], q.dg, s.T, s.F, q.act_ld, 64) || !enc(&q.a[1], q.du, s.T, s.F, q.act_ld, 64) ||
        !enc(&q.a[2], dy, s.T, s.D, s.D, 64) || !enc(&q.b[0], x, s.T, s.D, s.D, 64) || !enc(&q.b[2], q.h, s.T, s.F, s.fp, 64))
      return CAMERA_ERR_CUDA;
    q.b[1] = q.b[0];
    FFN_CK(launch_gemm<FFN_DW>(q, t, n_pairs, false, st));
  }
  if (dx != nullptr) {
    q.n_prob = 1;
    q.prob[0] = FfnProblem{(int)s.T, s.D, 0, 0, static_cast<__nv_bfloat16*>(dx), s.D};
    q.n_kb = (s.F + UMMA_BK - 1) / UMMA_BK;
    t = out_tile(s, true, n_pairs, workspace_bytes - l.part);
    if (!enc(&q.a[0], q.dg, s.T, s.F, q.act_ld, 128) || !enc(&q.a[1], q.du, s.T, s.F, q.act_ld, 128) ||
        !enc(&q.b[0], f->w_gate, s.F, s.D, s.D, 64) || !enc(&q.b[1], f->w_up, s.F, s.D, s.D, 64))
      return CAMERA_ERR_CUDA;
    FFN_CK(launch_gemm<FFN_DX>(q, t, n_pairs, false, st));
  }
  return CAMERA_OK;
}
