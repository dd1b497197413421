/*
 * camera.h — C ABI of the B200 (sm_100a) CAMERA micro-expert analysis library.
 *
 * The library computes, for one Mixture-of-Experts layer and a batch of
 * calibration tokens, the per-micro-expert energy of the CAMERA paper and the
 * two structured selections driven by it.  A micro-expert is intermediate
 * channel i of an expert: row i of W_gate and W_up plus column i of W_down
 * (paper Eq. 3).  Experts are ordered routed[0..n_routed) then
 * shared[0..n_shared); the global micro-expert index is off[e] + i with off the
 * prefix sum of d_ff (Algorithm 1's global index, generalised to unequal d_ff).
 *
 * General rules
 *  - "DEVICE" pointers are CUDA device memory of the current device, "HOST"
 *    pointers ordinary host memory.  The caller owns every buffer.  The
 *    library allocates no device memory: scratch comes from the caller's
 *    workspace (query the *_workspace_bytes function first; 256-byte aligned).
 *  - Calls enqueue work on `cuda_stream` (a cudaStream_t, NULL = default
 *    stream) and return without synchronising unless stated otherwise.
 *    HOST arrays passed in are consumed before the call returns.
 *  - Return value: CAMERA_OK or a negative camera_status_t.  Argument errors
 *    are reported before anything is launched.  Device-side trouble (a bounded
 *    wait inside a kernel that ran out) never traps: it is recorded in the
 *    workspace's status word, see camera_read_status.
 *  - No call is re-entrant on the same workspace: calls that share a workspace
 *    and overlap on the GPU race.
 */
#ifndef CAMERA_B200_H
#define CAMERA_B200_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  CAMERA_OK = 0,
  CAMERA_ERR_INVALID_ARG = -1,
  CAMERA_ERR_UNSUPPORTED_SHAPE = -2,
  CAMERA_ERR_WORKSPACE = -3,
  CAMERA_ERR_ARCH = -4,
  CAMERA_ERR_CUDA = -5,
  CAMERA_ERR_DEVICE_TIMEOUT = -6
} camera_status_t;

typedef enum { CAMERA_F32 = 0, CAMERA_BF16 = 1 } camera_dtype_t;

/* Storage of one expert's W_down: CAMERA_DOWN_HF is the paper's [d_model, d_ff]
 * (micro-expert i = column i); CAMERA_DOWN_ME_MAJOR is [d_ff, d_model] (row i). */
typedef enum { CAMERA_DOWN_HF = 0, CAMERA_DOWN_ME_MAJOR = 1 } camera_down_layout_t;

/* camera_layer_t.flags */
enum {
  CAMERA_ROUTER_NORM_TOPK = 1u,    /* divide the k kept probabilities by their sum ("Top&Norm") */
  CAMERA_SHARED_GATE_SIGMOID = 2u  /* shared expert s gets coefficient sigmoid(x . w_shared_gate[s]) instead of 1 */
};

/* camera_score_aux_t.flags */
enum {
  CAMERA_SCORE_FORCE_SIMT = 1u,    /* run the fp32-FMA kernels even where the tensor-core kernels apply */
  CAMERA_SCORE_CTA_PAIR = 2u,      /* force tensor-core scoring on CTA pairs (tcgen05 cta_group::2, 256 micro-experts per
                                      work unit: less L2 and shared-memory traffic per flop).  By default the library takes
                                      pairs unless padding d_ff to multiples of 256 would add more than 6 % of work */
  CAMERA_SCORE_SINGLE_CTA = 8u,    /* force one CTA per MMA (128 micro-experts per work unit) */
  CAMERA_SCORE_OMEGA_GIVEN = 32u,  /* omega2 (required) already holds ||w_i||^2 of this layer's W_down, e.g. from the call on
                                      the first batch of tokens: the pass over W_down is skipped */
  CAMERA_FORWARD_TOKEN_ROWS = 16u, /* camera_layer_forward only: force the gate/up kernel that keeps the tokens on the
                                      accumulator rows (CTA pairs, 256-token tiles; an epilogue thread writes runs of
                                      consecutive micro-experts of its token).  By default the library takes it when
                                      the experts' token lists are long enough for whole 256-token tiles to cost no
                                      more than they save; CTA_PAIR / SINGLE_CTA force the scoring orientation */
  CAMERA_SCORE_SINGLE_PASS = 64u,  /* camera_score_layer only: score all n_tokens in one pass even when they are more than
                                      65536 (needs camera_score_workspace_bytes_single_pass bytes of scratch) instead of
                                      walking them in batches of 65536; the two differ in the last bits of the energies
                                      (the batches' sums are rounded to fp32 between batches) */
  CAMERA_SCORE_ACCUMULATE = 4u     /* phi2 and phi_inf_sq (both required) already hold the result of earlier batches of
                                      calibration tokens of this layer; this call folds its batch in (the column sums of
                                      Algorithm 1 add up over batches, the column maxima take the maximum)
                                      and writes the energy of all batches so far; the workspace's status word is
                                      not cleared by such a call, so one camera_read_status after the last batch
                                      reports trouble in any of them (use the same workspace for all batches) */
};

/* Stages of camera_score_layer, for the optional timing events. */
enum {
  CAMERA_STAGE_ROUTER = 0, CAMERA_STAGE_PERMUTE = 1, CAMERA_STAGE_ROWNORM = 2,
  CAMERA_STAGE_SCORE = 3, CAMERA_STAGE_COMBINE = 4, CAMERA_N_STAGES = 5
};

/* What camera_layer_prepare keeps for a layer (opaque). */
typedef struct camera_prepared camera_prepared_t;

/* One MoE layer (paper Algorithm 1 inputs: expert weights and router R). */
typedef struct {
  int32_t d_model;              /* multiple of 8 */
  int32_t n_routed;             /* 0..256 routed experts */
  int32_t top_k;                /* 1..min(n_routed,16); ignored when n_routed == 0 */
  int32_t n_shared;             /* experts every token visits */
  const int32_t* d_ff;          /* HOST [n_routed+n_shared], each > 0 */
  int32_t dtype;                /* camera_dtype_t of x and of every weight */
  uint32_t flags;
  int32_t down_layout;          /* camera_down_layout_t */
  const void* w_router;         /* DEVICE [n_routed, d_model] row-major */
  const float* router_bias;     /* DEVICE [n_routed] fp32 added to the logits, or NULL */
  const void* w_shared_gate;    /* DEVICE [n_shared, d_model]; required iff CAMERA_SHARED_GATE_SIGMOID */
  const void* const* w_gate;    /* HOST array of DEVICE pointers, each [d_ff[e], d_model] row-major */
  const void* const* w_up;      /* same */
  const void* const* w_down;    /* each per down_layout */
  const int32_t* w_down_ld;     /* HOST [n_routed+n_shared] or NULL: leading dimension (elements) of each W_down in
                                   CAMERA_DOWN_HF layout when its rows are longer than d_ff[e] (a sliced layer kept in
                                   buffers of the original width); multiples of 8; NULL = d_ff[e] */
  const camera_prepared_t* prepared; /* NULL, or the handle camera_layer_prepare returned for exactly this layer */
} camera_layer_t;

/* Optional inputs/outputs of camera_score_layer; any pointer may be NULL. All DEVICE. */
typedef struct {
  float* phi2;                  /* [N_e]  ||Phi_i||_2^2       (Alg. 1, ColumnSum) */
  float* phi_inf_sq;            /* [N_e]  ||Phi_i||_inf^2     (Alg. 1, ColumnMax) */
  float* omega2;                /* [N_e]  ||w_i||_2^2         (Alg. 1, omega) */
  int32_t* topk_idx;            /* [T, top_k] chosen experts, by decreasing probability */
  float* topk_w;                /* [T, top_k] their coefficients A */
  const int32_t* topk_idx_in;   /* if both *_in are set the router is skipped and this routing is used */
  const float* topk_w_in;
  float* shared_w;              /* [n_shared, T] coefficients of the shared experts */
  int32_t* expert_token_counts; /* [n_routed+n_shared] tokens each expert saw */
  uint32_t flags;               /* CAMERA_SCORE_* */
  void* stage_events[2 * CAMERA_N_STAGES]; /* cudaEvent_t pairs (begin,end) recorded around each stage, or NULL */
} camera_score_aux_t;

const char* camera_strerror(int status);
int camera_version(void);

/*
 * Optional: what does not change from call to call, built once.  Without a handle every scoring / forward call
 * builds the layer's expert table and encodes 2 tensor maps per expert on the host and copies them to the workspace
 * (from pageable memory); a 64-token decode step through camera_layer_forward pays that each time.  With
 * layer->prepared set, those live in device memory the handle owns, and the few tensor maps that name the call's
 * tokens or workspace are rebuilt only when (workspace, x, n_tokens) differ from the previous call's, and then travel
 * as kernel arguments: a repeated call enqueues memsets and kernels only.  The paper has no counterpart.
 *
 * device_mem: DEVICE, camera_layer_prepared_bytes(layer) bytes, 256-byte aligned, owned by the handle until
 * camera_layer_release (nothing else may write there).  The layer's matrices must stay where they are while the handle
 * lives; a layer_t that differs from the one prepared (another pointer, shape or flag) is refused with
 * CAMERA_ERR_INVALID_ARG.  The call synchronises `cuda_stream` once.  Calls that share a handle must be ordered on the
 * GPU (one stream, or events) and come from one host thread at a time, like calls that share a workspace.
 * Results are bit-identical with and without a handle.
 */
size_t camera_layer_prepared_bytes(const camera_layer_t* layer);
int camera_layer_prepare(const camera_layer_t* layer, void* device_mem, size_t device_bytes, void* cuda_stream,
                         camera_prepared_t** prepared_out);
void camera_layer_release(camera_prepared_t* prepared);

/* Scratch needed by camera_score_layer for this layer shape and token count (0 on invalid arguments).  Token sets
 * longer than 65536 are walked in batches of 65536 through the scratch of one batch, so the size stops growing there
 * (3.8 GiB at the Qwen2-57B-A14B shape); camera_score_workspace_bytes_single_pass is the size CAMERA_SCORE_SINGLE_PASS
 * needs (14.4 GiB for 262144 tokens of that shape). */
size_t camera_score_workspace_bytes(const camera_layer_t* layer, int64_t n_tokens);
size_t camera_score_workspace_bytes_single_pass(const camera_layer_t* layer, int64_t n_tokens);

/*
 * Algorithm 1 of the paper (micro-expert ranking) up to and including the energies:
 *   A      <- Top&Norm(softmax(R x))
 *   omega2 <- ColumnSum(W_down * W_down)
 *   Lambda <- A[:,e] * SiLU(W_gate X) * (W_up X)                   (never stored)
 *   phi2   <- ColumnSum(Lambda*Lambda), phi_inf <- ColumnMax|Lambda|^2
 *   energy <- [(1-alpha) phi2 + alpha phi_inf] * omega2            Eq. 11
 * x: DEVICE [n_tokens, d_model] row-major, dtype layer->dtype.  energy: DEVICE [N_e] fp32.
 * The calibration set may be fed in several calls (batches of tokens) with CAMERA_SCORE_ACCUMULATE; a single call
 * with more than 65536 tokens walks them in batches of 65536 itself (same arithmetic as such calls; the batches
 * depend on n_tokens alone, so a given input gives the same bits every time; aux->stage_events then bracket the
 * stages of the last batch) unless CAMERA_SCORE_SINGLE_PASS asks for one pass.
 * Arithmetic: inputs as stored, products and sums in fp32 (bf16: tensor cores with fp32
 * accumulators), the final blend in fp64.  Routing ties go to the lower expert index.
 * An expert no token reaches gets energy 0.  0 <= alpha <= 1.  n_tokens >= 0.
 * The bf16 tensor-core path needs d_model % 64 == 0; other shapes (and fp32) run the fp32-FMA
 * kernel.
 */
int camera_score_layer(const camera_layer_t* layer, const void* x, int64_t n_tokens, float alpha,
                       float* energy, const camera_score_aux_t* aux,
                       void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Synchronises the stream, reads the workspace's status word (0 = fine, else a
 * camera_status_t recorded by a kernel) into *status_out and clears nothing.
 * Kernels record CAMERA_ERR_DEVICE_TIMEOUT (a bounded wait ran out), CAMERA_ERR_INVALID_ARG (a
 * token's routing cannot be used: a prescribed expert index out of range or named twice by one
 * token, or no finite softmax because x or the router holds a NaN or an infinity; such a token
 * is given coefficient 0 everywhere, so the call still finishes and every index stays in range)
 * and CAMERA_ERR_WORKSPACE (the token lists outgrew a workspace smaller than the query's size). */
int camera_read_status(const void* workspace, void* cuda_stream, int32_t* status_out);

/*
 * Limit of the waits inside the tensor-core kernels (a thread that waits for a copy or for
 * another warp gives up after this long, the kernel records CAMERA_ERR_DEVICE_TIMEOUT and
 * returns normally), and of the waits between CTAs that share a row of logits.  Process wide, read by every later call; 4 s unless set.  1 us .. 600 s,
 * else CAMERA_ERR_INVALID_ARG.  The paper has no counterpart: this is the library's error
 * convention (device-side trouble surfaces through the status word, never as a trap or a hang).
 */
int camera_set_wait_limit_ns(uint64_t limit_ns);
uint64_t camera_get_wait_limit_ns(void);

/*
 * Self-test of that convention: launches one small CTA whose threads wait, with the library's
 * bounded wait, on a barrier that nothing arrives on.  After limit_ns (1 us .. 1 s) the wait runs
 * out, the kernel writes CAMERA_ERR_DEVICE_TIMEOUT into the status word of `workspace` (cleared
 * first; at least 256 bytes, 256-byte aligned) and returns; camera_read_status then reports it.
 * Nothing else on the device is touched and the context stays usable.
 */
int camera_wait_probe(void* workspace, size_t workspace_bytes, uint64_t limit_ns, void* cuda_stream);

/* Scratch for camera_select_prune / camera_alloc_bits (n_levels = 2 for pruning), 256-byte aligned.  The selection
 * is one kernel whose CTAs meet at counters in this scratch (launched cooperatively, so that they are resident
 * together); its waits are bounded like those of the scoring kernels and report through the scratch's status word,
 * which camera_read_status reads like a scoring workspace's. */
size_t camera_select_workspace_bytes(int64_t n_total, int32_t n_segments, int32_t n_levels);

/*
 * CAMERA-P selection (Algorithm 2, S <- TopSelect(R, 1 - lambda)), for one or many
 * layers at once.  energy: DEVICE [n_total] fp32, non-negative.  seg_offsets: HOST
 * [n_segments+1] increasing, seg_offsets[0] = 0, last = n_total; one segment = one layer.  In
 * every segment of n elements the floor(prune_ratio * n + 1e-9) lowest-energy micro-experts get
 * keep_mask = 0, all others 1; among equal energies the lower index is pruned first.
 * 0 <= prune_ratio < 1.  Optional: expert_offsets DEVICE int64 [n_experts_total+1] (global
 * micro-expert offsets) with kept_per_expert DEVICE [n_experts_total]; thresholds DEVICE
 * [n_segments] receives the energy of the lowest retained micro-expert.
 */
int camera_select_prune(const float* energy, const int64_t* seg_offsets, int32_t n_segments,
                        double prune_ratio, const int64_t* expert_offsets, int32_t n_experts_total,
                        uint8_t* keep_mask, int32_t* kept_per_expert, float* thresholds,
                        void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * CAMERA-Q class split (Algorithm 3: ListSplitByRatio + GetSubIndex).  ratios: HOST
 * [n_levels] (2..8 levels), most important class first, summing to 1; bits: HOST [n_levels]
 * bit-widths 0..255.  Within a segment of n elements ranked from highest to lowest energy
 * (equal energies: higher index first), class j takes ranks [c_{j-1}, c_j) with
 * c_j = floor((r_1+..+r_j) n + 1e-9) and c_L = n.  bits_out: DEVICE [n_total] uint8;
 * class_counts (optional, with expert_offsets): DEVICE [n_experts_total, n_levels].
 */
int camera_alloc_bits(const float* energy, const int64_t* seg_offsets, int32_t n_segments,
                      const double* ratios, const int32_t* bits, int32_t n_levels,
                      const int64_t* expert_offsets, int32_t n_experts_total,
                      uint8_t* bits_out, int32_t* class_counts,
                      void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Several CAMERA-P masks (Algorithm 2, TopSelect at several prune ratios) and the CAMERA-Q bit-widths (Algorithm 3,
 * ListSplitByRatio) of the same energies from one set of radix passes: every threshold is a rank of the same keys, so
 * the four histogram passes find them together and all outputs are written at the end of the same kernel (one launch
 * where the separate calls take one each).  The results are those of camera_select_prune / camera_alloc_bits, bit for bit.
 * prune_ratios: HOST [n_prune];  keep_masks: DEVICE uint8 [n_prune][N] (mask p at keep_masks + p * N, N =
 * seg_offsets[n_segments]);  ratios, bits, n_levels, bits_out as for camera_alloc_bits, bits_out may be NULL (no
 * bit-widths; ratios, bits, n_levels are then ignored).  n_prune + n_levels - 1 <= 7, else CAMERA_ERR_INVALID_ARG.
 * workspace: camera_select_workspace_bytes(N, n_segments, n_prune + n_levels) bytes.
 */
int camera_select_all(const float* energy, const int64_t* seg_offsets, int32_t n_segments, const double* prune_ratios,
                      int32_t n_prune, uint8_t* keep_masks, const double* ratios, const int32_t* bits, int32_t n_levels,
                      uint8_t* bits_out, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * camera_select_prune without a workspace argument (the paper has no counterpart; this exists for
 * the sake of integration).  Some hosts of this library may not create device allocations at all:
 * a plug-in inside a serving process whose memory pool already owns the whole GPU, a callback that
 * runs where cudaMalloc's implicit device-wide synchronisation is not acceptable, or code that is
 * simply not handed an allocator.  For them the scratch of the selection lives in a fixed array
 * inside the library image: 288 KiB of every GPU that loads the library, held until the process ends.
 *
 * Same arguments and results as camera_select_prune (energy, keep_mask, thresholds: DEVICE;
 * seg_offsets: HOST), minus the per-expert counts.  Limit: n_segments <= 32; more returns
 * CAMERA_ERR_UNSUPPORTED_SHAPE and launches nothing.  The call itself allocates nothing on the
 * device (no cudaMalloc / cudaFree, no allocating library routine).
 *
 * The first call on each device looks up the array's device address (the device must be current);
 * make that first call outside of any stream capture.  All calls on a device share the one array
 * and each call overwrites what the previous one left there (the parts that have to start at zero
 * are cleared on the stream at the start of every call), so two calls that overlap on the GPU --
 * different streams, or different host threads -- race; issue them on one stream or order them with
 * events.
 */
int camera_select_prune_static(const float* energy, const int64_t* seg_offsets, int32_t n_segments,
                               double prune_ratio, uint8_t* keep_mask, float* thresholds,
                               void* cuda_stream);

/*
 * GetSubIndex (Algorithm 3; the per-expert retained sets S of Algorithm 2).
 * labels: DEVICE [N_e] uint8, one per micro-expert -- a keep mask of camera_select_prune, or the
 * bits_out of camera_alloc_bits.  expert_offsets: DEVICE int64 [n_experts+1], global micro-expert
 * offsets.  label_order: HOST [n_labels] (1..8 distinct values 0..255).  For every expert e the
 * channels (0 .. d_ff[e]-1) whose label is label_order[0] are written to
 * sub_index[expert_offsets[e] ...] in ascending order, followed by those of label_order[1], and
 * so on (a stable partition by label); micro-experts with any other label are left out and the
 * tail of the expert's segment is not written.  counts: DEVICE [n_experts, n_labels], how many
 * entries each label contributed.  With label_order = {1} on a keep mask the list is the retained
 * set; with every bit-width in label_order it is the reordering that puts micro-experts of equal
 * precision next to each other (Section "CAMERA-Q").
 */
int camera_sub_index(const uint8_t* labels, const int64_t* expert_offsets, int32_t n_experts,
                     const int32_t* label_order, int32_t n_labels, int32_t* sub_index, int32_t* counts,
                     void* cuda_stream);

/* Scratch for camera_compact_weights (256-byte aligned; it starts with a status word that camera_read_status reads:
 * the column gather waits, with the library's bounded wait, for the bulk copies that fill its tiles). */
size_t camera_compact_workspace_bytes(int32_t n_experts);

/*
 * The slicing step of Algorithm 2: W_up <- W_up[S,:], W_gate <- W_gate[S,:], W_down <- W_down[:,S], with S
 * the first m_e = counts[e,0] + .. + counts[e,n_take-1] entries of expert e's list in sub_index
 * (both as written by camera_sub_index; DEVICE).  w_gate_out / w_up_out / w_down_out: HOST arrays
 * of DEVICE pointers, one per expert, 16-byte aligned, with room for the worst case the caller
 * allows (d_ff[e] rows is always enough): row r of w_gate_out[e] receives row sub_index[r] of
 * w_gate[e], likewise w_up; W_down in CAMERA_DOWN_ME_MAJOR likewise; in CAMERA_DOWN_HF column j of
 * w_down_out[e] (a [d_model, down_ld[e]] matrix; down_ld HOST, NULL = d_ff[e]) receives column
 * sub_index[j].  Rows / columns from m_e on are not written.  Outputs must not overlap inputs.
 */
int camera_compact_weights(const camera_layer_t* layer, const int32_t* sub_index, const int32_t* counts,
                           int32_t n_labels, int32_t n_take, void* const* w_gate_out, void* const* w_up_out,
                           void* const* w_down_out, const int32_t* down_ld, void* workspace,
                           size_t workspace_bytes, void* cuda_stream);

/* Scratch for camera_layer_forward (holds the token lists, h and the per-expert output rows). */
size_t camera_forward_workspace_bytes(const camera_layer_t* layer, int64_t n_tokens);

/*
 * The layer's output, Eq. 1-2:  y_t = sum_e A_{t,e} W_down_e [ SiLU(W_gate_e x_t) * (W_up_e x_t) ],  with the
 * router coefficients A of camera_score_layer (aux: topk_idx_in / topk_w_in prescribe them, topk_idx / topk_w /
 * shared_w / expert_token_counts export them; flags CAMERA_SCORE_CTA_PAIR / CAMERA_SCORE_SINGLE_CTA /
 * CAMERA_FORWARD_TOKEN_ROWS force the gate/up kernel; other fields and flags are ignored).  Applied to a layer sliced by
 * camera_compact_weights it gives Y_hat = Phi[:,S] W[S,:], the retained micro-experts' output of Eq. 7.
 * x: DEVICE [n_tokens, d_model] bf16;  y: DEVICE [n_tokens, d_model] fp32, 16-byte aligned.
 * bf16 layers in CAMERA_DOWN_HF layout with d_model % 64 == 0 only (else CAMERA_ERR_UNSUPPORTED_SHAPE); d_ff[e] may
 * be any value >= 0 (an expert that lost every micro-expert contributes nothing), provided W_down rows start on
 * 16-byte boundaries: d_ff[e] % 8 == 0 or w_down_ld given.  Arithmetic: bf16 products with fp32 accumulation on
 * tensor cores, h rounded to bf16 between the two GEMMs, a token's k + n_shared expert outputs added in fp32 in a
 * fixed order.  Feed long calibration sets in batches: the workspace grows with n_tokens.
 */
int camera_layer_forward(const camera_layer_t* layer, const void* x, int64_t n_tokens, float* y,
                         const camera_score_aux_t* aux, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * The layer-output step and the scoring step of Algorithm 2's loop on one batch of tokens, from one pass over W_gate and W_up: the energies of
 * camera_score_layer (Algorithm 1: same alpha, energy, aux fields and flags, CAMERA_SCORE_ACCUMULATE included) and the
 * layer output y of camera_layer_forward (Eq. 1-2).  The gate/up GEMM runs once, in the scoring orientation; its
 * epilogue folds lambda into the per-micro-expert sums and maxima and stores it as h for the W_down GEMM.  The
 * energies are bit-identical to camera_score_layer's and y to camera_layer_forward's under the same kernel flags.
 * Arguments, layouts, restrictions and errors as for those two calls; energy must not be NULL (CAMERA_ERR_INVALID_ARG);
 * workspace: camera_forward_workspace_bytes.  With n_tokens == 0 only the energies are written.
 */
int camera_score_forward_layer(const camera_layer_t* layer, const void* x, int64_t n_tokens, float alpha, float* energy,
                               float* y, const camera_score_aux_t* aux, void* workspace, size_t workspace_bytes,
                               void* cuda_stream);

/*
 * The retained micro-experts' output Y_hat = Phi[:,S] W[S,:] (Eq. 7) without running the pruned layer again.  After
 * camera_score_forward_layer or camera_layer_forward the workspace still holds Phi as h (bf16) and the token lists;
 * once the selection S is known, Y_hat is h times W_down with the columns outside S set to zero: the W_down GEMM alone,
 * a third of the pruned layer's flops.  (The paper's loop, Algorithm 2, runs the pruned layer on the same input.)
 *
 * camera_mask_down_columns: w_down_out[e][r, i] = keep_mask[offset_e + i] ? w_down[e][r, i] : 0.  keep_mask: DEVICE
 * uint8 [N_e], 8-byte aligned (the mask of camera_select_prune); w_down_out: HOST array [n_experts] of DEVICE pointers
 * to buffers of the shape and pitch of the layer's W_down (not the layer's own).  bf16 layers in CAMERA_DOWN_HF
 * layout with d_ff[e] % 8 == 0, else CAMERA_ERR_UNSUPPORTED_SHAPE.
 *
 * camera_pruned_output: y_hat [n_tokens, d_model] fp32 from the h of the last forward call on this workspace.  layer,
 * n_tokens and aux->topk_idx (if that call exported the routing through it) must be those of that call, and nothing
 * else may have used the workspace since; w_down_masked as written by camera_mask_down_columns (any matrices of that
 * shape work: the call multiplies h by what it is given).  Other arguments and errors as for camera_layer_forward.
 * The result equals camera_layer_forward on the sliced layer up to the order of the fp32 sums over d_ff.
 */
int camera_mask_down_columns(const camera_layer_t* layer, const uint8_t* keep_mask, void* const* w_down_out,
                             void* cuda_stream);
int camera_pruned_output(const camera_layer_t* layer, const void* const* w_down_masked, int64_t n_tokens, float* y_hat,
                         const camera_score_aux_t* aux, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Scratch for camera_output_error. */
size_t camera_output_error_workspace_bytes(int64_t n_tokens);

/*
 * Distance between two layer outputs (the metrics of the paper's table of hidden-state errors):
 * out: DEVICE double[3] = { ||Y - Y_hat||_F^2 (the objective of Eq. 7), ||Y||_F^2, mean over tokens of the cosine
 * similarity of y_t and y_hat_t }.  y, y_hat: DEVICE [n_tokens, d_model] fp32.  Sums in float64, fixed order.
 */
int camera_output_error(const float* y, const float* y_hat, int64_t n_tokens, int32_t d_model, double* out,
                        void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Glue for running Algorithm 2's layer loop ("I <- O") on a synthetic stack of MoE layers, where no
 * attention block or trained norm exists (the paper has no counterpart: its layers are whole decoder layers):
 * out_t = (x_t + y_t) / sqrt(mean((x_t + y_t)^2) + eps), rounded to the dtype of x.  x: DEVICE [n_tokens, d_model]
 * bf16 (CAMERA_BF16) or fp32, y: DEVICE fp32 (a layer output), out: DEVICE like x (may be x itself).  d_model % 8 == 0.
 */
int camera_residual_norm(const void* x, int32_t dtype, const float* y, int64_t n_tokens, int32_t d_model, float eps,
                         void* out, void* cuda_stream);

/* The gated feed-forward block of one expert (Eq. 1-2 without the router), for training it after the slicing or for
 * running it as a dense layer.  bf16. */
typedef struct {
  int32_t d_model;              /* multiple of 8 */
  int32_t d_ff;                 /* micro-experts, any number >= 1 (what camera_compact_weights left of the expert) */
  int32_t down_ld;              /* leading dimension of w_down and its gradient, a multiple of 8, >= d_ff; 0 = d_ff */
  const void* w_gate;           /* DEVICE [d_ff, d_model] bf16, 16-byte aligned like every matrix here */
  const void* w_up;             /* DEVICE [d_ff, d_model] */
  const void* w_down;           /* DEVICE [d_model, down_ld], columns from d_ff on are not read */
} camera_ffn_t;

/* Scratch of camera_ffn_forward (backward = 0) and of camera_ffn_backward (1, which serves forward as well); size of the
 * gate and up products a forward call keeps for its backward call.  0 on invalid arguments.  The workspace starts with
 * a status word that camera_read_status reads.  A workspace of this size serves every call with no more tokens and no
 * larger d_ff (of the same d_model) as well, although the query may name more for some of them: a call cuts its sums over
 * d_ff into as many parts as it finds room for. */
size_t camera_ffn_workspace_bytes(const camera_ffn_t* ffn, int64_t n_tokens, int32_t backward);
size_t camera_ffn_saved_bytes(const camera_ffn_t* ffn, int64_t n_tokens);

/*
 * y = (SiLU(x W_gate^T) * (x W_up^T)) W_down^T.  x, y: DEVICE [n_tokens, d_model] bf16, 16-byte aligned.  saved: DEVICE,
 * camera_ffn_saved_bytes, 32-byte aligned, or NULL when no backward call follows.  Products of bf16 with fp32
 * accumulation; the gated product is rounded to bf16 between the two GEMMs, as in camera_layer_forward.
 */
int camera_ffn_forward(const camera_ffn_t* ffn, const void* x, int64_t n_tokens, void* y, void* saved, void* workspace,
                       size_t workspace_bytes, void* cuda_stream);

/*
 * Gradients of that call by its inputs, given dy (DEVICE [n_tokens, d_model] bf16) and what the call saved: dx
 * [n_tokens, d_model], dw_gate and dw_up [d_ff, d_model], dw_down [d_model, down_ld] (columns from d_ff on are not
 * written), all bf16, overwritten.  dx may be NULL, and may take the room of x or dy; no other output may overlap an input.
 * dw_* may be NULL together.  The gate and up products are kept with 24 of fp32's 32 bits (cut), their gradients formed
 * from those in fp32; h, dG and dU are rounded to bf16 as operands of the next product; the sums over tokens and
 * micro-experts are fp32.  `saved` is left as it is.  Results (of the forward call too) are the same bits on every run with
 * a workspace of the same size.
 */
int camera_ffn_backward(const camera_ffn_t* ffn, const void* x, const void* dy, int64_t n_tokens, const void* saved, void* dx,
                        void* dw_gate, void* dw_up, void* dw_down, void* workspace, size_t workspace_bytes,
                        void* cuda_stream);

/*
 * Recovery of a sliced model: what its output distribution says, and the loss that trains it towards the full model's.
 * (The paper evaluates perplexity and leaves recovery out; these calls have no counterpart there.)
 *
 * Rows of logits: DEVICE [n_rows, vocab] in CAMERA_BF16 or CAMERA_F32, rows `ld` elements apart (ld >= vocab), any
 * alignment of the element type.  vocab <= CAMERA_MAX_VOCAB.  The distribution of a row is softmax(x / temperature),
 * 0 < temperature < infinity, and 1.45 / temperature within fp32's range.  A logit of minus infinity is a token that cannot occur; a row of nothing else has no
 * distribution ("empty", see each call).  A row with a NaN or a logit of plus infinity gives NaN.  All statistics are
 * fp32 sums.  A row's results do not depend on what other rows hold; calls of one shape give the same bits on every run.
 * No workspace, and so no status word: a bounded wait between CTAs that share a row (camera_set_wait_limit_ns), should it
 * run out, gives NaN in that row and in the rows those CTAs have left to do.
 */
#define CAMERA_MAX_VOCAB (1 << 20)
#define CAMERA_MAX_TOP 128

/*
 * Log-probability of one given token per row, the entropy of the row's distribution (both in nats) and its top_n
 * alternatives.  targets: DEVICE int64 [n_rows]; logprob: DEVICE [n_rows]; both or neither may be NULL.  A target outside
 * [0, vocab) (an ignore index such as -100) gives 0.  entropy: DEVICE [n_rows] or NULL.  top_idx / top_logprob: DEVICE
 * [n_rows, top_n] int32 / fp32, by decreasing logit, ties by increasing index; entries beyond the tokens that can occur
 * are -1 / minus infinity.  0 <= top_n <= CAMERA_MAX_TOP (else CAMERA_ERR_UNSUPPORTED_SHAPE).
 * Empty row: logprob minus infinity, entropy 0, no alternatives.  Row with NaN: NaN, alternatives -1 / NaN.
 */
int camera_token_logprobs(const void* logits, int32_t dtype, int64_t ld, int64_t n_rows, int32_t vocab,
                          const int64_t* targets, int32_t top_n, float temperature, float* logprob, float* entropy,
                          int32_t* top_idx, float* top_logprob, void* cuda_stream);

/* camera_distill_t.flags */
enum { CAMERA_DISTILL_TAIL = 1u };  /* the probability outside the teacher's list is one more class (else the list is renormalised) */

/* The student's logits and the teacher's top log-probabilities, as camera_token_logprobs writes them. */
typedef struct {
  const void* logits;             /* DEVICE [n_rows, vocab] */
  int64_t ld;
  int64_t n_rows;
  int32_t dtype;                  /* camera_dtype_t */
  int32_t vocab;
  const int32_t* teacher_idx;     /* DEVICE [n_rows, k], distinct in a row; an index outside [0, vocab) is no entry, unless
                                     its log-probability is a NaN (what camera_token_logprobs writes for a row with one) */
  const float* teacher_logprob;   /* DEVICE [n_rows, k] log-probabilities at the same temperature (without TAIL any constant may be added) */
  int32_t k;                      /* 1 .. CAMERA_MAX_TOP */
  float temperature;
  uint32_t flags;
} camera_distill_t;

/*
 * Kullback-Leibler divergence of the student from the teacher's list, per row:
 *   loss = sum_j p_j (ln p_j - ln q_j),  p = softmax of the list;
 *   CAMERA_DISTILL_TAIL: p = exp(teacher_logprob), plus rest (ln rest - ln R), rest = max(0, 1 - sum p), R = the
 *   student's probability outside the list (below 2^-1022 it counts as none, and the rest's term is dropped).
 * The gradient is the derivative of that loss, whatever the list's probabilities add to.  A list without an entry, or
 * whose entries have no probability, gives loss and gradient 0 without TAIL (with it, all of the teacher is the rest).  A NaN
 * among a list's log-probabilities gives NaN.
 * forward: loss, and for a later backward lse (ln sum exp(x / temperature)) and, with TAIL, log_tail (the same sum over
 *   the tokens outside the list); lse and log_tail may be NULL.  All DEVICE fp32 [n_rows].
 * backward: d_logits = d_loss[r] d loss_r / d x, rows d_ld elements apart, dtype of the logits; d_logits may be the
 *   logits themselves (then d_ld == ld).
 * step: both from one call, for a d_loss known beforehand (a mean over tokens, a mask); loss of a row with d_loss 0 is 0.
 * A row with d_loss 0 has a gradient of 0 and its logits are not read.  An empty row has loss and gradient 0, and so has
 * one whose logits all overflow fp32 to minus infinity when divided by the temperature and multiplied by log2(e).
 * backward takes lse as fp32: its rounding, 6e-8 of the size of the scaled logits, is a relative error of that gradient;
 * step has no such error.
 * The factor temperature^2 that some recipes put before the loss goes into d_loss.
 */
int camera_distill_forward(const camera_distill_t* d, float* loss, float* lse, float* log_tail, void* cuda_stream);
int camera_distill_backward(const camera_distill_t* d, const float* d_loss, const float* lse, const float* log_tail,
                            void* d_logits, int64_t d_ld, void* cuda_stream);
int camera_distill_step(const camera_distill_t* d, const float* d_loss, float* loss, void* d_logits, int64_t d_ld,
                        void* cuda_stream);

/*
 * Training a sliced layer: what stands around its experts.  (The paper has no counterpart.)  Matrices of rows: DEVICE, in
 * CAMERA_BF16 or CAMERA_F32, rows `ld` elements apart (ld >= their width), any alignment of the element type; rows that
 * start on 16-byte boundaries are read and written 16 bytes at a time.  Sums are fp32, results rounded once.  Calls of one
 * shape give the same bits on every run.  A result may take the room of an input where its comment says so (same address,
 * same ld); otherwise outputs overlap nothing.
 */

/* camera_norm_t.flags */
enum { CAMERA_NORM_RMS = 1u };    /* root mean square: no mean is taken off */

/* The rows a norm works on and its weights. */
typedef struct {
  const void* x;                  /* [n_rows, d]; backward: what was normalised (`sum` where there was a residual) */
  int64_t ld;
  int64_t n_rows;
  int32_t dtype;                  /* camera_dtype_t of all matrices of the call */
  int32_t d;                      /* 1 .. 32768 */
  const void* weight;             /* DEVICE [d] or NULL (ones) */
  const void* bias;               /* DEVICE [d] or NULL (zeros) */
  int32_t weight_dtype;           /* camera_dtype_t of weight and bias */
  float eps;                      /* >= 0, finite */
  uint32_t flags;
} camera_norm_t;

/*
 * forward: z = x + residual, rounded to the dtype (z = x without one; sum [n_rows, d] receives z and goes with residual:
 *   both or neither);  mu = mean z (0 with CAMERA_NORM_RMS), s = 1 / sqrt(mean (z - mu)^2 + eps), y = (z - mu) s weight + bias.
 *   mean, rstd: DEVICE fp32 [n_rows], receive mu and s, either may be NULL.  y and sum may take the room of x or residual.
 * backward, given dy, n->x = z, and mu and s as the forward call left them (mean may be NULL with CAMERA_NORM_RMS):
 *   h = (z - mu) s, g = dy weight:  dx = s (g - mean g - h mean(g h)) + d_sum  (no mean g with CAMERA_NORM_RMS),
 *   d_weight = sum over rows of dy h, d_bias = sum over rows of dy (DEVICE fp32 [d], overwritten).
 *   d_sum: gradient of z from elsewhere (the residual stream's), or NULL.  dx is also the residual's gradient.  dx may be
 *   NULL (then d_sum too), d_weight and d_bias may be NULL, not all three.  dx may take the room of dy, d_sum or z.
 *   n->bias and n->eps do not enter; they are checked as in the forward call.
 * A NaN or an infinity stays in its row (and reaches d_weight and d_bias).  A row without variance and with eps 0 gives NaN.
 * Squares and sums are fp32: elements beyond about 1e17 (and, with eps 0, deviations below 1e-18) leave its range.
 * workspace (needed for d_weight or d_bias): camera_norm_backward_workspace_bytes, which serves every call with no more
 * rows of that width.  No kernel here waits, so it holds no status word.
 */
int camera_norm_forward(const camera_norm_t* n, const void* residual, int64_t residual_ld, void* sum, int64_t sum_ld, void* y,
                        int64_t y_ld, float* mean, float* rstd, void* cuda_stream);
size_t camera_norm_backward_workspace_bytes(int64_t n_rows, int32_t d);
int camera_norm_backward(const camera_norm_t* n, const void* dy, int64_t dy_ld, const float* mean, const float* rstd,
                         const void* d_sum, int64_t d_sum_ld, void* dx, int64_t dx_ld, float* d_weight, float* d_bias,
                         void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Tokens sorted by expert and back.  topk_idx, rows: DEVICE int32 [n_tokens, top_k]; topk_w: DEVICE fp32 [n_tokens, top_k]
 * or NULL (ones).  top_k 1 .. 16, n_experts 1 .. 1024, n_tokens * top_k < 2^31, d_model 1 .. 2^20.
 * dispatch: the pairs (token t, slot j) in order of their expert topk_idx[t, j], within one by token and slot: rows[t, j] is the
 *   pair's place, x_sorted[rows[t, j]] = x[t], and expert e's rows are offsets[e] .. offsets[e+1] (DEVICE int32 [n_experts + 1]).
 *   A pair whose index lies outside [0, n_experts) is left out (rows -1).  Rows of x_sorted from offsets[n_experts] on are left
 *   as they were; it has room for n_tokens * top_k rows.  A token may name an expert twice.
 * combine: y[t] = add[t] + sum over j of topk_w[t, j] y_sorted[rows[t, j]], added in the order of the slots, add last.  add may
 *   be NULL; y may take its room.  n_rows: rows that y_sorted has; an entry of `rows` outside [0, n_rows) adds nothing.  A weight
 *   of 0 still multiplies its row (NaN and infinity there give NaN).
 * combine_backward: dy_sorted[rows[t, j]] = topk_w[t, j] dy[t], d_topk_w[t, j] = <dy[t], y_sorted[rows[t, j]]> (0 for a pair that
 *   was left out).  Either may be NULL, not both; y_sorted is read for d_topk_w only.  Rows of dy_sorted that no pair names are
 *   left as they were.  Entries of `rows` are distinct.  dy_sorted may take the room of y_sorted.
 * dispatch_backward: dx[t] = add[t] + sum over j of dx_sorted[rows[t, j]]: combine without weights.
 * workspace: camera_moe_dispatch_workspace_bytes, which serves every call with no more tokens, slots and experts; no status word.
 */
size_t camera_moe_dispatch_workspace_bytes(int64_t n_tokens, int32_t top_k, int32_t n_experts);
int camera_moe_dispatch(const void* x, int32_t dtype, int64_t ld, int64_t n_tokens, int32_t d_model, const int32_t* topk_idx,
                        int32_t top_k, int32_t n_experts, void* x_sorted, int64_t sorted_ld, int32_t* rows, int32_t* offsets,
                        void* workspace, size_t workspace_bytes, void* cuda_stream);
int camera_moe_dispatch_backward(const void* dx_sorted, int32_t dtype, int64_t sorted_ld, int64_t n_rows, const int32_t* rows,
                                 int64_t n_tokens, int32_t top_k, int32_t d_model, const void* add, int64_t add_ld, void* dx,
                                 int64_t ld, void* cuda_stream);
int camera_moe_combine(const void* y_sorted, int32_t dtype, int64_t sorted_ld, int64_t n_rows, const int32_t* rows,
                       const float* topk_w, int64_t n_tokens, int32_t top_k, int32_t d_model, const void* add, int64_t add_ld,
                       void* y, int64_t ld, void* cuda_stream);
int camera_moe_combine_backward(const void* dy, int32_t dtype, int64_t ld, int64_t n_tokens, int32_t d_model, const int32_t* rows,
                                const float* topk_w, int32_t top_k, const void* y_sorted, int64_t sorted_ld, int64_t n_rows,
                                void* dy_sorted, int64_t dy_sorted_ld, float* d_topk_w, void* cuda_stream);

/* One matrix of camera_orthogonalize. */
typedef struct {
  const void* in;                 /* DEVICE [rows, cols], rows in_ld elements apart */
  void* out;                      /* DEVICE bf16 [rows, cols], rows out_ld elements apart; may be `in` (bf16, same ld) */
  int64_t in_ld, out_ld;
  int32_t rows, cols;             /* up to 131072, one of them up to 32768; either may be 0 */
} camera_matrix_t;

/*
 * The updates of a layer's matrices, orthogonalised: X = in / (|in| + eps) with the Frobenius norm, then `steps` times
 *   X <- a X + (b A + c A A) X,  A = X X^T (of the shorter side),
 * which takes every singular value s to a s + b s^3 + c s^5; out = X.  coefficients: HOST [steps][3], (a, b, c) of each step.
 * With those that take values towards 1, out is near the orthogonal factor of `in`.  mats: HOST [n_mats], in in `dtype`; the
 * matrices of a call, whatever their shapes, are worked on together.  1 <= steps <= 64.  Coefficients under which a singular
 * value or the step's factor of it could pass 1000 are refused (CAMERA_ERR_INVALID_ARG): they do not converge.
 * Products of fp16 operands with fp32 sums; factors that keep them in range follow from the coefficients; X itself is kept
 * in 22 bits.  Before its rounding to bf16, which adds 1.7e-3, the result is about 1e-3 off 64 bits (root mean square over the
 * matrix, relative), whatever the matrix' rank, and up to 4e-3 where the shorter side is below 16.  Where `in` has nothing,
 * roundings grow by the product of the steps' a (485 for five of 3.4445); beyond 1e4 they show.  A matrix of zeros gives zeros;
 * one with a NaN or an infinity gives NaN and leaves the others of the call as they are.
 * workspace: camera_orthogonalize_workspace_bytes of the same shapes (pointers are not read); it starts with a status word
 * that camera_read_status reads.
 */
size_t camera_orthogonalize_workspace_bytes(const camera_matrix_t* mats, int32_t n_mats);
int camera_orthogonalize(const camera_matrix_t* mats, int32_t n_mats, int32_t dtype, const float* coefficients, int32_t steps,
                         float eps, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Scratch for camera_analyze_layer_host: score + select scratch for one batch of tokens, two staging
 * buffers for batches of x, and the results. */
size_t camera_analyze_workspace_bytes(const camera_layer_t* layer, int64_t n_tokens, int32_t n_levels);

/*
 * One whole analysis step with HOST token and result buffers: copies x_host (pinned or
 * pageable, [n_tokens, d_model]) to the device in batches on a copy stream of its own (the first
 * batch 8192 tokens, every later one half as large again, up to 65536), scoring batch b
 * (camera_score_layer, accumulating) while batch b+1 is on its way; then runs camera_select_all
 * (every prune mask of prune_ratios, HOST [n_prune], may be empty, and the bit-widths from one
 * set of radix passes; separate camera_select_prune / camera_alloc_bits calls where n_prune +
 * n_levels - 1 > 7) and copies energy [N_e] fp32, keep masks [n_prune, N_e] and bits_out [N_e]
 * back to the given HOST buffers (any may be NULL).  The layer's weights stay DEVICE resident.
 * Synchronises the stream before returning, and returns the workspace's status word if a kernel
 * recorded one.  The batch sizes depend on n_tokens alone, so a given input gives the same bits
 * on every run.
 */
int camera_analyze_layer_host(const camera_layer_t* layer, const void* x_host, int64_t n_tokens,
                              float alpha, const double* prune_ratios, int32_t n_prune,
                              const double* ratios, const int32_t* bits, int32_t n_levels,
                              float* energy_host, uint8_t* keep_host, uint8_t* bits_host,
                              void* workspace, size_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* CAMERA_B200_H */
