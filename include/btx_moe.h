/*
 * btx_moe.h - C ABI of the MI355X (gfx950) Mixture-of-Experts feed-forward layer
 * of Branch-Train-MiX (arXiv 2403.07816).
 *
 * The layer (Sec. 3.2):   FF_MoE(x) = sum_i g_i(W_l x) * FF_i(x)
 * with a linear router W_l, a sparse routing function g, and per-expert SwiGLU
 * feed-forward sublayers FF_i(x) = (silu(x W1_i) * (x W3_i)) W2_i taken from the
 * branched expert models.
 *
 * Conventions for every entry point
 *   - All data pointers are DEVICE pointers unless the comment says "host".
 *   - Tensors are row-major and contiguous.  T = tokens, d = model width,
 *     f = feed-forward width per expert, E = experts, k = experts per token,
 *     R = T*k routed rows.
 *   - The caller owns every buffer, including the workspace; the library
 *     allocates nothing.  No result depends on an earlier call.  The only
 *     process-wide state is set-up and tooling: per device, the kernels'
 *     raised dynamic-LDS limit (btx_init) and the optional stage-event table
 *     (btx_profile_stages).
 *   - Work is enqueued on `stream` (a hipStream_t passed as void*, NULL = the
 *     default stream) and the call returns without synchronising.  Group sizes
 *     never travel to the host.
 *   - The return value is a btx_status.  Nothing throws, aborts or prints.
 *     Arguments are validated before anything is launched; on an error status
 *     no kernel has been enqueued.
 *   - T == 0 is a valid no-op (BTX_OK).
 *   - A workspace query never falls as T grows: a workspace sized for the largest batch
 *     serves every smaller one.
 *   - Rows move as 16-byte pieces: every tensor of rows (x, the expert weights and their
 *     gradients, saved activations, outputs, workspaces) starts on a 16-byte boundary, and
 *     the expert strides are multiples of 8 elements; BTX_ERR_INVALID_ARG otherwise.
 *   - Every kernel is free of atomics: results are bit-identical run to run.  The order
 *     of every sum is fixed by the shapes, the routing counts and the number of compute
 *     units of the device (the bf16 up-projection, down-projection and input-gradient
 *     products cut the tiles of a partly filled last round of workgroups, or with few rows per
 *     expert every tile, into up to eight K ranges; fp32 does so with the tiles of the
 *     down-projection and the input gradient when they are few; a second kernel, after the
 *     down-projection of few rows the one that combines them, adds the ranges in ascending order).
 *   - Outputs must not alias inputs unless stated.  NaN/Inf inputs give
 *     unspecified results.
 */
#ifndef BTX_MOE_H
#define BTX_MOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  BTX_OK = 0,
  BTX_ERR_INVALID_ARG = 1, /* null pointer, bad size, bad enum, k > E, ...            */
  BTX_ERR_UNSUPPORTED = 2, /* valid by the paper but outside what the kernels accept  */
  BTX_ERR_WORKSPACE = 3,   /* workspace smaller than the matching *_workspace_bytes() */
  BTX_ERR_HIP = 4          /* a HIP launch reported an error                          */
} btx_status;

typedef enum {
  BTX_F32 = 0, /* float                                    */
  BTX_BF16 = 1 /* bfloat16 storage, fp32 accumulation      */
} btx_dtype;

/* Routing function g (Sec. 3.2 and Sec. 3.3 "Routing method"). */
typedef enum {
  /* Top-k: keep the k largest logits, softmax over the kept ones (equal to the
   * full softmax renormalised over the chosen k).  Gates sum to 1 per token. */
  BTX_ROUTE_TOPK_RENORM = 0,
  /* Switch: k = 1, expert = argmax, gate = that expert's full-softmax probability. */
  BTX_ROUTE_SWITCH_TOP1 = 1,
  /* Sample top-1: k = 1, expert = first e with cumsum_{j<=e} softmax_j > U[t]
   * (E-1 if none), gate = that expert's full-softmax probability. */
  BTX_ROUTE_SAMPLE_TOP1 = 2,
  /* Sec. 3.3 "Sample Top-1" as printed, training time: soft sample y = softmax((logits + G) / tau)
   * with Gumbel noise G supplied by the caller, all but its largest entry zeroed: that expert
   * is run with gate y_max.  The load-balancing probabilities stay softmax(logits). */
  BTX_ROUTE_GUMBEL_TOP1 = 3
} btx_route_mode;

/* u_i of the load-balancing loss L_LB = alpha * E * sum_i u_i p_i (Sec. 3.3),
 * p_i = batch mean of softmax_i. */
typedef enum {
  BTX_LB_TOKEN_FRAC = 0, /* u_i = counts_i / (T*k): share of routed (token,slot) pairs */
  BTX_LB_GATE_MEAN = 1   /* u_i = (sum_t g_i) / T: the formula as printed              */
} btx_lb_mode;

/* btx_moe_ff_backward flags */
#define BTX_FLAG_LB_GRAD_THROUGH_U 1u /* BTX_LB_GATE_MEAN only: also differentiate u_i */

const char* btx_status_string(int status);
int btx_version(void);

/* One-time set-up on the CURRENT device: raises the dynamic-LDS limit of every expert-GEMM
 * kernel (they use all 160 KB of a compute unit's LDS).  Optional: the first bf16 call of
 * btx_moe_ff_forward / btx_moe_ff_backward, and the first of btx_moe_ff_forward_mx4,
 * btx_moe_ff_forward_fp8 and btx_fp8_matmul, on a device does the same by itself, but that set-up cannot be recorded into a HIP graph, so a caller that captures its very first step
 * calls btx_init() before beginning the capture (once per device that it uses).  It also
 * looks up the device address of btx_moe_route_noalloc's fixed workspace.
 * Idempotent.  Errors: BTX_ERR_HIP. */
int btx_init(void);

/* Profiling aid (the one piece of process-wide state; not thread-safe; off by default).
 * events: HOST array of 2*n_pairs hipEvent_t handles owned by the caller.  While set,
 * stage s of any later call records events[2s] before and events[2s+1] after its
 * kernels on the caller's stream, so that single kernels can be timed inside the real
 * sequence.  n_pairs = 0 switches it off.  Stage ids: */
enum {
  BTX_STAGE_ROUTE = 0,        /* btx_moe_route: its two or four kernels;
                                 btx_moe_group_route: its one or two              */
  BTX_STAGE_GATHER_X = 1,     /* forward: x -> expert-grouped rows (bf16, only when
                                  x has 2^32 bytes or more: else UP reads x itself);
                                  4-bit experts: x quantised                         */
  BTX_STAGE_UP = 2,           /* forward: xs W1, xs W3, SwiGLU; small fp32 layers:
                                  and the work of DOWN, which is then empty          */
  BTX_STAGE_DOWN = 3,         /* forward: act W2                                   */
  BTX_STAGE_COMBINE = 4,      /* forward: gate-weighted un-permute                 */
  BTX_STAGE_GATHER_DY = 5,    /* backward: dY -> grouped rows (as GATHER_X)        */
  BTX_STAGE_BWD_ACT = 6,      /* backward: dys W2^T + SwiGLU backward              */
  BTX_STAGE_BWD_DX = 7,       /* backward: dh1 W1^T + dh3 W3^T; fp32: and the work of
                                  DW13 and DW2, which are then empty                */
  BTX_STAGE_GATHER_X_BWD = 8, /* backward: x (and dY) -> transposed grouped rows for
                                  the weight gradients (bf16 and experts of many rows; none
                                  with frozen experts)                              */
  BTX_STAGE_DW13 = 9,         /* backward: dW1, dW3; bf16 without GATHER_X_BWD: and
                                  dW2, DW2 is then empty                            */
  BTX_STAGE_DW2 = 10,         /* backward: dW2                                     */
  BTX_STAGE_ROUTER_BWD = 11,  /* backward: router gradients and final dX (small
                                  batches: its first part runs beside the weight
                                  gradients); for gates of another router dgates
                                  (dX: COMBINE); btx_moe_group_route_backward        */
  BTX_STAGE_NORM_BWD = 12,    /* btx_rmsnorm_backward: both kernels                */
  BTX_STAGE_COUNT = 13
};
int btx_profile_stages(void** events, int n_pairs);

/* ---------------------------------------------------------------------------
 * btx_moe_route - router linear, softmax, selection, gates, load-balancing
 * statistics and the token -> expert grouping (Sec. 3.2: W_l x and
 * g = SoftMax(TopK(.)); Sec. 3.3: load balancing, Switch, sample top-1; the
 * grouping is what "skip FF_i where the gate is zero" needs).
 *
 *   x          [T,d]   x_dtype (BTX_F32 or BTX_BF16)
 *   W_router   [d,E]   fp32
 *   b_router   [E]     fp32, may be NULL (the paper's router has no bias)
 *   U          [T]     fp32 in [0,1); required iff route_mode == SAMPLE_TOP1;
 *              [T,E]   fp32 Gumbel noise (-log(-log(uniform))) iff route_mode == GUMBEL_TOP1
 *   tau                temperature of GUMBEL_TOP1 (> 0); ignored by the other modes
 *   capacity_factor    0 = dropless.  > 0: every expert keeps its first
 *                      ceil(capacity_factor * T*k / E) pairs in (t,j) order (Sec. 4.3: "a hard
 *                      limit after which routed tokens will be dropped"; the product is taken in
 *                      double precision on the float passed, so 0.8f, which lies above 0.8,
 *                      gives 209 and not 208 at T*k/E = 260); a dropped pair gets
 *                      inv_pos = -1, no grouped row and contributes nothing to the layer's output
 *                      or to dg; counts, gate_sum and lb_loss describe the routing before drops,
 *                      offsets the kept rows; perm[r] = 0 for r >= offsets[E]
 * Selection: logits are accumulated in fp32; ties go to the lower expert index;
 * topk_idx lists the chosen experts by descending logit.
 * Outputs
 *   topk_idx   [T,k]   int32 expert ids
 *   gates      [T,k]   fp32
 *   probs      [T,E]   fp32 full softmax (kept for the backward pass)
 *   counts     [E]     int32 routed pairs per expert (before any capacity drop)
 *   offsets    [E+1]   int32 exclusive prefix of counts
 *   perm       [R]     int32: perm[r] = t*k+j of the pair stored at grouped row r;
 *                      rows of expert e are offsets[e]..offsets[e+1]-1, in (t,j) order
 *   inv_pos    [T,k]   int32: inverse of perm (-1: pair dropped)
 *   gate_sum   [E]     fp32 sum_t g_{t,e}
 *   prob_sum   [E]     fp32 sum_t softmax_{t,e}
 *   lb_loss    [1]     fp32 lb_alpha * E * sum_e u_e * prob_sum_e / T
 * Requirements: 1 <= k <= E <= 64; d % 8 == 0; SWITCH/SAMPLE/GUMBEL need k == 1;
 * T*k < 2^31.  workspace >= btx_moe_route_workspace_bytes(T,d,E,k).
 */
size_t btx_moe_route_workspace_bytes(int T, int d, int E, int k);
int btx_moe_route(const void* x, int x_dtype, const float* W_router, const float* b_router, const float* U,
                  int T, int d, int E, int k, int route_mode, int lb_mode, float lb_alpha, float tau,
                  float capacity_factor, int32_t* topk_idx, float* gates, float* probs, int32_t* counts, int32_t* offsets,
                  int32_t* perm, int32_t* inv_pos, float* gate_sum, float* prob_sum, float* lb_loss,
                  void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * btx_moe_route_noalloc - btx_moe_route for callers that cannot allocate device memory: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, same kernels and bit-identical results, but without the workspace pair: the
 * workspace is a fixed array of btx_moe_route_noalloc_max_workspace_bytes() (4 MiB) inside the
 * library's device image, which every GPU the library runs on holds until the process ends.
 * The call allocates and frees nothing.
 *   - A problem whose btx_moe_route_workspace_bytes(T,d,E,k) exceeds that size is refused with
 *     BTX_ERR_WORKSPACE before anything else is checked or launched (T = 16384, d = 4096,
 *     E = 64 needs 2 MiB).
 *   - All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (two
 *     streams, two threads) race and give unspecified results; calls on one stream are safe.
 *     Nothing in the array has to start at zero, every call overwrites what it reads.
 *   - The array's device address is looked up on the first call on a device (or by btx_init);
 *     that look-up is not a stream operation and may precede a capture.
 */
size_t btx_moe_route_noalloc_max_workspace_bytes(void);
int btx_moe_route_noalloc(const void* x, int x_dtype, const float* W_router, const float* b_router, const float* U,
                          int T, int d, int E, int k, int route_mode, int lb_mode, float lb_alpha, float tau,
                          float capacity_factor, int32_t* topk_idx, float* gates, float* probs, int32_t* counts,
                          int32_t* offsets, int32_t* perm, int32_t* inv_pos, float* gate_sum, float* prob_sum,
                          float* lb_loss, void* stream);

/* ---------------------------------------------------------------------------
 * btx_moe_norm_route - btx_moe_route with the block's pre-normalisation folded into the
 * router's read of the rows.  The seed model (Sec. 4.1: Llama-2 7B) normalises the residual
 * stream h before its feed-forward sublayer,
 *     xn[t,c] = gain[c] * h[t,c] * rstd[t],   rstd[t] = 1 / sqrt(mean_c h[t,c]^2 + eps),
 * and the block's output is h + FF_MoE(xn): xn is the x of Sec. 3.2, h goes to
 * btx_moe_ff_forward as `residual`.  One kernel reads h, writes xn (for the expert
 * GEMMs) and rstd (for the backward pass) and routes on xn.
 *
 *   h      [T,d]  x_dtype   raw rows
 *   gain   [d]    fp32
 *   eps           >= 0
 *   xn     [T,d]  x_dtype   out; must not alias h
 *   rstd   [T]    fp32      out
 * Mean square, rstd and the product are evaluated in fp64 and xn is rounded once to x_dtype;
 * the logits are computed from those rounded values, exactly as btx_moe_route would from xn (more
 * than 8 experts and 512 tokens: to the rounding of fp32 sums, which may run in another order).
 * Everything else as btx_moe_route (same workspace size).
 */
int btx_moe_norm_route(const void* h, int x_dtype, const float* gain, float eps, void* xn, float* rstd,
                       const float* W_router, const float* b_router, const float* U, int T, int d, int E, int k,
                       int route_mode, int lb_mode, float lb_alpha, float tau, float capacity_factor,
                       int32_t* topk_idx, float* gates, float* probs, int32_t* counts, int32_t* offsets, int32_t* perm,
                       int32_t* inv_pos, float* gate_sum, float* prob_sum, float* lb_loss, void* workspace,
                       size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * btx_rmsnorm_backward - backward of that normalisation (chain rule; the paper prints no
 * backward pass).  dXn is the dX that btx_moe_ff_backward returns when it is given xn as x:
 *     dH[t]    = rstd[t] * gain * dXn[t] - h[t] * rstd[t]^3 * (sum_c gain_c dXn[t,c] h[t,c]) / d  (+ dres[t])
 *     dgain[c] = sum_t dXn[t,c] * h[t,c] * rstd[t]
 *
 *   dXn, h  [T,d]  dtype
 *   gain    [d]    fp32;  rstd [T] fp32 as written by btx_moe_norm_route
 *   dres    [T,d]  dtype, may be NULL: added to dH (the gradient that reaches h through the
 *                  residual connection, i.e. the dY given to btx_moe_ff_backward)
 *   dH      [T,d]  dtype  out; may alias dXn or dres
 *   dgain   [d]    fp32   out (overwritten)
 * fp32 arithmetic, sums in a fixed order (bit-reproducible).
 * Requirements: d % 8 == 0, d <= 16384; workspace >= btx_rmsnorm_backward_workspace_bytes(T,d).
 */
size_t btx_rmsnorm_backward_workspace_bytes(int T, int d);
int btx_rmsnorm_backward(const void* dXn, const void* h, const float* gain, const float* rstd, const void* dres,
                         int dtype, int T, int d, void* dH, float* dgain, void* workspace, size_t workspace_bytes,
                         void* stream);

/* ---------------------------------------------------------------------------
 * btx_moe_ff_forward - gather tokens into expert groups, the expert SwiGLU
 * FFNs as grouped GEMMs, and the gate-weighted combine (layer equation of
 * Sec. 3.2; FF_i is the seed model's 3-matrix feed-forward, Sec. 4.1).
 *
 *   x   [T,d]            dtype
 *   W1, W3  expert e at  W + e*w13_expert_stride elements, [d,f] row-major
 *   W2      expert e at  W2 + e*w2_expert_stride elements, [f,d] row-major
 *   gates, offsets, perm, inv_pos: as written by btx_moe_route
 *   residual [T,d]       dtype, may be NULL: the transformer block's input, added to the sum
 *                        (h + FF_MoE(norm(h)) in one pass; with a capacity limit a token whose
 *                        pairs were all dropped passes through as the residual alone).  May be x
 *                        itself or out (elementwise in t).
 *   out [T,d]            dtype:  out[t] = residual[t] + sum_j gates[t,j] * FF_{idx[t,j]}(x[t]),
 *                        summed in fp32 (residual first, then j ascending), rounded once
 *   save_h1, save_h3 [R,f] dtype, grouped-row order: x W1_e and x W3_e, kept for
 *                        the backward pass.  Both NULL = forward only.
 * dtype BTX_BF16: bf16 storage, bf16 MFMA products, fp32 accumulation; the
 * activation silu(h1)*h3 and the expert output are rounded to bf16 once each.
 * dtype BTX_F32: fp32 matrix-instruction products (exact products, fp32 accumulation), fp32 storage.
 * Requirements: 1 <= k <= E <= 64, d % 8 == 0, f % 8 == 0, strides >= d*f and multiples of 8.
 * Limits (BTX_ERR_UNSUPPORTED beyond them; also for btx_moe_ff_backward): the bf16 kernels address the
 * padded grouped rows with 32-bit byte offsets, ceil(R/64)*64 + 64*E < 2^23 (about 8.3 M routed rows);
 * fp32, and bf16 with a d or f that is no multiple of 32 (or below 64), take R/64 + E <= 65535 row tiles
 * (about 4.1 M routed rows).  Weight gradients in bf16 address 32 or 64 grouped rows of f elements with 32 bits: f <= 2^25 - 24
 * (few routed rows: min(R, 32) * f <= 2^31 is enough).
 */
size_t btx_moe_ff_forward_workspace_bytes(int T, int d, int f, int E, int k, int dtype);
int btx_moe_ff_forward(const void* x, const void* W1, const void* W3, const void* W2, int dtype,
                       int64_t w13_expert_stride, int64_t w2_expert_stride, int T, int d, int f, int E, int k,
                       const float* gates, const int32_t* offsets, const int32_t* perm, const int32_t* inv_pos,
                       const void* residual, void* out, void* save_h1, void* save_h3,
                       void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * btx_moe_ff_backward - gradients of  <dY, out> + lb_grad_scale * lb_loss  with
 * the discrete expert selection held fixed (chain rule on Sec. 3.2's layer
 * equation and Sec. 3.3's load-balancing loss; the paper trains the layer by
 * gradient descent but prints no backward).
 *
 *   dY [T,d] dtype; x, W*, strides, routing outputs, save_h1/save_h3 as in forward
 *   lb_grad_scale: upstream gradient of lb_loss (1 when it is added to the
 *                  training loss as in Sec. 3.3; 0 = no load-balancing gradient)
 *   noise [T,E], tau: the Gumbel noise and temperature given to btx_moe_route when
 *                  route_mode == GUMBEL_TOP1 (the soft sample is recomputed from probs,
 *                  noise and tau); noise must be NULL for the other modes
 * Outputs (overwritten, never accumulated into)
 *   dX        [T,d]  dtype
 *   dW_router [d,E]  fp32
 *   db_router [E]    fp32, may be NULL
 *   dW1, dW3, dW2    stacked like W1/W3/W2 (same strides), dW_dtype; all three
 *                    NULL = frozen experts (router and input gradients only).
 *                    Experts with no routed rows get zeros.
 * Requirements as forward; dW_dtype must equal dtype or be BTX_F32.
 */
size_t btx_moe_ff_backward_workspace_bytes(int T, int d, int f, int E, int k, int dtype);
int btx_moe_ff_backward(const void* dY, const void* x, const float* W_router, const void* W1, const void* W3,
                        const void* W2, int dtype, int64_t w13_expert_stride, int64_t w2_expert_stride,
                        int T, int d, int f, int E, int k, int route_mode, int lb_mode, float lb_alpha,
                        float lb_grad_scale, unsigned flags, const float* noise, float tau,
                        const int32_t* topk_idx, const float* gates, const float* probs,
                        const int32_t* offsets, const int32_t* perm, const int32_t* inv_pos,
                        const float* gate_sum, const float* prob_sum, const int32_t* counts,
                        const void* save_h1, const void* save_h3,
                        void* dX, float* dW_router, float* db_router, void* dW1, void* dW3, void* dW2,
                        int dW_dtype, void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * btx_merge_average - elementwise mean of N same-shape tensors: how the
 * non-feed-forward parameters (attention, embeddings, ...) of the branched
 * models are merged (Sec. 3.2).
 *
 *   inputs  HOST array of N device pointers, each [numel] of dtype
 *   out     [numel] dtype; may alias any inputs[i]
 * BTX_BF16: the sum is taken in fp32 in input order and its quotient by N is
 * rounded to bf16 once (no double rounding through fp32).  BTX_F32: sum and
 * division in fp64, rounded once to fp32.  The mean of N equal tensors is
 * that tensor, bit for bit.
 * Requirements: 1 <= N <= 16, numel >= 0, pointers aligned to 16 bytes.
 */
int btx_merge_average(const void* const* inputs, int N, void* out, int64_t numel, int dtype, void* stream);

/* ---------------------------------------------------------------------------
 * btx_merge_weighted - the merge of Sec. 3.2 with caller-chosen coefficients:
 * out = sum_n weights[n] * inputs[n], elementwise.  (The paper only averages;
 * this is the same pass with the 1/N replaced by a weight per model, e.g. to
 * favour the seed model or a domain.  The weights are used as given, they are
 * not normalised.)
 *
 *   inputs   HOST array of N device pointers, each [numel] of dtype
 *   weights  HOST array of N finite floats
 *   out      [numel] dtype; may alias any inputs[i]
 * The sum is accumulated in fp64 in input order (every product is exact there)
 * and rounded once to the storage type, for bf16 without a detour through fp32.
 * Requirements: 1 <= N <= 16, numel >= 0, pointers aligned to 16 bytes.
 */
int btx_merge_weighted(const void* const* inputs, const float* weights, int N, void* out, int64_t numel, int dtype,
                       void* stream);

/* ---------------------------------------------------------------------------
 * btx_mix_experts - MiX construction utilities of Sec. 3.3: "Splitting Experts"
 * (each of the N FFs is cut along d_ff into C chunks, giving N*C experts of width
 * f/C: expert i*C+c owns columns [c*f/C, (c+1)*f/C) of W1_i and W3_i and the same
 * rows of W2_i) and "Blending Experts" (each FF is cut into N chunks and expert n is
 * built from the n-th chunk of FF 0, FF 1, ... in that order; width stays f).  A
 * one-off copy made when the MoE is built; every element is moved unchanged.
 *   W1, W3: DEVICE [N,d,f]; W2: DEVICE [N,f,d]; contiguous, element type `dtype`.
 *   mode: BTX_MIX_SPLIT (C >= 1, f % C == 0, N*C <= 64) or BTX_MIX_BLEND (C ignored,
 *         f % N == 0).
 *   oW1, oW3: DEVICE [N*C,d,f/C] (split) or [N,d,f] (blend); oW2: [N*C,f/C,d] or
 *         [N,f,d].  Caller-owned, must not be the input buffers.
 * Errors: BTX_ERR_INVALID_ARG (NULL or aliased pointers, bad mode or chunk count),
 * BTX_ERR_HIP. */
typedef enum { BTX_MIX_SPLIT = 0, BTX_MIX_BLEND = 1 } btx_mix_mode;
int btx_mix_experts(const void* W1, const void* W3, const void* W2, int dtype, int N, int d, int f, int mode, int C,
                    void* oW1, void* oW3, void* oW2, void* stream);

/* ---------------------------------------------------------------------------
 * btx_adamw_step - fused AdamW update (Sec. 4.1: "AdamW optimizer with weight decay
 * 0.1"; the moment decay rates and eps are not stated and are arguments), for the
 * weight gradients btx_moe_ff_backward returns:
 *   m <- beta1 m + (1-beta1) g;  v <- beta2 v + (1-beta2) g^2
 *   p <- p - lr * ( (m/(1-beta1^step)) / (sqrt(v/(1-beta2^step)) + eps) + weight_decay * p )
 * in fp32, elementwise, in place.
 *   master, m, v  DEVICE [numel] fp32, 16-byte aligned: master weights and moments
 *   grad          DEVICE [numel] grad_dtype (BTX_BF16 or BTX_F32), 16-byte aligned
 *   lowp          DEVICE [numel] bf16, 8-byte aligned, may be NULL: receives the updated
 *                 weights rounded once to bf16 (the copy the layer's GEMMs read)
 *   step          1-based count of updates, for the bias corrections
 *   lr, beta1, beta2, eps, weight_decay: floats; the arithmetic runs on the float values as
 *                 passed (1 - 0.999f is 1.3e-5 relative away from 0.001)
 * Errors: BTX_ERR_INVALID_ARG (NULL / misaligned pointers, step < 1, beta outside [0,1),
 * negative eps), BTX_ERR_HIP. */
int btx_adamw_step(float* master, float* m, float* v, const void* grad, int grad_dtype, void* lowp, int64_t numel,
                   int step, float lr, float beta1, float beta2, float eps, float weight_decay, void* stream);

/* ---------------------------------------------------------------------------
 * btx_moe_group_route - routing from logits, for mixtures of many experts: softmax or sigmoid
 * scores, a bias that balances the experts' loads and that only the selection sees, groups of
 * experts of which the best are kept, top-k, renormalised and scaled gates; then the same token ->
 * expert grouping as btx_moe_route's, so that btx_moe_ff_forward_mx4 takes its outputs, and up to 64
 * experts btx_moe_ff_forward and btx_moe_ff_backward_gates do (they refuse more: beyond that there
 * is no layer to train).
 *     s = sigmoid(l) or softmax(l)                      (of a token's E logits l)
 *     v = s + bias                                      (bias NULL: s)
 *     a group's value = its largest v, or the sum of its two largest; the topk_groups groups of the
 *     largest values are kept; the k experts of the largest v in them are chosen
 *     gates_j = scale * s_j / (sum_j s_j + 1e-20)       (renorm 0: scale * s_j)
 *
 *   logits     [T,E]   logits_dtype (BTX_F32 or BTX_BF16): the router's product, made by the caller
 *   bias       [E]     fp32, may be NULL
 *   score_fn           btx_score_fn
 *   n_groups           groups of E / n_groups consecutive experts; 1: no groups
 *   topk_groups        groups kept, 1 <= topk_groups <= n_groups
 *   group_score        btx_group_score (ignored with one group)
 * The selection is that of v and of the groups' values in double precision (what differs by no more than its
 * own rounding may go either way); ties go to the lower index; topk_idx lists the chosen experts by descending
 * v. A logit of -inf masks its expert: its score is 0 and it is chosen only where the kept groups have fewer
 * than k others (TOP2 adds nothing for a masked one; a group of masked experts only is behind all others). A
 * NaN logit counts as -inf, +inf as the largest float; whatever the logits hold, a token's experts are in
 * range and distinct.
 * Outputs
 *   topk_idx   [T,k]   int32 expert ids
 *   gates      [T,k]   fp32
 *   scores     [T,E]   fp32 s, may be NULL
 *   counts, offsets, perm, inv_pos: as btx_moe_route's (without a capacity limit)
 * Requirements: E <= 256, n_groups <= 16, n_groups divides E, 1 <= k <= min(16, topk_groups * E / n_groups);
 * T*k < 2^30; scale finite.  workspace >= btx_moe_group_route_workspace_bytes(T,E,k) (16-byte aligned; may be NULL
 * where that is 0, which it is up to 64 tokens).
 */
typedef enum { BTX_SCORE_SOFTMAX = 0, BTX_SCORE_SIGMOID = 1 } btx_score_fn;
typedef enum { BTX_GROUP_MAX = 0, BTX_GROUP_TOP2 = 1 } btx_group_score;
size_t btx_moe_group_route_workspace_bytes(int T, int E, int k);
int btx_moe_group_route(const void* logits, int logits_dtype, const float* bias, int T, int E, int k, int score_fn,
                        int n_groups, int topk_groups, int group_score, int renorm, float scale, int32_t* topk_idx,
                        float* gates, float* scores, int32_t* counts, int32_t* offsets, int32_t* perm, int32_t* inv_pos,
                        void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * btx_moe_group_route_backward - gradient of the logits from those of the gates (and of the scores),
 * with the selection held fixed; the bias has none.
 *   logits, score_fn, renorm, scale: as given to btx_moe_group_route;  topk_idx [T,k] as it wrote them
 *   dgates   [T,k]  fp32
 *   dscores  [T,E]  fp32, may be NULL: gradient that reaches the scores directly (an auxiliary loss)
 *   dlogits  [T,E]  logits_dtype, out; may alias logits
 * A masked expert's gradient is 0, and its dgates and dscores go into no other one, whatever they hold.  Entries of
 * topk_idx outside 0..E-1 are passed over.
 * Requirements: as btx_moe_group_route, T <= 2^28 - 16 (BTX_ERR_UNSUPPORTED); no workspace.
 */
int btx_moe_group_route_backward(const void* logits, int logits_dtype, const int32_t* topk_idx, const float* dgates,
                                 const float* dscores, int T, int E, int k, int score_fn, int renorm, float scale,
                                 void* dlogits, void* stream);

/* ---------------------------------------------------------------------------
 * btx_moe_ff_backward_gates - btx_moe_ff_backward for gates of another router than btx_moe_route's: the
 * gradients of <dY, out> with respect to the gates, x and the experts' weights.  What the router adds to
 * x's gradient is the caller's (for btx_moe_group_route: dlogits W_router^T).
 *   dX     [T,d]  dtype  out: through the experts alone
 *   dgates [T,k]  fp32   out: <dY[t], FF_{idx[t,j]}(x[t])>; 0 for a dropped pair
 * The other arguments, limits (E <= 64 among them) and the workspace's size as btx_moe_ff_backward's;
 * T <= 2^26 - 4 (BTX_ERR_UNSUPPORTED).
 */
int btx_moe_ff_backward_gates(const void* dY, const void* x, const void* W1, const void* W3, const void* W2, int dtype,
                              int64_t w13_expert_stride, int64_t w2_expert_stride, int T, int d, int f, int E, int k,
                              const float* gates, const int32_t* offsets, const int32_t* perm, const int32_t* inv_pos,
                              const void* save_h1, const void* save_h3, void* dX, float* dgates, void* dW1, void* dW3,
                              void* dW2, int dW_dtype, void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Microscaled 4-bit floats (MXFP4): values 0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives (e2m1), of which 32
 * consecutive ones along the quantised axis (of length K) share a power of two (e8m0).
 *   codes   [.., n, K/2]   uint8: element 2i of a row in the low half of byte i, element 2i+1 in the high half
 *   scales  [.., n, btx_mx4_scale_pitch(K)]   uint8: byte b stands for 2^(b-127), 255 for NaN; the K/32 scales of a
 *           row, then zeros up to a multiple of 16 bytes
 * btx_mx4_quantize: a block's scale is 2^(floor(log2 of its largest magnitude) - 2), at least 2^-127; its values divided
 * by that are rounded to the nearest code, ties to the even one, and saturate at 6.  A block that holds an infinity or a NaN gets
 * the scale 255: all its values are NaN.
 * btx_mx4_dequantize: code value * scale, exact in fp32 and, down to 2^-133, in bf16.
 *   x, out  [batch, rows, cols]  dtype (BTX_F32 or BTX_BF16)
 *   axis    1: blocks along the rows: K = cols, n = rows (activations: [T,d] with batch 1)
 *           0: blocks down the columns: K = rows, n = cols; codes and scales are [batch, cols, ..].  So are the
 *              experts' weights quantised whose products sum over their rows: W1, W3 [E,d,f] and W2 [E,f,d].
 * Requirements: K a multiple of 32, n >= 0, batch >= 0 (nothing to do where one of them is 0); x, out, codes, scales on
 * 16-byte boundaries.  batch * rows * cols < 2^40.  axis 0: batch <= 65535, cols <= 4194240 and
 * ceil(rows / 256) * ceil(cols / 64) < 2^24 (BTX_ERR_UNSUPPORTED).
 */
int64_t btx_mx4_scale_pitch(int64_t K);
int btx_mx4_quantize(const void* x, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, uint8_t* codes,
                     uint8_t* scales, void* stream);
int btx_mx4_dequantize(const uint8_t* codes, const uint8_t* scales, int dtype, int64_t batch, int64_t rows, int64_t cols,
                       int axis, void* out, void* stream);

/* ---------------------------------------------------------------------------
 * btx_moe_ff_forward_mx4 - the layer of 4-bit experts, for serving (forward only): btx_moe_ff_forward with both
 * operands of every product in microscaled 4-bit floats.  Token rows are quantised along d once each; per expert
 *     act = silu(xq W1_e) * (xq W3_e)   (fp32 sums), quantised along f from its fp32 values;   y = actq W2_e, rounded to bf16
 *     (but for sums that are cut into ranges, which stay in fp32)
 *     out[t] = residual[t] + sum_j gates[t,j] * y            as in btx_moe_ff_forward
 *   x [T,d] bf16;  residual [T,d] bf16, may be NULL;  out [T,d] bf16; aliasing as in btx_moe_ff_forward
 *   W1, W3: codes [E,f,d/2] and scales [E,f,btx_mx4_scale_pitch(d)];  W2: [E,d,f/2] and [E,d,btx_mx4_scale_pitch(f)], as
 *   btx_mx4_quantize (axis 0) writes them
 *   gates, offsets, perm, inv_pos: as written by btx_moe_route or btx_moe_group_route
 * Requirements: d % 32 == 0, f % 32 == 0, 1 <= k <= E <= 256, T <= 2^26 - 4, T*k < 2^28 - 256, T*k*max(d,f) < 2^40,
 * E*d*f < 2^40; x, residual, out, the weights and the workspace on 16-byte boundaries. d and f <= 2097120, T *
 * btx_mx4_scale_pitch(d) < 2^30 (BTX_ERR_UNSUPPORTED).
 */
size_t btx_moe_ff_forward_mx4_workspace_bytes(int T, int d, int f, int E, int k);
int btx_moe_ff_forward_mx4(const void* x, const uint8_t* W1_codes, const uint8_t* W1_scales, const uint8_t* W3_codes,
                           const uint8_t* W3_scales, const uint8_t* W2_codes, const uint8_t* W2_scales, int T, int d, int f,
                           int E, int k, const float* gates, const int32_t* offsets, const int32_t* perm,
                           const int32_t* inv_pos, const void* residual, void* out, void* workspace,
                           size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Block-scaled 8-bit floats: e4m3 values (3 bits of fraction, largest 448, smallest 2^-9), of which 128 consecutive ones along the quantised axis
 * (of length K) share a power of two (e8m0).  For serving: btx_rmsnorm_fp8 or btx_fp8_quantize makes the rows, btx_moe_ff_forward_fp8 and
 * btx_fp8_matmul multiply them with weights that were quantised once.  For training a linear layer y = x W^T, all three products are
 * btx_fp8_matmul's: y of x and W; dx of dy and W^T; dW of dy^T and x^T (quantised with axis 0).
 *   codes   [.., n, btx_fp8_code_pitch(K)]    uint8, one an element, zeros from K up to a multiple of 128
 *   scales  [.., n, btx_fp8_scale_pitch(K)]   uint8: byte b stands for 2^(b-127), 255 for NaN; the ceil(K/128) scales of a row, then zeros up
 *           to a multiple of 16 bytes
 * btx_fp8_quantize: a block's scale is the smallest power of two, at least 2^-127, of which its largest magnitude is at most 448 times; its values
 * divided by that are rounded to the nearest e4m3 value, ties to the even one.  A block that holds an infinity or a NaN gets the scale
 * 255: all its values are NaN.
 * btx_fp8_dequantize: value of the code * scale, exact in fp32, and down to 2^-133 in bf16; from 2^128 on an infinity (as fp32 values from 248 * 2^120 on are
 * quantised to).
 *   x, out      [batch, rows, cols]  dtype (BTX_F32 or BTX_BF16)
 *   axis        1: blocks along the rows: K = cols, n = rows (activations: [T,d] with batch 1)
 *               0: blocks down the columns: K = rows, n = cols; codes and scales are [batch, cols, ..].  So are the experts' weights
 *                  quantised whose products sum over their rows: W1, W3 [E,d,f] and W2 [E,f,d].
 *   block_rows  1: a block is 128 elements along K.  128: blocks of 128 x 128 elements, whose scale each of the 128 rows has: a matrix and its
 *               transpose (the other axis) then have the same values.
 * K, n and batch may be any sizes (nothing to do where one of them is 0); x, out, codes, scales on 16-byte boundaries.
 * batch * n * btx_fp8_code_pitch(K) < 2^40.  axis 0 or block_rows 128: batch <= 65535, ceil(rows / 128) * ceil(cols / 128) < 2^24
 * (BTX_ERR_UNSUPPORTED).
 */
int64_t btx_fp8_code_pitch(int64_t K);
int64_t btx_fp8_scale_pitch(int64_t K);
int btx_fp8_quantize(const void* x, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, int block_rows, uint8_t* codes,
                     uint8_t* scales, void* stream);
int btx_fp8_dequantize(const uint8_t* codes, const uint8_t* scales, int dtype, int64_t batch, int64_t rows, int64_t cols, int axis, void* out,
                       void* stream);

/* ---------------------------------------------------------------------------
 * btx_rmsnorm_fp8 - the residual's addition and the block's pre-normalisation, with the result in 8 bits:
 *     sum[t,c] = h[t,c] + residual[t,c], rounded to dtype;   rstd[t] = 1 / sqrt(mean_c sum[t,c]^2 + eps);
 *     xn[t,c] = gain[c] * sum[t,c] * rstd[t]
 *   h         [T,d]  dtype
 *   residual  [T,d]  dtype, may be NULL: sum is h
 *   gain      [d]    fp32;   eps >= 0
 *   sum       [T,d]  dtype  out, may be NULL; may be h or residual itself
 *   xn        [T,d]  dtype  out, may be NULL (a router reads it); must not be h, residual or sum
 *   rstd      [T]    fp32   out
 *   codes [T,btx_fp8_code_pitch(d)], scales [T,btx_fp8_scale_pitch(d)]: out, xn as btx_fp8_quantize (axis 1, block_rows 1) writes fp32 values: of xn before it
 *             is rounded to dtype.  Both NULL: xn alone.
 * Mean square, rstd and the product are evaluated in fp64, as by btx_moe_norm_route.  The backward pass is btx_rmsnorm_backward with `sum` in h's
 * place, rstd, and the gradient of sum as dres: its dH is that of h and of residual.
 * Requirements: d % 8 == 0; d <= 16384 (BTX_ERR_UNSUPPORTED); all but rstd on 16-byte boundaries.
 */
int btx_rmsnorm_fp8(const void* h, const void* residual, int dtype, const float* gain, float eps, int T, int d, void* sum, void* xn, float* rstd,
                    uint8_t* codes, uint8_t* scales, void* stream);

/* ---------------------------------------------------------------------------
 * btx_fp8_matmul - out[m,n] = residual[m,n] + sum_k A[m,k] B[n,k] of two matrices in block-scaled 8-bit floats: sums in fp32 in an order that the sizes
 * fix (the same bits every time), rounded once.  fp32 results: exact products (of values under 2^-126, those to bf16's precision there, and of infinities for
 * those from 2^128 on).  bf16 results: of every 8 neighbouring products what lies 13 bits or more below the largest is dropped before they are added up (2e-5
 * of the result's norm, where rounding it to bf16 is 1.7e-3), in up to twice the rate.
 *   A         codes [M,btx_fp8_code_pitch(K)], scales [M,btx_fp8_scale_pitch(K)];   B: the same with N rows
 *   residual  [M,N]  dtype, may be NULL; may be out itself (a gradient that is added to)
 *   out       [M,N]  dtype (BTX_F32 or BTX_BF16)
 * What lies behind K in the codes' rows has to be zeros, as btx_fp8_quantize writes them.
 * Requirements: N % 8 == 0, K >= 1, M * max(N, pitch) < 2^40, N * pitch < 2^40; M < 2^28 - 256, N and K <= 2097120, in fp32
 * ceil(M/128) * ceil(N/128) < 2^24 (BTX_ERR_UNSUPPORTED); everything on 16-byte boundaries; workspace >= btx_fp8_matmul_workspace_bytes(M,N,K) (may be NULL
 * where that is 0).
 */
size_t btx_fp8_matmul_workspace_bytes(int M, int N, int K);
int btx_fp8_matmul(const uint8_t* A_codes, const uint8_t* A_scales, const uint8_t* B_codes, const uint8_t* B_scales, int M, int N, int K,
                   const void* residual, void* out, int dtype, void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * btx_moe_ff_forward_fp8 - the layer of 8-bit experts, for serving (forward only): btx_moe_ff_forward with both operands of every product in block-scaled
 * 8-bit floats.  Per expert
 *     act = silu(x W1_e) * (x W3_e)   (fp32 sums), quantised along f from its fp32 values;   y = actq W2_e, rounded to bf16
 *     (but for up to 2^22 values, T*k*d of them, and for sums that are cut into ranges, which stay in fp32; with more than 8 experts a token, of 8192 tokens
 *     and more with more than 4, all are rounded)
 *     out[t] = residual[t] + sum_j gates[t,j] * y            as in btx_moe_ff_forward
 * Products as btx_fp8_matmul's: for act as its fp32 results' up to 64 rows an expert on average and in small layers, else as its bf16 ones', with which one
 * code in a few thousand is the neighbour of the one that exact sums have (out 2.1e-3 of its norm from the formula instead of 1.7e-3); for y as its bf16 ones'.
 *   x         codes [T,btx_fp8_code_pitch(d)] and scales [T,btx_fp8_scale_pitch(d)], as btx_rmsnorm_fp8 or btx_fp8_quantize (axis 1) writes them
 *   W1, W3    codes [E,f,btx_fp8_code_pitch(d)] and scales [E,f,btx_fp8_scale_pitch(d)];   W2: [E,d,btx_fp8_code_pitch(f)] and
 *             [E,d,btx_fp8_scale_pitch(f)], as btx_fp8_quantize (axis 0; any block_rows) writes them
 *   residual  [T,d] bf16, may be NULL;   out [T,d] bf16;   residual may be out
 *   gates, offsets, perm, inv_pos: as written by btx_moe_route or btx_moe_group_route
 * Requirements: d % 8 == 0, f % 8 == 0, 1 <= k <= E <= 256, T <= 2^26 - 4, T*k < 2^28 - 256, T*k*max(pitches) < 2^40,
 * E*max(f*btx_fp8_code_pitch(d), d*btx_fp8_code_pitch(f)) < 2^40; codes, scales, residual, out and the workspace on 16-byte boundaries.
 * d and f <= 2097120, T*btx_fp8_code_pitch(d) <= 2^32 - 2048 (BTX_ERR_UNSUPPORTED).
 */
size_t btx_moe_ff_forward_fp8_workspace_bytes(int T, int d, int f, int E, int k);
int btx_moe_ff_forward_fp8(const uint8_t* x_codes, const uint8_t* x_scales, const uint8_t* W1_codes, const uint8_t* W1_scales,
                           const uint8_t* W3_codes, const uint8_t* W3_scales, const uint8_t* W2_codes, const uint8_t* W2_scales, int T, int d, int f,
                           int E, int k, const float* gates, const int32_t* offsets, const int32_t* perm, const int32_t* inv_pos, const void* residual,
                           void* out, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* BTX_MOE_H */
