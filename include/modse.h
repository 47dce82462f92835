/*
 * modse.h - C ABI of the MoDSE (Mixture of Diverse Size Experts) feed-forward
 * layer for NVIDIA B200 (sm_100a).
 *
 * The layer is the one of "Mixture of Diverse Size Experts" (arXiv 2409.12210):
 *   gate     G(x) = Softmax(KeepTopK(H(x), k)),  H(x) = x . W_g      (Sec. 2, Eq. 2-3)
 *   output   y    = sum_i G_i(x) E_i(x)                               (Sec. 3.1, Eq. 4)
 * where expert E_i is a bias-free SwiGLU feed-forward block (the Llama-2 FFN
 * the paper's models are built on, Sec. 4.1) whose hidden width h_i differs
 * from expert to expert (Sec. 3.1).  Experts outside the top-k have gate
 * softmax(-inf) = 0 and are never evaluated; every token is served by exactly
 * k experts (no capacity limit, no dropped tokens).
 *
 * Notation: T tokens, d = d_model, N experts, k = top_k, h[e] = hidden width of
 * expert e, S = sum_e h[e], off[e] = sum_{e'<e} h[e'].
 *
 * All pointers named "device" are CUDA device pointers owned by the caller.
 * The library allocates no device memory; every call only enqueues kernels on
 * the given stream and returns without synchronising.  No exception crosses
 * this boundary and no call aborts: errors are returned as modse_status_t.
 */
#ifndef MODSE_H
#define MODSE_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct modse_layer modse_layer_t; /* opaque host object owned by the library */

typedef enum {
    MODSE_OK = 0,
    MODSE_ERR_INVALID_ARG = 1,         /* NULL/misaligned pointer, size out of range            */
    MODSE_ERR_UNSUPPORTED = 2,         /* legal layer the CUDA path cannot run (see modse_create) */
    MODSE_ERR_WORKSPACE_TOO_SMALL = 3, /* workspace_bytes < modse_workspace_bytes(...)           */
    MODSE_ERR_STATE = 4,               /* backward without a matching saved forward              */
    MODSE_ERR_CUDA = 5,                /* a CUDA runtime/driver call or launch failed            */
    MODSE_ERR_DEVICE_TIMEOUT = 6,      /* a bounded wait inside a kernel expired                 */
    MODSE_ERR_DEVICE_BOUNDS = 7        /* a kernel met an index outside its buffers              */
} modse_status_t;

typedef enum {
    MODSE_F32 = 0, /* fp32 storage, fp32 FMA arithmetic                                   */
    MODSE_BF16 = 1, /* bf16 storage, tensor-core products with fp32 accumulation          */
    MODSE_E4M3 = 2  /* 8-bit operands of modse_linear (e4m3 with a scale a row); no layer */
} modse_dtype_t;

/* ---- layer object ------------------------------------------------------- */

/* Describes a layer (Sec. 3.1): d_model, N experts with hidden widths
 * ffn_sizes[0..N) (copied), and k.  Host only; touches no GPU.
 * Requirements: d_model >= 8 and a multiple of 8; 1 <= n_experts <= 256;
 * 1 <= top_k <= n_experts; every width >= 16 and a multiple of 16.
 * top_k > 2 is a legal layer the CUDA path does not run (MODSE_ERR_UNSUPPORTED).
 * The bf16 type further needs d_model % 128 == 0 and every width % 64 == 0
 * (checked by forward/backward, MODSE_ERR_UNSUPPORTED).
 * The pair rule of Eq. 5-6 is not enforced (query it with modse_check_pairs).
 * Returns NULL on error; modse_last_create_error() says why.                 */
modse_layer_t *modse_create(int d_model, int n_experts, const int *ffn_sizes, int top_k);
modse_status_t modse_last_create_error(void); /* per calling thread */
modse_status_t modse_destroy(modse_layer_t *layer); /* NULL is accepted */

/* Sec. 3.1, Eq. 5-6: returns 1 iff n_experts is even and every adjacent pair
 * (2p, 2p+1) - the pairs that the expert-pair allocation of Sec. 3.2 places on
 * one GPU each - has the same width sum 2h; *pair_sum_out (may be NULL) gets it. */
int modse_check_pairs(const int *ffn_sizes, int n_experts, int *pair_sum_out);

const char *modse_status_string(modse_status_t status);

/* ---- tensors ------------------------------------------------------------ */

/* Weights, all row-major in the layer dtype, 16-byte aligned device pointers:
 *   w_router [N, d]   row i gives logit i of H(x) = x . W_g             (Eq. 2)
 *   w_gate   [S, d]   rows off[e] .. off[e]+h[e]-1 belong to expert e
 *   w_up     [S, d]   same
 *   w_down   [d, S]   columns off[e] .. off[e]+h[e]-1 belong to expert e
 * Expert e computes  E_e(x) = W_down_e (silu(W_gate_e x) * (W_up_e x)).      */
typedef struct {
    const void *w_router;
    const void *w_gate;
    const void *w_up;
    const void *w_down;
} modse_weights_t;

/* Weight gradients, same shapes and layouts; dw_router is always fp32, the
 * others are in the layer dtype.  Overwritten (not accumulated) by backward;
 * rows/columns of an expert that received no token are written as zeros.    */
typedef struct {
    void *dw_router;
    void *dw_gate;
    void *dw_up;
    void *dw_down;
} modse_wgrads_t;

/* ---- calls -------------------------------------------------------------- */

/* Bytes of device scratch a forward (and its backward, if save_for_backward)
 * needs for n_tokens tokens.  0 on bad arguments.  The buffer must be 256-byte
 * aligned and is owned by the caller; its content after forward holds the
 * routing tables and, if saved, the activations backward consumes.           */
size_t modse_workspace_bytes(const modse_layer_t *layer, modse_dtype_t dtype, int n_tokens,
                             int save_for_backward);

/* Eq. 2-4.  x [T, d] and y [T, d] device, layer dtype, row-major.
 * Steps, all on `cuda_stream` (a cudaStream_t, NULL = legacy default stream):
 * router logits + top-k + gates, per-expert counts/offsets and the stable
 * permutation (expert groups ascending, tokens ascending inside a group),
 * gather into expert groups, grouped up/gate projection with SwiGLU, grouped
 * down projection, gate-weighted sum back in token order (slot 0 then slot 1).
 * n_tokens == 0 is MODSE_OK and does nothing.                                */
modse_status_t modse_forward(modse_layer_t *layer, modse_dtype_t dtype, const modse_weights_t *weights,
                             const void *x, int n_tokens, void *y, void *workspace,
                             size_t workspace_bytes, int save_for_backward, void *cuda_stream);

/* The same function for the few tokens of a generation step, at most
 * MODSE_DECODE_MAX_TOKENS (more: MODSE_ERR_UNSUPPORTED; modse_forward takes any number):
 * two kernels that stream the weights of the experts met once, where modse_forward lays
 * tokens out in groups of 128 rows.  Any layer that modse_create accepts (d and widths to 2^26), in either dtype;
 * the second router term (modse_set_noise_gate) and fp32 outputs (modse_set_output_f32) as
 * in modse_forward.  topk_idx and topk_gate [T, k] (each may be NULL) receive the routing.
 * Sums are fp32, in an order that does not depend on the run but is not modse_forward's: values agree to
 * rounding, and so do the logits, so that a token whose k-th and k+1-st logits are equal to their last
 * bits may be routed differently (equal logits: the lower index in both).  A logit that is NaN counts as the largest, the
 * lower index first: the token's gates and its row of y are NaN (modse_forward may pass such an expert over).
 * The layer object is only read: calls on several streams may share it, with a workspace
 * each (256-byte aligned; its size never falls with n_tokens).  It takes no part in
 * modse_backward, modse_get_routing, stage timing and launch counts.  y overlaps no input.
 * The workspace's first bytes hold a status word that modse_check_workspace_status reads. */
#define MODSE_DECODE_MAX_TOKENS 32
size_t modse_decode_workspace_bytes(const modse_layer_t *layer, modse_dtype_t dtype, int n_tokens);
modse_status_t modse_decode(const modse_layer_t *layer, modse_dtype_t dtype, const modse_weights_t *weights, const void *x,
                            int n_tokens, void *y, int *topk_idx, float *topk_gate, void *workspace, size_t workspace_bytes,
                            void *cuda_stream);

/* Exact gradient of modse_forward with the top-k selection held fixed (the
 * selection is piecewise constant in x).  Needs the workspace of a preceding
 * modse_forward(..., save_for_backward=1) on the same layer object, dtype and
 * n_tokens (else MODSE_ERR_STATE) and the same x and weights.  dy [T, d] is
 * the upstream gradient, dx [T, d] the result (layer dtype).  Gate and router
 * gradients are computed and kept in fp32.  May be called repeatedly on one
 * saved forward.                                                             */
modse_status_t modse_backward(modse_layer_t *layer, modse_dtype_t dtype, const modse_weights_t *weights,
                              const void *x, const void *dy, int n_tokens, void *dx,
                              const modse_wgrads_t *wgrads, void *workspace, size_t workspace_bytes,
                              void *cuda_stream);

/* Device pointers to the routing tables inside `workspace`, valid after a
 * forward with the same layer/n_tokens until the workspace is reused.  Any
 * output pointer may be NULL.  (Per-slot counts are what the paper's Appendix A
 * tables list as "top0"/"top1".)
 *   topk_idx [T,k] int32 (slot 0 = largest logit; ties go to the lower index)
 *   topk_gate [T,k] fp32, counts [N], counts_slot [k,N], offsets [N+1],
 *   row_of [T,k] (row of assignment (t,j) in expert-grouped order),
 *   token_of [k*T] (inverse map)                                             */
modse_status_t modse_get_routing(const modse_layer_t *layer, const void *workspace, int n_tokens,
                                 const int **topk_idx, const float **topk_gate, const int **counts,
                                 const int **counts_slot, const int **offsets, const int **row_of,
                                 const int **token_of);

/* Device pointers to the fp32 gate gradients dg [T,k] and logit gradients of
 * the kept logits dz [T,k] written by modse_backward.                        */
modse_status_t modse_get_gate_grads(const modse_layer_t *layer, const void *workspace, int n_tokens,
                                    const float **dg, const float **dz);

/* Synchronises the stream and reads the status word kernels write when a
 * bounded wait expires (MODSE_ERR_DEVICE_TIMEOUT) or an index check fails
 * (MODSE_ERR_DEVICE_BOUNDS); MODSE_OK if none did.  The word is cleared by the
 * next modse_forward.  Index checks are always on: every kernel that follows a
 * row or token index read from the routing tables compares it with the table's
 * extent first and skips the access if it lies outside.
 *
 * modse_set_debug_checks(layer, 1) (or the environment variable MODSE_DEBUG=1
 * at modse_create) adds guard blocks: every region of the workspace is followed
 * by 256 spare bytes whose head modse_forward fills with a pattern and this
 * call compares; a kernel that wrote past its region turns up as
 * MODSE_ERR_DEVICE_BOUNDS.  (The blocks are part of modse_workspace_bytes in
 * either mode.)  No counterpart in the paper.                                */
modse_status_t modse_check_device_status(modse_layer_t *layer, const void *workspace, void *cuda_stream);
modse_status_t modse_set_debug_checks(modse_layer_t *layer, int on);

/* Number of kernel launches the last forward/backward call on this layer
 * enqueued (for launch accounting in benchmarks).                            */
int modse_last_launch_count(const modse_layer_t *layer);

/* Auxiliary load-balance loss of Sec. 3.2, Eq. 7-10 (the Switch-Transformer loss):
 *   L_a = alpha * N * sum_i f_i * P_i,
 * p(x) = softmax over all N router logits, f_i = fraction of tokens whose largest
 * probability is expert i (Eq. 8; equals the slot-0 count / T), P_i = mean of p_i
 * over the batch (Eq. 10).
 *
 * modse_aux_loss evaluates it for the batch of the last modse_forward on this layer
 * and workspace: loss (1 float), f [N] and P [N] are device pointers written on the
 * stream (f and P may be NULL).
 *
 * modse_set_aux_loss(alpha) makes the following modse_backward calls differentiate
 * the objective  sum(dy * y) + L_a : dx and dw_router receive, in addition,
 * dL_a/dz[t,m] = (alpha N / T) p_m (f_m - sum_i f_i p_i) for every expert m (f is
 * piecewise constant and is held fixed).  alpha = 0 (default) switches it off.
 * The fp32 dz returned by modse_get_gate_grads stays the layer-output part only. */
modse_status_t modse_aux_loss(modse_layer_t *layer, const void *workspace, int n_tokens, float alpha, float *loss,
                              float *f, float *P, void *cuda_stream);
modse_status_t modse_set_aux_loss(modse_layer_t *layer, float alpha);

/* Output precision of a bf16 layer.  Off (default): y, dx and the expert weight
 * gradients are bf16 like the inputs.  On: the same fp32 accumulators are
 * written as fp32 instead ([T,d] y and dx, [S,d]/[d,S] weight gradients of 4
 * bytes per element), which removes the last bf16 rounding - e.g. for gradient
 * accumulation over micro-batches in fp32.  No effect on fp32 layers.        */
modse_status_t modse_set_output_f32(modse_layer_t *layer, int on);

/* Choice of kernel shape per device (no counterpart in the paper: a property of this implementation).
 * Each grouped product of the bf16 layer exists with 128-row tiles, with 256-row tiles computed by one CTA and
 * with 256-row tiles computed by a pair of CTAs; which is fastest for the two forward products depends on how
 * fast the GPU at hand feeds shared memory from L2, which differs between otherwise identical boards.
 * modse_tune_forward runs the forward pass (arguments as modse_forward) a few times per candidate on the caller's own buffers, times it with CUDA events, and keeps the fastest plan in
 * the layer object for all later calls.  It allocates no device memory, SYNCHRONISES the stream, and leaves y
 * and the workspace as one modse_forward would.  Results do not depend on the plan (the K order of every sum
 * is the same).  fp32 layers have one kernel shape: the call returns MODSE_OK at once.
 * The plan it finds is the fastest for forward passes run on their own (serving); inside a training step the
 * stages share the GPU's power budget and the library default (CTA pairs for every product) has been the faster
 * choice on every board measured, so training code need not call it.
 * modse_get_tile_plan returns the plan: -1 for the library default, else a bit set with, for product k (0 up/gate,
 * 1 down, 2 down dgrad, 3 down wgrad, 4 up/gate dgrad, 5 up/gate wgrad), bit 8 + k set: 256-row tiles computed
 * by a pair of CTAs on neighbouring SMs; otherwise bit k set: 256-row tiles computed by one CTA, clear: 128-row
 * tiles.  modse_set_tile_plan installs one (e.g. a plan found earlier on the same device). */
modse_status_t modse_tune_forward(modse_layer_t *layer, modse_dtype_t dtype, const modse_weights_t *weights,
                                  const void *x, int n_tokens, void *y, void *workspace, size_t workspace_bytes,
                                  int save_for_backward, void *cuda_stream);
int modse_get_tile_plan(const modse_layer_t *layer);
modse_status_t modse_set_tile_plan(modse_layer_t *layer, int plan);

/* Fusions across the permutation (bf16 layers; Sec. 2 Eq. 1 and Sec. 3.1 Eq. 4 say "select the top-k experts
 * and combine their outputs" and fix no intermediate buffers).  `flags` is a sum of
 *   MODSE_FUSE_GATHER   the up/gate product gathers its rows from x through the permutation (TMA row gather)
 *                       instead of reading the grouped copy of x; a forward that saves nothing for backward
 *                       then skips the permute kernel altogether;
 *   MODSE_FUSE_DG_ROWDOT  the gate gradient dg[t,j] = <dY_t W_down_e, Hm_row> / g is accumulated inside the
 *                       down-dgrad epilogue (one partial per 128 columns, summed in column order), so
 *                       backward no longer reads the fp32 expert outputs o;
 *   MODSE_FUSE_SCATTER  with fp32 outputs (modse_set_output_f32) and top_k <= 2: the down product adds its
 *                       rows straight into y and the up/gate dgrad into dx (both zeroed first; two addends
 *                       into a zeroed element commute, so the result is the same bits in any order), the
 *                       buffers o and dxp and the combine pass disappear; implies MODSE_FUSE_DG_ROWDOT.
 * A flag that does not apply to a call (fp32 layer, bf16 outputs, top_k > 2) is ignored by that call.
 * A backward call follows the forward call it belongs to.  Results: GATHER and SCATTER give the same bits as
 * the unfused path; DG_ROWDOT sums dg in another order (same tolerance).  Default: none.              */
#define MODSE_FUSE_GATHER 1
#define MODSE_FUSE_DG_ROWDOT 2
#define MODSE_FUSE_SCATTER 4
modse_status_t modse_set_fusion(modse_layer_t *layer, int flags);
int modse_get_fusion(const modse_layer_t *layer);

/* Second term of the router logits (Sec. 2, Eq. 2 with the RMSNorm and Softplus
 * definitions that follow it):
 *   H(x)_i = (x W_g)_i + RMSNorm(Softplus((x W_n)_i)),
 *   RMSNorm(v)_i = gamma v_i / sqrt(mean_j v_j^2 + eps),
 * read as: W_n is a second [N,d] router matrix, the mean runs over the N expert
 * entries of a token, gamma is one learnable scalar.  The term is a function of
 * x alone (the paper draws no random number here), so it is simply part of the
 * logits that top-k, the gates, the auxiliary loss and the backward pass see.
 *
 * modse_set_noise_gate: w_noise is a DEVICE pointer to [N,d] in the layer's
 * dtype, 16-byte aligned, borrowed until it is replaced (it must stay valid for
 * every later forward/backward); NULL switches the term off (the default).
 * gamma any finite value, eps >= 0.
 * modse_set_noise_grads: where modse_backward writes dW_n ([N,d] fp32, device,
 * 16-byte aligned) and dgamma (one fp32, device); both overwritten.  Required
 * before a backward whose forward ran with the term on (else
 * MODSE_ERR_INVALID_ARG); a backward whose on/off state differs from its
 * forward's returns MODSE_ERR_STATE.
 * dx and the router gradients then include the term's contribution; every sum
 * has a fixed order as elsewhere.                                            */
modse_status_t modse_set_noise_gate(modse_layer_t *layer, const void *w_noise, float gamma, float eps);
modse_status_t modse_set_noise_grads(modse_layer_t *layer, float *dw_noise, float *dgamma);

/* Routing only, with no device allocation by anyone.  (The paper has no
 * counterpart: this is a packaging variant of the router stage of Eq. 2-3.)
 *
 * For callers that cannot allocate device memory - a plugin invoked from a
 * framework callback where cudaMalloc is off limits because it synchronises
 * the device and can fail mid-step, code living inside a memory pool it does
 * not own, or a tool that only wants the routing tables - the scratch of the
 * router and rank kernels lives in a fixed 4 MiB array inside the library
 * (every GPU that loads the library holds it until the process exits).  The
 * caller passes only inputs and outputs, all device pointers:
 *   x [T,d], w_router [N,d]  in `dtype`, 16-byte aligned
 *   topk_idx [T,k] int32, topk_gate [T,k] fp32, counts [N], counts_slot [k,N],
 *   offsets [N+1], row_of [T,k], token_of [k*T]  - same meaning and the same
 *   values as modse_get_routing after modse_forward.
 * Limits: the scratch must fit the array - about 4*k*T*3 + 1016*N bytes plus
 * k*N*4 bytes per 64 tokens, e.g. T <= 100000 tokens for 8 experts, top-2;
 * larger batches return MODSE_ERR_WORKSPACE_TOO_SMALL (nothing is launched).
 * modse_route_static_scratch_capacity() returns the array size in bytes.
 * The first call on each device looks up the array's device address (a host
 * call, no allocation); make that first call before any stream capture.
 * All calls share the one array and it keeps the last call's contents (the
 * call clears what must start at zero): two calls that overlap on the GPU -
 * different streams, or different host threads - race on it; serialise them.
 * Calls no cudaMalloc/cudaFree and no allocating library routine.
 * The array's device address is cached per process and per device context:
 * serialise the first calls of several host threads, and do not use the
 * library across a cudaDeviceReset.
 * modse_route_static_scratch_status synchronises `cuda_stream` and returns what
 * the kernels of the last call on the current device recorded in the array's
 * status word (MODSE_OK, MODSE_ERR_DEVICE_BOUNDS, MODSE_ERR_DEVICE_TIMEOUT);
 * it plays the part of modse_check_device_status, which needs a workspace.   */
modse_status_t modse_route_static_scratch(modse_dtype_t dtype, int d_model, int n_experts, int top_k,
                                          const void *x, const void *w_router, int n_tokens, int *topk_idx,
                                          float *topk_gate, int *counts, int *counts_slot, int *offsets,
                                          int *row_of, int *token_of, void *cuda_stream);
size_t modse_route_static_scratch_capacity(void);
modse_status_t modse_route_static_scratch_status(void *cuda_stream);

/* Per-stage device timing (profiling aid).  After modse_stage_timing_begin the
 * next max_calls forward/backward calls on this layer bracket each of their
 * stages with a pair of CUDA events on the call's stream (no work is skipped
 * or reordered).  modse_stage_timing_end waits for those events, writes
 * ms_out[call * MODSE_N_STAGES + stage] (milliseconds; -1 for a stage the call
 * did not run), the number of calls seen, and switches timing off again.
 * Stages 0-5 belong to forward (router, rank, permute, up/gate GEMM + SwiGLU,
 * down GEMM, combine), 6-11 to backward (dg + permute of dY, down dgrad +
 * SwiGLU backward, down wgrad, up/gate dgrad, up/gate wgrad, router backward). */
#define MODSE_N_STAGES 12
modse_status_t modse_stage_timing_begin(modse_layer_t *layer, int max_calls);
modse_status_t modse_stage_timing_end(modse_layer_t *layer, float *ms_out, int *calls_out);
const char *modse_stage_name(int stage);

/* ---- operators around the layer ------------------------------------------
 * What a transformer block needs on either side of modse_forward/backward.
 * None of them uses a layer object; tensors are row-major and contiguous unless
 * said otherwise, every pointer 16-byte aligned unless said otherwise, every
 * workspace 256-byte aligned and in use by one call at a time (two calls that may
 * overlap, or two captured graphs that may, need one each).  Outputs of a call do
 * not overlap one another.  Results do not depend on the order in which blocks run.  (The paper fixes none of them: its
 * blocks are Llama-2's, Sec. 4.1, whose pre-norm residual form this is.)      */

/* Residual addition and root-mean-square norm, the step that makes a sub-layer's
 * input (x of modse_forward) out of the residual stream and the previous
 * sub-layer's output:
 *   s = x + residual,  y = s / sqrt(mean_c(s_c^2) + eps) * weight,
 *   y_scale[t] = max_c |y_tc| / 448,  y_e4m3 = e4m3(y / y_scale).
 * x, residual, sum, y [T, d] and weight [d] in `dtype`; d a multiple of 8, at most
 * 32768 (else MODSE_ERR_UNSUPPORTED).  residual NULL: s = x; weight NULL: ones.
 * Outputs, each of them optional, at least one: sum (may be x or residual
 * itself), y, and y_e4m3 [T, d] bytes together with y_scale [T].  The norm is
 * taken from the fp32 sum, not from its rounding into `sum`; each output is
 * rounded once.  A row of zeros has scale 0 and zero bytes (with eps > 0); a row
 * that holds a NaN or an infinity has scale NaN.  Squares are summed in fp32:
 * magnitudes above 1e19 overflow the mean.                                   */
modse_status_t modse_add_rms_norm(modse_dtype_t dtype, int n_tokens, int d_model, const void *x, const void *residual,
                                  const void *weight, float eps, void *sum, void *y, void *y_e4m3, float *y_scale,
                                  void *cuda_stream);

/* Gradient of the above as a function of `sum` (as forward wrote it): dy [T, d] is
 * the gradient of y, dsum [T, d] (may be NULL) the one that reaches s past the
 * norm, along the residual stream;
 *   dx = rstd (u - s rstd^2 mean_c(u_c s_c)) + dsum,  u = dy weight,
 * is the gradient of x and of residual alike (dx may be dy or dsum itself);
 * dweight [d] fp32 (may be NULL, then no workspace is needed) = sum_t dy s rstd,
 * overwritten, summed in a fixed order.                                      */
size_t modse_add_rms_norm_backward_workspace_bytes(int n_tokens, int d_model);
modse_status_t modse_add_rms_norm_backward(modse_dtype_t dtype, int n_tokens, int d_model, const void *sum,
                                           const void *weight, float eps, const void *dy, const void *dsum, void *dx,
                                           float *dweight, void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Dense product with bias, activation and residual in its epilogue, for the
 * projections of the block the layer sits in:
 *   z = x w^T + bias,  y = act(z) + residual.
 * x [T, d_in], w [d_out, d_in], bias [d_out], residual and y [T, d_out], z [T, d_out].
 * MODSE_BF16: everything bf16.  MODSE_E4M3: x and w are e4m3 bytes with one fp32
 * scale a row each (x_scale [T], w_scale [d_out], e.g. from modse_add_rms_norm):
 * z = (x w^T) x_scale w_scale + bias; bias, residual, z and y are bf16.  MODSE_F32
 * is MODSE_ERR_UNSUPPORTED.  d_in a multiple of 8 (e4m3: 16), d_out of 8.
 * bias, residual and z may be NULL; y may be residual itself, otherwise outputs do
 * not overlap inputs.  z, what
 * modse_linear_backward reads, is rounded once from the fp32 value, and y, from
 * the unrounded z, once.  Products are accumulated in fp32.
 * relu, gelu (z Phi(z), Phi the normal distribution function), silu (z / (1 + e^-z)).
 * Infinities give the functions' limits, a NaN gives NaN.
 * The workspace's first bytes hold a status word that modse_check_workspace_status
 * reads (a bounded wait inside a kernel may expire, as in modse_forward).  Its size,
 * and that of the gradient's, never falls with n_tokens: one that serves a batch
 * serves every smaller one.                                                  */
typedef enum {
    MODSE_ACT_NONE = 0,
    MODSE_ACT_RELU = 1,
    MODSE_ACT_GELU = 2,
    MODSE_ACT_SILU = 3
} modse_activation_t;
typedef struct {
    const void *x, *w;
    const float *x_scale, *w_scale; /* MODSE_E4M3 only, else NULL */
    const void *bias, *residual;
    void *z, *y;
} modse_linear_t;
size_t modse_linear_workspace_bytes(modse_dtype_t dtype, int n_tokens, int d_in, int d_out);
modse_status_t modse_linear(modse_dtype_t dtype, int n_tokens, int d_in, int d_out, modse_activation_t activation,
                            const modse_linear_t *args, void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Gradient of the bf16 product, from dy [T, d_out] and the z that forward saved (may
 * be NULL for MODSE_ACT_NONE):
 *   dz = dy act'(z),  dx = dz w,  dw = dz^T x,  dbias = sum_t dz
 * (the residual's gradient is dy itself; relu'(0) = 0, and where relu's slope is 0
 * dz is 0 whatever dy holds).  dx [T, d_in] and
 * dw [d_out, d_in] bf16, dbias [d_out] fp32; each may be NULL, all overwritten, none
 * overlaps an input.  At most 4194240 tokens.
 * dz enters the products rounded to bf16 once (they read 16-bit operands) and
 * dbias unrounded.                                                           */
typedef struct {
    const void *x, *w, *dy, *z;
    void *dx, *dw;
    float *dbias;
} modse_linear_grads_t;
size_t modse_linear_backward_workspace_bytes(int n_tokens, int d_in, int d_out);
modse_status_t modse_linear_backward(int n_tokens, int d_in, int d_out, modse_activation_t activation,
                                     const modse_linear_grads_t *args, void *workspace, size_t workspace_bytes,
                                     void *cuda_stream);

/* Orthogonalised updates (the step of the Muon optimiser): for each matrix G of a
 * set, by `steps` Newton-Schulz iterations on X0 = G / (|G|_F + eps),
 *   A = X X^T,  X <- a X + (b A + c A^2) X,   update = scale X,
 * where the shorter side of G plays the part of X's rows.  Muon's coefficients are
 * a, b, c = 3.4445, -4.7750, 2.0315 and five steps.  A matrix of zeros gives zeros
 * (with eps > 0).
 * grad and update [rows, cols] with ld_grad, ld_update elements from row to row
 * (>= cols), so a matrix may be a column block of a wider one; no alignment beyond the
 * element's.  grad in `dtype` (MODSE_F32 or MODSE_BF16), update bf16, not
 * overlapping any grad.  rows, cols in 1 .. 2^20, the shorter of them at most 2^17.
 * The products read fp16 factors and accumulate in fp32, X is carried in 22 bits:
 * the relative error of an update is of the order of its bf16 rounding.
 * Coefficients that let a singular value of the iteration pass 7.5 are
 * MODSE_ERR_UNSUPPORTED.  The workspace holds up to 16 matrices at a time; longer
 * sets are worked off in order.  Its size is that of the very set it was asked for: a
 * part of the set may need more (the whole may take another form).
 *
 * modse_orthogonalize_wgrads does it for the expert matrices of a layer, straight
 * from the gradients modse_backward wrote (dw_gate, dw_up, dw_down of `grads`; the
 * router's is left out) into `updates` of the same layouts in bf16.  dtype says what
 * the gradients are (MODSE_F32 for those of modse_set_output_f32 layers too).
 * scales: NULL, or host floats [N][3], one a matrix: gate, up, down of expert 0, 1, ... */
typedef struct {
    const void *grad;
    void *update;
    long long ld_grad, ld_update;
    int rows, cols;
    float scale;
} modse_matrix_t;
size_t modse_orthogonalize_workspace_bytes(int n_matrices, const modse_matrix_t *matrices);
modse_status_t modse_orthogonalize(modse_dtype_t dtype, int n_matrices, const modse_matrix_t *matrices, int steps,
                                   const float *coefficients, float eps, void *workspace, size_t workspace_bytes,
                                   void *cuda_stream);
size_t modse_orthogonalize_wgrads_workspace_bytes(const modse_layer_t *layer);
modse_status_t modse_orthogonalize_wgrads(const modse_layer_t *layer, modse_dtype_t dtype, const modse_wgrads_t *grads,
                                          const modse_wgrads_t *updates, const float *scales, int steps,
                                          const float *coefficients, float eps, void *workspace, size_t workspace_bytes,
                                          void *cuda_stream);

/* Embedding lookup with scaling, what the first block's residual stream is made of:
 *   y_t = scale table[id_t].
 * ids [T], of 4 or 8 bytes each (id_bytes; int32 or int64, aligned to that), table
 * [vocabulary, d] and y [T, d] in `dtype`, y not overlapping the table; d a multiple
 * of 8, at most 32768 (else MODSE_ERR_UNSUPPORTED); at most 2^30 tokens and rows.  A
 * negative id is padding: its row of y is zeros.  So is that of an id past the table,
 * which is an error: `status` (a device word, or NULL) then becomes nonzero, as
 * modse_check_workspace_status reads it.  No call clears it, so one word may serve many.
 * The product is formed in fp32 and rounded once.                             */
modse_status_t modse_embedding(modse_dtype_t dtype, int n_tokens, int d_model, int vocabulary, const void *ids, int id_bytes,
                               const void *table, float scale, void *y, int *status, void *cuda_stream);

/* Gradient of the above: from dy [T, d] in `dtype`, into dtable [vocabulary, d] in
 * grad_dtype,
 *   dtable_v = scale sum of dy_t over all t with id_t = v,
 * overwritten (rows that no id names are zeros), or, with accumulate, added to what is
 * there (rows that no id names are not touched): to the gradient of a head that shares
 * the table, or of earlier micro-batches.  Sums are fp32, over ascending t, in an order
 * that does not depend on the run; each element is rounded once a call.  Ids as above: padding
 * and ids past the table give nothing, the latter leave MODSE_ERR_DEVICE_BOUNDS in the
 * workspace's status word.  dtable overlaps no input.  The workspace's size never falls
 * with n_tokens.                                                              */
size_t modse_embedding_backward_workspace_bytes(int n_tokens, int d_model, int vocabulary);
modse_status_t modse_embedding_backward(modse_dtype_t dtype, int n_tokens, int d_model, int vocabulary, const void *ids,
                                        int id_bytes, const void *dy, float scale, modse_dtype_t grad_dtype, int accumulate,
                                        void *dtable, void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Softmax cross entropy over a vocabulary, straight from the rows that would be multiplied
 * by the output matrix: the logits z = x w^T are formed tile by tile and never stored.
 *   lse_t = log sum_v exp z_tv,   loss_t = lse_t - z_t,label_t.
 * x [T, d] and w [vocabulary, d] bf16, d a multiple of 8, any vocabulary; labels [T], of
 * 4 or 8 bytes each (label_bytes, aligned to that); loss and lse [T] fp32.  A token with a negative label is
 * not counted: its loss is 0 (its lse is written all the same).  So is one with a label
 * past the vocabulary, which is an error: MODSE_ERR_DEVICE_BOUNDS in the workspace's
 * status word.  total [2] (or NULL): the sum of the losses and how many tokens were counted,
 * both fp32; their quotient is the mean loss.  Logits are accumulated in fp32 and enter the
 * exponentials unrounded.  Infinities and NaN go where the formulas lead; finite logits
 * are below 2e38.  d at most 2^20, T and vocabulary at most 2^28, and their product at most
 * 2^45.                                                                       */
typedef struct {
    const void *x, *w, *labels;
    float *loss, *lse, *total;
    int label_bytes;
} modse_cross_entropy_t;
size_t modse_cross_entropy_workspace_bytes(int n_tokens, int d_model, int vocabulary);
modse_status_t modse_cross_entropy(int n_tokens, int d_model, int vocabulary, const modse_cross_entropy_t *args, void *workspace,
                                   size_t workspace_bytes, void *cuda_stream);

/* Gradient of sum_t f_t loss_t, from the lse that forward wrote:
 *   dz_tv = f_t (exp(z_tv - lse_t) - [v = label_t]),  dx = dz w,  dw = dz^T x,
 *   f_t = scale dloss_t / total[1]   for counted tokens, 0 for the others.
 * dloss [T] fp32 (NULL: ones), total as forward wrote it (NULL: no division), so that
 * the gradient of the mean loss takes neither arithmetic nor a copy to the host in between.
 * A row whose f is 0 has a dz of zeros, whatever its logits are (so that dw has a NaN in the columns where such a row of x is
 * infinite or NaN, and only there).  No exponential is above 1.  The logits are formed again,
 * in fp32 sums that may be cut at other places than forward's: an exponential is off by as much of itself as the rounding of
 * the two sums moves its logit.  dx [T, d] and dw
 * [vocabulary, d] bf16; either may be NULL; both are overwritten and overlap no input.  The
 * logits are formed again, a piece of the vocabulary at a time (the workspace holds one
 * piece's dz: at most 128 MB or 2048 columns, whichever is more, and 255 columns; and one to eight sums of
 * T d fp32 numbers where dx is summed up in several pieces or parts); dz enters the products rounded to bf16 once, sums are
 * fp32.  The workspaces' sizes, forward's and the gradient's, never fall with n_tokens.  */
typedef struct {
    const void *x, *w, *labels;
    const float *lse, *dloss, *total;
    void *dx, *dw;
    float scale;
    int label_bytes;
} modse_cross_entropy_grads_t;
size_t modse_cross_entropy_backward_workspace_bytes(int n_tokens, int d_model, int vocabulary);
modse_status_t modse_cross_entropy_backward(int n_tokens, int d_model, int vocabulary, const modse_cross_entropy_grads_t *args,
                                            void *workspace, size_t workspace_bytes, void *cuda_stream);

/* Synchronises the stream and reads the status word of the last call that used this
 * workspace (modse_linear, modse_linear_backward, modse_orthogonalize,
 * modse_embedding_backward, modse_cross_entropy and its gradient, modse_decode): MODSE_OK,
 * MODSE_ERR_DEVICE_TIMEOUT or MODSE_ERR_DEVICE_BOUNDS.  A call without tokens or matrices leaves MODSE_OK there. */
modse_status_t modse_check_workspace_status(const void *workspace, void *cuda_stream);

/* Debugging aid, process-wide: when on, bf16 layers run their grouped GEMMs on
 * the fp32-FMA kernels of the fp32 type (with bf16 storage) instead of the
 * tensor-core kernels - slow, meant for cross-checking.  Such a forward must
 * be called with save_for_backward = 1.  Off by default.                    */
void modse_debug_use_fma_path(int on);

/* Tuning aid, process-wide: the tile plan (see modse_get_tile_plan) of layers that have none of their own.
 * The library's default (0x3F3A) puts every product on CTA pairs, and, where that kernel does not apply (the
 * row-gathering up/gate product), products 1, 3, 4 and 5 on one-CTA 256-row tiles.  Every choice gives
 * bit-identical results (the order in which each output element is summed does not depend on the tile shape). */
void modse_debug_set_default_tile_plan(int plan);

/* Tuning aid, process-wide: 1 (default) - the CTAs of a grouped product take tiles, longest K first, from a
 * counter in the workspace; 0 - the tiles are dealt to the CTAs round-robin.  Same results either way.   */
void modse_debug_set_dynamic_tiles(int on);

/* Tuning aid, process-wide: how many warps of a CTA run the epilogue of a grouped product.  Bit k of mask_128 /
 * mask_256 / mask_pair set: product k (numbered as in modse_get_tile_plan) runs sixteen epilogue warps when it
 * is on 128-row tiles / one-CTA 256-row tiles / CTA-pair tiles, clear: eight.  Default: sixteen for the up/gate
 * product and the down dgrad on one-CTA 256-row tiles (mask_256 = 5), eight elsewhere.  Same results either way,
 * except that the gate gradient of MODSE_FUSE_DG_ROWDOT is summed from twice as many partials (same tolerance). */
void modse_debug_set_epilogue_warps(int mask_128, int mask_256, int mask_pair);

/* Failure-path aids, process-wide.  Every wait inside a kernel gives up after a limit (default 2000 ms),
 * records MODSE_ERR_DEVICE_TIMEOUT in the status word, lets its copies in flight land, frees its tensor
 * memory and returns; modse_debug_set_wait_limit_ms changes the limit (1..60000).
 * modse_debug_skip_tile_loads(product, tile) makes the CTA that is handed tile `tile` of grouped product
 * `product` (0..5; 6: the products of modse_linear, its gradient, modse_orthogonalize and modse_cross_entropy, whose
 * `tile` counts a launch's work items; 7: modse_decode on bf16 layers whose extents are multiples of 64, whose
 * `tile` is a block of its first kernel) issue no loads for it and stop producing, so that its consumers run into that limit
 * with nothing in flight; (-1, -1) switches it off.  For tests of the time-out path on tiny inputs.          */
void modse_debug_set_wait_limit_ms(int ms);
void modse_debug_skip_tile_loads(int product, int tile);

/* Test aid: byte offsets, inside a workspace of the given shape, of the padded row table prow_of [T,k] and of
 * the guard block behind topk_idx, and the number of padded rows (the extent row indices are checked against). */
modse_status_t modse_debug_workspace_offsets(const modse_layer_t *layer, modse_dtype_t dtype, int n_tokens,
                                             int save_for_backward, size_t *prow_of_offset, size_t *first_guard_offset,
                                             int *padded_rows);

#ifdef __cplusplus
}
#endif
#endif /* MODSE_H */
