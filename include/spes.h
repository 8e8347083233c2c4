/*
 * spes.h -- C ABI of the SPES MoE-layer hot path for AMD MI355X (gfx950).
 *
 * One node of SPES-style decentralised MoE pretraining stores every expert of a
 * routed feed-forward layer but trains only its assigned subset (paper Sec. 3.3,
 * "Expert Assignment and Local Training", Eq. 3).  This library is that node's
 * training step through one such layer, plus the periodic synchronisation of
 * node-local expert copies (Sec. 3.3 "Sparse Synchronization", Eq. 4) and the
 * expert-merging warm-up (Sec. 3.3 "Expert-Merging Warm-Up", Eq. 5-6).
 *
 * Conventions that hold for every entry point
 *  - Plain C linkage, plain pointers and sizes.  "DEVICE" pointers address GPU
 *    memory of the current HIP device, "HOST" pointers ordinary host memory.
 *  - The library allocates no device memory and the entry points declared here keep
 *    no state between calls.  Inputs, outputs, the context buffer and scratch are
 *    owned by the caller.  (The benchmark aids of spes_bench.h are the exception:
 *    they hold a process-wide set of timing events.)
 *  - All work is enqueued on `stream` (a hipStream_t passed as void*; NULL is
 *    the default stream).  No entry point synchronises or copies device memory
 *    back to the host; per-expert token counts are consumed on the device.
 *  - HOST arrays are read before the call returns and may be freed afterwards.
 *  - Return value: SPES_OK (0) or a negative spes_status.  Arguments are checked
 *    before anything is launched, so a failed check has no side effects.
 *  - Tensors are row-major with the innermost dimension contiguous.  Weight
 *    matrices are stored [out_features, in_features].  DEVICE pointers must be
 *    16-byte aligned.  Outputs must not alias inputs.
 *  - dtype selects the storage type of parameters and activations (fp32, or
 *    bf16 with round-to-nearest-even on every store); every accumulation is fp32.
 *    Router logits, gates and all weight gradients are fp32 in both modes.
 *  - Results are reproducible bit for bit.  Within a call, rows with equal operands
 *    get equal bits wherever they stand: copies of a token, and a token's rows at
 *    experts that are copies of one another.
 */
#ifndef SPES_H_
#define SPES_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SPES_API __attribute__((visibility("default")))

typedef enum {
  SPES_OK = 0,
  SPES_EINVAL = -1, /* null pointer, non-positive size, top_k > n_experts, bad dtype   */
  SPES_ESHAPE = -2, /* a size this build does not support (see each call)              */
  SPES_EALIGN = -3, /* a DEVICE pointer is not 16-byte aligned                         */
  SPES_EHIP = -4    /* a kernel launch failed; see hipGetLastError                     */
} spes_status;

typedef enum { SPES_F32 = 0, SPES_BF16 = 1 } spes_dtype;

/* Shape of one routed feed-forward layer (Sec. 3.1 Eq. 2; Sec. 3.2).
 * Supported: 1 <= top_k <= n_experts <= 64; d_model and d_ff multiples of 8;
 * T*top_k at most 2^22 - 4224; in bf16 storage T*d_model, T*top_k*d_ff and
 * n_experts*d_ff*d_model each below 2^31 (SPES_ESHAPE otherwise). */
typedef struct {
  int32_t T;           /* tokens in the batch                                         */
  int32_t d_model;     /* d                                                           */
  int32_t n_experts;   /* M                                                           */
  int32_t d_ff;        /* f, hidden width of one SwiGLU expert                        */
  int32_t top_k;       /* k experts per token                                         */
  int32_t dtype;       /* spes_dtype                                                  */
  int32_t renorm_topk; /* 1: gates are renormalised over the k chosen (Sec. 4,
                          upcycled model); 0: gate = softmax probability over all M   */
} spes_moe_shape;

/* Byte offsets of the regions inside the context buffer; exposed so that tests
 * can inspect routing tables and saved activations.  R = T*top_k routed rows. */
typedef struct {
  size_t total;
  size_t logits;    /* [T,M] f32 router scores                                        */
  size_t lse;       /* [T] f32 log-sum-exp of the scores                              */
  size_t topk_idx;  /* [T,k] i32 copy of the selected experts                          */
  size_t topk_gate; /* [T,k] f32 copy of their gates                                  */
  size_t offset;    /* [M+1] i32 first row of each expert in expert-contiguous order  */
  size_t perm;      /* [R] i32 row r holds routed pair perm[r] = t*k+j                */
  size_t inv;       /* [R] i32 inverse of perm                                        */
  size_t a;         /* [R,f] gate projection  W_g x, in the storage type               */
  size_t b;         /* [R,f] up projection    W_u x, in the storage type               */
  size_t h;         /* [R,f] SiLU(a)*b                                                */
  size_t yp;        /* [R,d] expert outputs before gating                             */
  size_t dlogits;   /* [T,M] f32, written by the backward                             */
  size_t dgate;     /* [T,k] f32, written by the backward                             */
} spes_moe_ctx_layout;

/* Size and layout of the context buffer that spes_moe_fwd fills and spes_moe_bwd
 * consumes (it also holds the backward's scratch).  Returns 0 on a bad shape. */
SPES_API size_t spes_moe_ctx_bytes(const spes_moe_shape* shape);
SPES_API int spes_moe_ctx_describe(const spes_moe_shape* shape, spes_moe_ctx_layout* out);

/* Forward of the routed SwiGLU layer: y_t = sum_j G_j(x_t) E_j(x_t) (Sec. 3.1 Eq. 2)
 * with softmax routing over all M experts followed by top-k selection, drop-less
 * dispatch (every selected pair is computed; Sec. 3.2) and SwiGLU experts
 * E(x) = W_d (SiLU(W_g x) * W_u x).
 *
 *  x            DEVICE [T,d]      w_router DEVICE [M,d]
 *  router_bias  DEVICE [M] f32 or NULL (added to the scores; receives no gradient)
 *  w_gate,w_up  DEVICE [M,f,d]    w_down   DEVICE [M,d,f]
 *  y            DEVICE [T,d] out
 *  topk_idx     DEVICE [T,k] i32 out: selected experts in descending score order,
 *               equal scores resolved to the lower expert id
 *  topk_gate    DEVICE [T,k] f32 out
 *  expert_count DEVICE [M] i32 out: routed pairs per expert (sums to T*k)
 *  ctx          DEVICE, spes_moe_ctx_bytes(shape) bytes, 256-byte aligned
 */
SPES_API int spes_moe_fwd(const spes_moe_shape* shape, const void* x, const void* w_router,
                          const float* router_bias, const void* w_gate, const void* w_up,
                          const void* w_down, void* y, int32_t* topk_idx, float* topk_gate,
                          int32_t* expert_count, void* ctx, void* stream);

/* The permuted copy of the input that drop-less dispatch defines (Sec. 3.2): row r of xp is
 * the input row of the routed pair that the forward placed at position r of the
 * expert-contiguous order, xp[inv[t*k+j], :] = x[t, :].  spes_moe_fwd and spes_moe_bwd do not
 * need it (their grouped GEMMs read x through the same table); this entry point materialises
 * it for callers that want the dispatched activations, and is the stand-alone form of the
 * dispatch step.
 *
 *  x    DEVICE [T,d]       ctx  DEVICE, as left by spes_moe_fwd for this shape
 *  xp   DEVICE [T*k,d] out, must not alias x
 */
SPES_API int spes_moe_permute(const spes_moe_shape* shape, const void* x, const void* ctx, void* xp,
                              void* stream);

/* Backward of the weighted combine of Eq. 2 as a stand-alone step: for the k routed pairs of
 * every token,  dyp[inv[t*k+j], :] = gate[t,j] * dy[t, :]  (the upstream gradient of each routed
 * row, in expert-contiguous order) and  dgate[t,j] = <dy[t, :], yp[inv[t*k+j], :]>  with yp the
 * expert outputs the last spes_moe_fwd left in ctx.  spes_moe_bwd does not run this kernel: it
 * gathers and scales the dy rows inside its first GEMM and takes the gate gradient from that
 * GEMM's accumulators (yp is stored in the storage type; in bf16 that rounding is too coarse for
 * the router gradient of near-identical experts).  This entry point materialises the step as the
 * chain rule states it.
 *
 *  dy     DEVICE [T,d]                 ctx    DEVICE, as left by spes_moe_fwd for this shape
 *  dyp    DEVICE [T*k, d] out          dgate  DEVICE [T,k] f32 out
 */
SPES_API int spes_moe_grad_scatter(const spes_moe_shape* shape, const void* dy, const void* ctx,
                                   void* dyp, float* dgate, void* stream);

/* Backward of the same layer for upstream gradient dy.  The selected expert set
 * is treated as constant.  The input gradient flows through every routed expert,
 * trainable or frozen; weight gradients are produced only for experts whose mask
 * byte is non-zero (Sec. 3.3 Eq. 3; App. A, block mask U_i), into compact
 * buffers with one slot per trainable expert in ascending expert id, so frozen
 * experts own no gradient memory.  The router belongs to the shared modules that
 * every node trains, so d_w_router is always produced.
 *
 *  dy, x          DEVICE [T,d]; weights as in the forward, ctx as left by it
 *  trainable_mask HOST  [M] bytes
 *  dx             DEVICE [T,d] out
 *  d_w_router     DEVICE [M,d] f32
 *  d_w_gate,d_w_up DEVICE [n_trainable,f,d] f32;  d_w_down DEVICE [n_trainable,d,f] f32
 *                 (may be NULL when no expert is trainable)
 *  accumulate     0: weight gradients are overwritten; 1: added to (micro-batches)
 */
SPES_API int spes_moe_bwd(const spes_moe_shape* shape, const void* dy, const void* x,
                          const void* w_router, const void* w_gate, const void* w_up,
                          const void* w_down, void* ctx, const uint8_t* trainable_mask, void* dx,
                          float* d_w_router, float* d_w_gate, float* d_w_up, float* d_w_down,
                          int32_t accumulate, void* stream);

/* The layer behind a routing that the caller made (spes_router_fwd, or another): spes_moe_fwd and spes_moe_bwd without their
 * router.  Choice and gates come in, the gates' gradient goes out; dx is the experts' part alone.  renorm_topk of the shape is
 * not looked at, and spes_moe_router_aux has no scores to work on.  An entry of topk_idx that is no expert counts as expert 0
 * with gate 0.
 *
 *  topk_idx   DEVICE [T,k] i32      topk_gate  DEVICE [T,k] f32 (both copied into ctx, for the backward)
 *  dgate      DEVICE [T,k] f32 out
 *  all others as above
 */
SPES_API int spes_moe_fwd_routed(const spes_moe_shape* shape, const void* x, const int32_t* topk_idx,
                                 const float* topk_gate, const void* w_gate, const void* w_up,
                                 const void* w_down, void* y, int32_t* expert_count, void* ctx,
                                 void* stream);
SPES_API int spes_moe_bwd_routed(const spes_moe_shape* shape, const void* dy, const void* x,
                                 const void* w_gate, const void* w_up, const void* w_down, void* ctx,
                                 const uint8_t* trainable_mask, void* dx, float* dgate,
                                 float* d_w_gate, float* d_w_up, float* d_w_down, int32_t accumulate,
                                 void* stream);

/* Auxiliary router losses (Sec. 3.3 "Training Losses"; coefficients App. B: load-balancing
 * 0.01, router z-loss 0.001).  The paper names the two losses and cites their sources; the
 * formulas used are the cited ones:
 *      L_lb = M * sum_e f_e * P_e     f_e = share of the T*k routed pairs sent to expert e,
 *                                     P_e = mean over tokens of the softmax probability of e
 *      L_z  = mean over tokens of (log sum_e exp(score_te))^2
 * on the scores (router bias included) of the forward pass whose record is in ctx.
 * Call it after spes_moe_fwd and before spes_moe_bwd on the same ctx.  It writes the two loss
 * values and arms ctx so that the next spes_moe_bwd adds
 *      grad_scale * (lb_coef * dL_lb/dscores + z_coef * dL_z/dscores)
 * to the gating gradient before it reaches d_w_router and dx (f_e is a count and carries no
 * gradient).  grad_scale is whatever factor the caller's total loss applies to this layer's
 * auxiliary terms (1 for a plain sum, 1/n for n micro-batches, a loss scale).  The next
 * spes_moe_fwd on the ctx disarms it; without this call spes_moe_bwd is unchanged.
 *
 *  ctx     DEVICE, as left by spes_moe_fwd for this shape
 *  losses  DEVICE [2] f32 out: L_lb, L_z (unweighted)
 */
SPES_API int spes_moe_router_aux(const spes_moe_shape* shape, void* ctx, float lb_coef,
                                 float z_coef, float grad_scale, float* losses, void* stream);

/* AdamW step on the trainable subset of one parameter matrix of the expert store.  A node keeps
 * gradients and the two optimizer moments only for its assigned experts and for the shared
 * parameters (Sec. 3.3 "Efficiency Analysis", the 3 x |Phi_i| term of the memory model), so all
 * optimizer state is compact: one slot per expert whose mask byte is non-zero, in ascending expert
 * id, exactly like the gradient buffers of spes_moe_bwd.  Per element, with g = grad_scale * grad,
 *      m <- beta1 m + (1-beta1) g          v <- beta2 v + (1-beta2) g^2
 *      w <- w - lr ( (m / (1-beta1^step)) / (sqrt(v / (1-beta2^step)) + eps) + weight_decay w )
 * in fp32 (Table A1: beta 0.9 / 0.95, eps 1e-8, weight decay 0.1), then the expert's row of the
 * full store is overwritten with w rounded to the storage type.  Frozen experts are not touched.
 * A shared matrix such as the router is the case n_experts = 1, mask = {1}.
 *
 *  n_experts >= 1; elems = elements of the matrix per expert, a multiple of 8
 *  param        DEVICE [n_experts, elems] storage dtype, in/out
 *  trainable_mask HOST [n_experts] bytes
 *  master       DEVICE [n_trainable, elems] f32 in/out: the fp32 weights; NULL is allowed for
 *               dtype f32 only, then param itself is the weight
 *  m, v         DEVICE [n_trainable, elems] f32 in/out
 *  grad         DEVICE [n_trainable, elems] f32
 *  step         >= 1, the number of this update (bias correction)
 */
SPES_API int spes_masked_adamw(int32_t n_experts, int64_t elems, int32_t dtype, void* param,
                               const uint8_t* trainable_mask, float* master, float* m, float* v,
                               const float* grad, float lr, float beta1, float beta2, float eps,
                               float weight_decay, int32_t step, float grad_scale, void* stream);

/* Upcycling initialiser (Sec. 4, upcycling settings: the dense FFN is replicated into the experts
 * and Gaussian noise of standard deviation 0.02 is added to 50 % of the parameters), for one
 * parameter matrix:  out[e][i] = dense[i] + select(e,i) * sigma * z(e,i),  rounded to the storage type.
 * The draws are a pure function of (seed, stream_id, e*elems + i): Philox-4x64-10 with key (seed, 0)
 * and counter (g, stream_id, 0, 0) yields words w_0..w_3 for the group g of four consecutive flat
 * indices; element j is selected iff (w_j & 255) < floor(fraction * 256); z of elements 2q, 2q+1 is
 * r cos(2 pi u2), r sin(2 pi u2) with r = sqrt(-2 ln u1), u1 = ((w_2q >> 40) + 0.5) / 2^24,
 * u2 = ((w_2q+1 >> 40) + 0.5) / 2^24.  Use a different stream_id per parameter matrix.
 *
 *  n_experts >= 1; elems a multiple of 8; 0 <= fraction <= 1; sigma >= 0
 *  dense  DEVICE [elems]            out  DEVICE [n_experts, elems]
 */
SPES_API int spes_upcycle_init(int32_t n_experts, int64_t elems, int32_t dtype, const void* dense,
                               float fraction, float sigma, uint64_t seed, uint64_t stream_id,
                               void* out, void* stream);

/* Gather (to_store = 0) or scatter (to_store = 1) of the rows of the experts whose mask byte is
 * non-zero between the full store and a contiguous buffer with one row per such expert in ascending
 * expert id: what a node uploads at a synchronisation is only what it trained (Sec. 3.3, Eq. 4),
 * and the buffer has the layout spes_expert_merge reads as a node store.
 *
 *  store   DEVICE [n_experts, elems]   packed  DEVICE [n_trainable, elems]   elems a multiple of 8
 *  trainable_mask HOST [n_experts] bytes
 */
SPES_API int spes_expert_pack(int32_t n_experts, int64_t elems, int32_t dtype, void* store,
                              const uint8_t* trainable_mask, void* packed, int32_t to_store,
                              void* stream);

/* Synchronisation of node-local expert copies (Sec. 3.3 Eq. 4; App. A sync rules),
 * for one parameter matrix of every expert.  Expert j becomes the weighted mean
 * of the copies held by the nodes that trained it,
 *      dst[j] = sum_i w_i * store_i[slot[i][j]] / sum_i w_i   over i with slot[i][j] >= 0,
 * which is FedAvg when all nodes train it with equal weights and a direct
 * (bit-exact) assignment when a single node does.  An expert nobody trained keeps
 * the value already in dst.
 *
 *  n_experts >= 1; elems = elements of the matrix per expert, a multiple of 8
 *  node_store   HOST  [n_nodes] DEVICE pointers; store i is [n_i, elems]
 *  slot         HOST  [n_nodes, n_experts] i32: row of expert j in store i, or -1
 *  node_weight  HOST  [n_nodes] f32 (> 0) or NULL for equal weights
 *  dst          DEVICE [n_experts, elems] in/out
 *  trainer_count DEVICE [n_experts] i32 out or NULL: number of trainers per expert
 *  At most 224 trainers per expert (SPES_ESHAPE beyond).
 */
SPES_API int spes_expert_merge(int32_t n_experts, int64_t elems, int32_t dtype, int32_t n_nodes,
                               const void* const* node_store, const int32_t* slot,
                               const float* node_weight, void* dst, int32_t* trainer_count,
                               void* stream);

/* Expert-merging warm-up (Sec. 3.3 Eq. 5-6; App. A merge step).  Cosine similarity
 * A[j][k] between the flattened input projections w_in[j], w_in[k]; Q_j = the top_K
 * most similar experts to j, j excluded, equal similarities resolved to the lower
 * id; then for each of the n_mats parameter matrices
 *      dst[m][j] = src[m][j] + (alpha/top_K) * sum_{k in Q_j} (src[m][k] - src[m][j]),
 * every right-hand side being the pre-merge value (out of place: dst[m] != src[m]).
 *
 *  1 <= top_K < n_experts <= 64
 *  w_in     DEVICE [M, elems_in], elems_in a multiple of 8
 *  src,dst  HOST arrays of n_mats DEVICE pointers, matrix m is [M, elems[m]]
 *  elems    HOST  [n_mats], each a multiple of 8
 *  sim      DEVICE [M,M] f32 out or NULL;  nbr DEVICE [M,top_K] i32 out
 *           (a pair with a zero-norm projection, for which Eq. 5 is 0/0, gets similarity 0;
 *           every entry of nbr is a valid expert other than the row's own, whatever w_in holds)
 *  scratch  DEVICE, spes_warmup_scratch_bytes(M, elems_in) bytes
 */
SPES_API size_t spes_warmup_scratch_bytes(int32_t n_experts, int64_t elems_in);
SPES_API int spes_expert_warmup_merge(int32_t n_experts, int32_t dtype, int32_t top_K, float alpha,
                                      const void* w_in, int64_t elems_in, int32_t n_mats,
                                      const void* const* src, void* const* dst,
                                      const int64_t* elems, float* sim, int32_t* nbr,
                                      void* scratch, void* stream);

/* spes_expert_warmup_merge for callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same computation with the
 * same arguments, except that the Gram partial sums go to a buffer that is part of the library's
 * own device image (8 MiB, held by every GPU the library runs on until the process ends) instead
 * of a caller-provided scratch.  The call allocates and frees nothing.  That buffer covers every
 * supported problem (n_experts <= 64, at most 512 chunks of the contraction); a problem that
 * would need more is rejected with SPES_ESHAPE.  All calls on one GPU share the buffer: calls
 * that overlap in time on one GPU (different streams) race on it; calls on one stream are safe.
 * Nothing in it needs clearing between calls: every partial a call reads was written by that call.
 */
SPES_API int spes_expert_warmup_merge_static(int32_t n_experts, int32_t dtype, int32_t top_K,
                                             float alpha, const void* w_in, int64_t elems_in,
                                             int32_t n_mats, const void* const* src,
                                             void* const* dst, const int64_t* elems, float* sim,
                                             int32_t* nbr, void* stream);

/* ---- Operators around the expert layer ------------------------------------------------------------------------------
 * What a training program runs beside the routed layer: the norm ahead of it, routing of other kinds than the layer's own, and an
 * optimizer step that orthogonalises the update.  Zero rows or tokens are a valid call.
 */

/* Layer norm (kind SPES_NORM_LAYER) or root-mean-square norm (SPES_NORM_RMS) of every row, with the residual stream's addition:
 *      v = x + add (rounded to the storage type)   or  v = x  without add
 *      mean = sum v / cols (layer norm; 0 otherwise)      rstd = (sum (v - mean)^2 / cols + eps)^-1/2
 *      y = (v - mean) rstd weight + bias
 *
 *  rows >= 0; 1 <= cols <= 16384
 *  x, add     DEVICE [rows, cols], rows x_stride and add_stride elements apart (>= cols); add may be NULL.  Here and in
 *             spes_norm_bwd a tensor with a stride needs no other alignment than its element's
 *  weight     DEVICE [cols]      bias  DEVICE [cols] or NULL
 *  eps        >= 0
 *  sum        DEVICE [rows, cols] out: v; NULL exactly if add is
 *  y          DEVICE [rows, cols] out
 *  mean       DEVICE [rows] f32 out, layer norm only (else NULL)     rstd  DEVICE [rows] f32 out
 */
typedef enum { SPES_NORM_LAYER = 0, SPES_NORM_RMS = 1 } spes_norm_kind;
SPES_API int spes_norm_fwd(int32_t kind, int32_t rows, int32_t cols, int32_t dtype, const void* x,
                           int64_t x_stride, const void* add, int64_t add_stride,
                           const void* weight, const void* bias, float eps, void* sum, void* y,
                           float* mean, float* rstd, void* stream);

/* Backward of spes_norm_fwd for the upstream gradient dy.  With hat = (v - mean) rstd and h = dy weight
 *      dx = rstd (h - hat (sum h hat / cols) - (sum h / cols, layer norm only)) + dres
 *      d_weight = sum over rows of dy hat           d_bias = sum over rows of dy
 * dx is the gradient of v, hence of x and of add alike; dres is the gradient that reaches v along the residual stream.
 *
 *  dy, x, dres  DEVICE [rows, cols] with strides as above; x is v (the forward's sum, or its x without add); dres may be NULL
 *  mean, rstd   as the forward left them
 *  dx           DEVICE [rows, cols] out
 *  d_weight     DEVICE [cols] f32, d_bias DEVICE [cols] f32.  d_bias may be NULL; both may (a frozen norm), then scratch may as well
 *  accumulate   0: d_weight and d_bias are overwritten; 1: added to
 *  scratch      DEVICE, spes_norm_scratch_bytes(rows, cols) bytes
 */
SPES_API size_t spes_norm_scratch_bytes(int32_t rows, int32_t cols);
SPES_API int spes_norm_bwd(int32_t kind, int32_t rows, int32_t cols, int32_t dtype, const void* dy,
                           int64_t dy_stride, const void* x, int64_t x_stride, const void* weight,
                           const float* mean, const float* rstd, const void* dres,
                           int64_t dres_stride, void* dx, float* d_weight, float* d_bias,
                           int32_t accumulate, void* scratch, void* stream);

/* Routing to experts from given scores.  Per token, with logits l over M experts
 *      s = softmax(l) or sigmoid(l)        c = s + bias
 *      c = -inf where l is -inf or the lowest finite value, which keep an expert from a token, and where it would be NaN
 *      with groups > 1 the experts stand in `groups` groups of M / groups each; a group counts the sum of its two largest c that are
 *      not -inf (its only one, where there is one; -inf, where there is none), and only the kept_groups best groups are open,
 *      equal ones to the lower group
 *      idx = the top_k largest c in open groups in descending order, equal ones to the lower expert
 *      gate = scale * s[idx], with renorm scale * s[idx] / sum of s[idx]
 * The bias steers the choice only: it enters no gate and has no gradient (a program moves it by the counts to balance the load).
 * An expert whose logit is -inf, the lowest finite value or NaN is taken only where nothing else is left in the open groups,
 * whatever its bias; indices are valid and different from one another whatever the logits hold.  A row of -inf alone has gates 0.
 * With renorm, shares keep their bits however small the chosen scores are beside the others, as do their gradients; sigmoid scores lose
 * bits below e^-187 and are 0 below e^-204, and where all chosen ones are, the gates are.
 *
 *  Supported: 1 <= top_k <= 16; n_experts <= 512; groups <= 16, dividing n_experts; top_k <= kept_groups * n_experts / groups
 */
typedef enum { SPES_SCORE_SOFTMAX = 0, SPES_SCORE_SIGMOID = 1 } spes_score;
typedef struct {
  int32_t score;       /* spes_score                                       */
  int32_t groups;      /* 1: no groups                                     */
  int32_t kept_groups; /* 1 <= kept_groups <= groups                       */
  int32_t renorm;      /* 1: gates are renormalised over the chosen ones   */
  float scale;         /* factor of the gates, finite                      */
} spes_router_opts;

/*  logits  DEVICE [T, n_experts] f32      bias   DEVICE [n_experts] f32 or NULL
 *  idx     DEVICE [T, top_k] i32 out      gate   DEVICE [T, top_k] f32 out
 *  count   DEVICE [n_experts] i32 out: tokens that chose the expert
 */
SPES_API int spes_router_fwd(int32_t T, int32_t n_experts, int32_t top_k, const spes_router_opts* opts,
                             const float* logits, const float* bias, int32_t* idx, float* gate,
                             int32_t* count, void* stream);

/* Gradient of the gates with respect to the logits, the choice held fixed.  A gate of 0 has none.
 *
 *  logits, idx  as above, idx as the forward left it      dgate  DEVICE [T, top_k] f32
 *  dlogits      DEVICE [T, n_experts] f32 out
 */
SPES_API int spes_router_bwd(int32_t T, int32_t n_experts, int32_t top_k, const spes_router_opts* opts,
                             const float* logits, const int32_t* idx, const float* dgate,
                             float* dlogits, void* stream);

/* Orthogonalisation of a stack of matrices by Newton-Schulz steps: every matrix is scaled to Frobenius norm 1, then `steps` times
 *      X <- a X + (b X X^T + c (X X^T)^2) X
 * which takes each singular value through a s + b s^3 + c s^5 and leaves the singular vectors.  Products and sums: bf16 storage
 * on fp16 operands with fp32 sums, the result, ahead of its rounding to bf16, within 2e-3 of the formula's in norm, whatever the rank (3e-3
 * where a side is 64 or less: a single direction of so few entries averages less of its rounding out);
 * fp32 storage as products in fp32 (full rank 2e-6, rank one 1.2e-4).  Both for up to five steps with the default coefficients: what rounding
 * leaves in empty directions grows a-fold a step.  A matrix of
 * zeros gives zeros, one that holds an infinity or a NaN gives NaN.  Copies of a matrix in a call get the same bits, whatever stands
 * beside them; n decides how products are cut, so in a call with another n the last bits of the same matrix can be others.
 *
 *  1 <= n <= 65535 matrices of rows x cols, each side at most 16384; 1 <= steps <= 64
 *  src    DEVICE [n, rows, cols] storage dtype      out  DEVICE [n, rows, cols] storage dtype out
 *  coef   HOST [3] f32: a, b, c, or NULL for 3.4445, -4.7750, 2.0315, which lift small singular values to near 1 in five steps.
 *         Values that let singular values grow to 5 overflow the stored operands
 *  scratch DEVICE, spes_orthogonalize_scratch_bytes(n, rows, cols, dtype) bytes
 */
SPES_API size_t spes_orthogonalize_scratch_bytes(int32_t n, int32_t rows, int32_t cols, int32_t dtype);
SPES_API int spes_orthogonalize(int32_t n, int32_t rows, int32_t cols, int32_t dtype, const void* src,
                                void* out, int32_t steps, const float* coef, void* scratch,
                                void* stream);

/* Optimizer step with an orthogonalised update on the trainable subset of one parameter matrix of the expert store; state and
 * gradients are compact, as for spes_masked_adamw.  Per matrix, with g = grad_scale * grad,
 *      m <- beta m + g       u = nesterov ? g + beta m : m       o = spes_orthogonalize(u)
 *      w <- w (1 - lr weight_decay) - lr update_scale o
 * in fp32 (o as above for the storage type), then the expert's row of the full store is overwritten with w rounded to the storage
 * type.  Frozen experts are not touched.  update_scale is the caller's, commonly 0.2 sqrt(max(rows, cols)).
 *
 *  n_experts >= 1; rows, cols: sides of the matrix per expert, each at most 16384
 *  param        DEVICE [n_experts, rows, cols] storage dtype, in/out
 *  trainable_mask HOST [n_experts] bytes
 *  master       DEVICE [n_trainable, rows, cols] f32 in/out; NULL is allowed for dtype f32 only, then param itself is the weight
 *  m            DEVICE [n_trainable, rows, cols] f32 in/out      grad  DEVICE [n_trainable, rows, cols] f32
 *  0 <= beta < 1; steps, coef as above
 *  scratch      DEVICE, spes_orthogonalize_scratch_bytes(n_trainable, rows, cols, dtype) bytes
 */
SPES_API int spes_masked_muon(int32_t n_experts, int32_t rows, int32_t cols, int32_t dtype, void* param,
                              const uint8_t* trainable_mask, float* master, float* m,
                              const float* grad, float lr, float beta, int32_t nesterov,
                              float weight_decay, float update_scale, int32_t steps,
                              const float* coef, float grad_scale, void* scratch, void* stream);

/* ---- The attention half of a block -----------------------------------------------------------------------------------
 * What stands between the projections of a block's attention: the norm of every head of the queries and keys with the rotation by
 * the token's position, and attention over sequences of unequal length with its gradients.
 */

/* Norm and rotation of T tokens' queries (heads of them) and keys (kv_heads).  Per head x of head_dim elements
 *      hat = x (sum x^2 / head_dim + eps)^-1/2        y = hat weight      (without weights y = x)
 *      pair i < rot_dim / 2 of y, (a, b), becomes (a cos - b sin, a sin + b cos) with cos = table[pos][i], sin = table[pos][rot_dim / 2 + i]
 * A pair is elements i and i + rot_dim / 2, or with `interleaved` elements 2 i and 2 i + 1; elements from rot_dim on are not rotated.
 * What angles the table holds is the caller's.  A position that it does not have gives NaN in what is rotated.
 *
 *  Supported: head_dim a multiple of 8, at most 256; rot_dim a multiple of 16, at most head_dim, or 0; heads + kv_heads at most 2^22, T times these below 2^31
 */
typedef struct {
  int64_t q_row, k_row; /* elements from one token's q and k to the next one's, where the projection wrote them (a token's heads stand
                           side by side): multiples of 16 bytes                                     */
  int32_t T;            /* tokens, >= 0                                                             */
  int32_t heads, kv_heads, head_dim, rot_dim;
  int32_t dtype;        /* spes_dtype of q, k, weights and results                                  */
  int32_t interleaved;
  int32_t n_pos;        /* rows of the table                                                        */
  float eps;            /* >= 0                                                                     */
} spes_qk_shape;

/*  q         DEVICE [T, heads, head_dim], k DEVICE [T, kv_heads, head_dim], rows q_row and k_row elements apart
 *  q_weight, k_weight  DEVICE [head_dim], or both NULL
 *  table     DEVICE [n_pos, rot_dim] f32       pos  DEVICE [T] i32, or NULL: token t has position t (then n_pos >= T).  rot_dim 0: both NULL
 *  q_out     DEVICE [T, heads, head_dim] out   k_out  DEVICE [T, kv_heads, head_dim] out
 */
SPES_API int spes_qk_rope_fwd(const spes_qk_shape* shape, const void* q, const void* k, const void* q_weight,
                              const void* k_weight, const float* table, const int32_t* pos, void* q_out,
                              void* k_out, void* stream);

/* Its backward for the upstream gradients dq and dk of q_out and k_out.  A token whose position the table does not have gets gradients of NaN, and so do
 * the weights.
 *
 *  dq        DEVICE [T, heads, head_dim]       dk  DEVICE [T, kv_heads, head_dim]
 *  q, k      as above (NULL is allowed without weights)
 *  dq_in, dk_in  DEVICE out, laid out as q and k are (q_row, k_row)
 *  d_q_weight, d_k_weight  DEVICE [head_dim] f32; both NULL without weights or where they are frozen, then scratch may be NULL as well
 *  accumulate    0: d_q_weight and d_k_weight are overwritten; 1: added to
 *  scratch   DEVICE, spes_qk_rope_scratch_bytes(shape) bytes
 */
SPES_API size_t spes_qk_rope_scratch_bytes(const spes_qk_shape* shape);
SPES_API int spes_qk_rope_bwd(const spes_qk_shape* shape, const void* dq, const void* dk, const void* q,
                              const void* k, const void* q_weight, const void* k_weight, const float* table,
                              const int32_t* pos, void* dq_in, void* dk_in, float* d_q_weight,
                              float* d_k_weight, int32_t accumulate, void* scratch, void* stream);

/* Attention of n_seq sequences' queries over their keys.  Per query and head, over the keys j that the query sees,
 *      s_j = scale <q, k_j>        lse = ln sum_j exp s_j        o = sum_j exp(s_j - lse) v_j
 * Head h of the queries reads head h / (heads / kv_heads) of keys and values.  Sequence b has the queries in rows q_start[b] up to q_start[b+1], and
 * its keys and values in rows k_start[b] up to k_start[b+1], or, where k_len is given, in k_len[b] rows from k_start[b] on (a cache with room for more;
 * in the forward sequences may share rows of it).  With `causal` the last query sees the last key and every one before it a key less: query i of
 * lq sees the keys up to i + lk - lq, with a window the last `window` of these.  A query that sees no key has o = 0 and lse = -infinity, its dq is 0.
 * Rows outside of all sequences are not read, and those of o, lse, dq, dk and dv are left as they are.  What the descriptors
 * hold is cut to the tensors' rows; queries of two sequences must not overlap, nor in the backward keys.  Rows of a sequence must be finite: an
 * infinity or a NaN in one can reach other rows of its sequence, whether they see it or not.
 * Products in bf16 storage take bf16 operands, the probabilities and their gradient among them, and are summed in fp32; in fp32 storage they are fp32.
 * Lengths stay on the device, so a captured call takes new ones; how the work is cut follows from n_seq, q_rows and k_rows alone.  A batch of unlike sequences (a prompt
 * beside single tokens), places of no queries, and chunks of queries in a cache with much more room than keys are answered all the same, but take longer.
 *
 *  Supported: head_dim a multiple of 8, at most 128; heads a multiple of kv_heads, at most 1024; q_rows heads at most 2^30, k_rows at most 2^31 - 2^16
 *  (in the backward k_rows kv_heads at most 2^29), n_seq kv_heads at most 2^22; strides multiples of 16 bytes, rows at most 2^20 elements
 *  apart, heads / kv_heads heads of q within 2^28 elements
 */
typedef struct {
  int64_t q_row, q_head; /* elements from a token's q to the next one's, and from a head's to the next one's; of dq as well     */
  int64_t k_row, k_head; /* the same of k and dk                                                                                */
  int64_t v_row, v_head; /* the same of v and dv                                                                                */
  int32_t n_seq;         /* >= 0                                                                                                */
  int32_t q_rows;        /* rows of q, o and lse                                                                                */
  int32_t k_rows;        /* rows of k and v                                                                                     */
  int32_t heads, kv_heads, head_dim;
  int32_t dtype;         /* spes_dtype                                                                                          */
  int32_t causal;
  int32_t window;        /* 0: none; > 0 with causal only                                                                       */
  float scale;           /* > 0, at most 2^95; in the backward of bf16 storage at least 2^-120                                  */
} spes_attn_shape;

/*  q         DEVICE [q_rows, heads, head_dim]     k, v  DEVICE [k_rows, kv_heads, head_dim], strides in the shape
 *  q_start   DEVICE [n_seq + 1] i32, ascending    k_start  DEVICE [n_seq + 1] i32, ascending (with k_len [n_seq], in any order)
 *  k_len     DEVICE [n_seq] i32 or NULL
 *  o         DEVICE [q_rows, heads, head_dim] out
 *  lse       DEVICE [heads, q_rows] f32 out
 *  scratch   DEVICE, spes_attn_scratch_bytes(shape, 0) bytes
 */
SPES_API size_t spes_attn_scratch_bytes(const spes_attn_shape* shape, int32_t backward);
SPES_API int spes_attn_fwd(const spes_attn_shape* shape, const void* q, const void* k, const void* v,
                           const int32_t* q_start, const int32_t* k_start, const int32_t* k_len, void* o,
                           float* lse, void* scratch, void* stream);

/* Its backward for the upstream gradient d_o of o.  The probabilities are formed again from q, k and lse, and sum d_o o is taken of o as it is stored.
 *
 *  d_o       DEVICE [q_rows, heads, head_dim]
 *  o, lse    as the forward left them; all other inputs as above
 *  dq        DEVICE out, laid out as q is;  dk, dv  DEVICE out, laid out as k and v are.  They are overwritten.  These layouts must not put two
 *            elements into one place: rows lie beyond all heads of the one before, or heads beyond all rows
 *  scratch   DEVICE, spes_attn_scratch_bytes(shape, 1) bytes
 */
SPES_API int spes_attn_bwd(const spes_attn_shape* shape, const void* d_o, const void* q, const void* k,
                           const void* v, const int32_t* q_start, const int32_t* k_start,
                           const int32_t* k_len, const void* o, const float* lse, void* dq, void* dk,
                           void* dv, void* scratch, void* stream);

SPES_API const char* spes_strerror(int code);

#ifdef __cplusplus
}
#endif
#endif /* SPES_H_ */
