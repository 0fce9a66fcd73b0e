/*
 * libmhlmoe — the per-GPU hot path of Multi-Head LatentMoE on AMD MI355X
 * (gfx950): IO-aware routing and IO-aware expert computation.
 *
 * Paper: "Multi-Head LatentMoE" (arXiv 2602.04870).
 *
 * Each of the N_h heads is an independent Mixtral-style MoE (Eq. (1)-(4),
 * Sec. 2.2) applied to its d_h-wide slice of the latent token (Eq. (5)-(6),
 * Sec. 3.1).  The library computes, for every token t and head h:
 *
 *   s[e]    = X[t,h,:] . W_router[h,e,:]                     (FP32 router)
 *   key[e]  = s[e] + bias[h,e]                   (Algorithm 1, bias optional)
 *   idx     = the top_k experts by key, descending; ties -> lower index
 *   gate[j] = softmax_j( s[idx_j] )             (bias removed, Eq. (2)-(3))
 *   Y[t,h]  = sum_j gate[j] * W2 (silu(W1 x) * (W3 x)) with the weights of
 *             expert idx_j of head h                        (Eq. (1), SwiGLU)
 *
 * without writing the T x N_e score matrix or the d_ff-wide expert
 * intermediate to device memory (Sec. 3.3, Sec. 3.4).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Tensor pointers are DEVICE pointers owned by the caller; the library
 *    never allocates device memory for tensors, frees or synchronises (the
 *    latent-layer entry points create a hipBLASLt handle once per device).  All work is enqueued on
 *    `stream` (a hipStream_t; NULL = the default stream) and the call returns
 *    without waiting.  Inputs must stay valid until that work completes.
 *  - Layouts are dense row-major; element (a,b,c) of [A][B][C] is at
 *    (a*B + b)*C + c.  Pointers must be 16-byte aligned.
 *  - `dtype` selects the element type of X, W1, W3, W2, Y, dY and dX:
 *    MHLMOE_F32 (float) or MHLMOE_BF16 (bfloat16 stored as uint16).
 *    W_router and bias are always float; idx, counts, offsets and perm are
 *    int32; gate is float; weight gradients are float.
 *  - Scratch memory comes from `workspace`, a device buffer of at least
 *    mhlmoe_workspace_size(...) bytes, 256-byte aligned, owned by the
 *    caller.  Its contents need no initialisation and are clobbered.
 *    Concurrent calls must use distinct workspaces.
 *  - Supported shapes: d_head in {64, 128}; d_ff a multiple of 32 in [32, 512];
 *    1 <= top_k <= 32; top_k <= n_experts <= 1024; 1 <= n_heads <= 1024;
 *    0 <= T and T * top_k < 2^31.  T = 0 is a valid no-op.
 *  - Errors: every call returns a mhlmoe_status; on failure nothing has
 *    been enqueued (argument errors) or a launch failed (MHLMOE_EHIP), and
 *    mhlmoe_last_error() gives a message for the calling thread.
 *  - Determinism: every forward output (idx, gate, counts, offsets, perm, Y)
 *    and every gradient is bitwise reproducible for identical inputs and
 *    shapes; no floating-point atomics are used.
 */
#ifndef MHLMOE_H
#define MHLMOE_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum mhlmoe_status {
    MHLMOE_OK = 0,
    MHLMOE_EINVAL = 1,       /* bad pointer, shape or alignment; k > N_e    */
    MHLMOE_EUNSUPPORTED = 2, /* shape outside the compiled set              */
    MHLMOE_EWORKSPACE = 3,   /* workspace missing or smaller than required  */
    MHLMOE_EHIP = 4          /* a HIP launch or runtime call failed         */
} mhlmoe_status;

typedef enum mhlmoe_dtype {
    MHLMOE_F32 = 0,
    MHLMOE_BF16 = 1,
    /* widens the type to every non-negative int, so that a caller's
     * out-of-range value is a defined value the library rejects */
    MHLMOE_DTYPE_FORCE_INT32 = 0x7FFFFFFF
} mhlmoe_dtype;

typedef enum mhlmoe_op {
    MHLMOE_OP_ROUTE = 0,
    MHLMOE_OP_BUCKET = 1,
    MHLMOE_OP_EXPERTS = 2,
    MHLMOE_OP_LAYER = 3,
    MHLMOE_OP_LAYER_BACKWARD = 4,
    MHLMOE_OP_LATENT_LAYER = 5,
    MHLMOE_OP_LATENT_BACKWARD = 6,
    MHLMOE_OP_ROUTE_BACKWARD = 7,
    MHLMOE_OP_FORCE_INT32 = 0x7FFFFFFF /* as MHLMOE_DTYPE_FORCE_INT32 */
} mhlmoe_op;

/* Library version as MAJOR*10000 + MINOR*100 + PATCH. */
int mhlmoe_version(void);

/* Message describing the last failure on the calling thread ("" if none).
 * The pointer stays valid until the next libmhlmoe call on this thread. */
const char *mhlmoe_last_error(void);

/*
 * Workspace bytes that entry point `op` needs for this shape (d_ff and dtype
 * are ignored by MHLMOE_OP_ROUTE and MHLMOE_OP_BUCKET).  Writes *bytes and
 * returns MHLMOE_OK, or an error status for an invalid or unsupported shape.
 */
mhlmoe_status mhlmoe_workspace_size(mhlmoe_op op, int64_t T, int n_heads,
                                    int d_head, int n_experts, int top_k,
                                    int d_ff, mhlmoe_dtype dtype,
                                    size_t *bytes);

/*
 * IO-aware routing forward: Algorithm 1 (Sec. 3.3) with the gate of
 * Eq. (2)-(4) and the per-expert load counts.
 *
 *   X        [T][n_heads][d_head]        dtype          (in)
 *   W_router [n_heads][n_experts][d_head] float          (in)  — the paper's
 *            W_r[h] is d_head x n_experts; this is its transpose, so each
 *            expert's row is contiguous.
 *   bias     [n_heads][n_experts] float or NULL           (in)  — Algorithm
 *            1's load-balancing bias: added to the scores before the top-k,
 *            removed after, so it steers selection but never the gates.
 *   idx      [T][n_heads][top_k] int32                    (out) — selected
 *            experts in descending biased-score order, ties to the lower
 *            expert index.
 *   gate     [T][n_heads][top_k] float                    (out) — softmax
 *            over the k selected unbiased scores.
 *   counts   [n_heads][n_experts] int32                   (out) — number of
 *            (t, j) with idx[t][h][j] == e.
 * Scores are computed to fp32 accuracy (the paper's FP32 router) and never
 * leave the chip.  Non-finite scores give unspecified indices.
 */
mhlmoe_status mhlmoe_route(const void *X, const float *W_router,
                           const float *bias, int64_t T, int n_heads,
                           int d_head, int n_experts, int top_k,
                           mhlmoe_dtype dtype, int32_t *idx, float *gate,
                           int32_t *counts, void *workspace,
                           size_t workspace_bytes, hipStream_t stream);

/*
 * mhlmoe_route without a workspace, for callers that cannot allocate device
 * memory: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc.  Arguments, results and kernels are those of
 * mhlmoe_route; the scratch (per-block expert histograms, counts) lives in a
 * static device array of 32 MiB that the library holds on every device it
 * runs on until the process ends (its device address is looked up once per
 * device, on the first call there).  The call allocates nothing and frees
 * nothing.  Shapes needing more than 32 MiB of scratch (4 (n_heads *
 * ceil(T / 128) + 1) n_experts bytes, roughly; e.g. T = 65536, 8 heads,
 * 1024 experts needs 16 MiB) return MHLMOE_EWORKSPACE before anything is
 * enqueued.  Nothing in the scratch needs to start at zero.  All calls on
 * one device share its array: calls that overlap in time on one device
 * (other streams, other threads) race and must be ordered by the caller.
 */
mhlmoe_status mhlmoe_route_static(const void *X, const float *W_router,
                                  const float *bias, int64_t T, int n_heads,
                                  int d_head, int n_experts, int top_k,
                                  mhlmoe_dtype dtype, int32_t *idx,
                                  float *gate, int32_t *counts,
                                  hipStream_t stream);

/*
 * IO-aware routing backward, Algorithm 2 (Sec. 3.3) on its own: given the
 * forward's idx and gate and the gradient dgate of a loss with respect to
 * the gates,
 *   dS_j = g_j (dgate_j - sum_j' g_j' dgate_j')       (softmax backward)
 *   dX[t][h] = sum_j dS_j W_router[h][e_j]
 *   dW_router[h][e] = sum over the (t, j) with e_j = e of dS_j X[t][h]
 * Gradients reach only the k selected experts of each token (no T x N_e
 * matrix); none reaches the bias or the selection.
 *
 *   X, W_router, idx, gate    the forward's inputs and outputs      (in)
 *   dgate [T][n_heads][top_k] float                                (in)
 *   dX    [T][n_heads][d_head] dtype                               (out)
 *   dW_router [n_heads][n_experts][d_head] float (out, overwritten;
 *             experts that received no slot get exact zeros)
 * dW_router is a fixed-order segmented sum over the clustered slots, so the
 * results are bitwise reproducible.  idx entries must lie in [0, n_experts).
 * Workspace: MHLMOE_OP_ROUTE_BACKWARD (d_ff ignored).
 */
mhlmoe_status mhlmoe_route_backward(const void *X, const float *W_router,
                                    const int32_t *idx, const float *gate,
                                    const float *dgate, int64_t T, int n_heads,
                                    int d_head, int n_experts, int top_k,
                                    mhlmoe_dtype dtype, void *dX,
                                    float *dW_router, void *workspace,
                                    size_t workspace_bytes, hipStream_t stream);

/*
 * Token clustering (Sec. 3.4, Fig. 2): a stable counting sort of every
 * head's routed slots by expert, so each expert's tokens are contiguous.
 *
 *   idx     [T][n_heads][top_k] int32    (in)  values in [0, n_experts)
 *   counts  [n_heads][n_experts] int32   (out, may be NULL)
 *   offsets [n_heads][n_experts + 1]     (out) exclusive prefix sum of counts;
 *           offsets[h][n_experts] = T * top_k.
 *   perm    [n_heads][T * top_k] int32   (out) perm[h][offsets[h][e] + r] is
 *           the slot id t*top_k + j of the r-th slot, in ascending (t, j)
 *           order, routed to expert e in head h.
 * Out-of-range idx values give unspecified results (no fault).
 */
mhlmoe_status mhlmoe_bucket(const int32_t *idx, int64_t T, int n_heads,
                            int n_experts, int top_k, int32_t *counts,
                            int32_t *offsets, int32_t *perm, void *workspace,
                            size_t workspace_bytes, hipStream_t stream);

/*
 * IO-aware expert computation (Sec. 3.4), dropless, and the gate-weighted
 * combine of Eq. (1); the per-head outputs are laid side by side, which is
 * the concat of Eq. (6).
 *
 *   X    [T][n_heads][d_head]                 dtype   (in)
 *   idx  [T][n_heads][top_k] int32                    (in)
 *   gate [T][n_heads][top_k] float                    (in)
 *   W1   [n_heads][n_experts][d_ff][d_head]   dtype   (in) gate projection
 *   W3   [n_heads][n_experts][d_ff][d_head]   dtype   (in) up projection
 *   W2   [n_heads][n_experts][d_head][d_ff]   dtype   (in) down projection
 *   Y    [T][n_heads][d_head]                 dtype   (out)
 * Every slot is computed (no capacity limit); the d_ff-wide intermediate
 * stays on chip.  Accumulation is fp32; bf16 results are rounded to nearest
 * even once per output element.
 */
mhlmoe_status mhlmoe_experts(const void *X, const int32_t *idx,
                             const float *gate, const void *W1, const void *W3,
                             const void *W2, int64_t T, int n_heads,
                             int d_head, int n_experts, int top_k, int d_ff,
                             mhlmoe_dtype dtype, void *Y, void *workspace,
                             size_t workspace_bytes, hipStream_t stream);

/*
 * The whole per-GPU layer: mhlmoe_route then mhlmoe_experts, sharing the
 * routing kernel's per-block expert histograms with the clustering step.
 * Arguments as above.  idx, gate and counts are optional outputs (NULL keeps
 * them in the workspace); pass idx and gate to run mhlmoe_layer_backward.
 */
mhlmoe_status mhlmoe_layer(const void *X, const float *W_router,
                           const float *bias, const void *W1, const void *W3,
                           const void *W2, int64_t T, int n_heads, int d_head,
                           int n_experts, int top_k, int d_ff,
                           mhlmoe_dtype dtype, void *Y, int32_t *idx,
                           float *gate, int32_t *counts, void *workspace,
                           size_t workspace_bytes, hipStream_t stream);

/*
 * The paper's own expert form (Sec. 3.4): each expert is the two-matrix
 * GELU MLP  y = W_out gelu(W_in x),  gelu(z) = z Phi(z) (the exact, erf
 * form), which Sec. 3.4 evaluates as block-sparse attention with
 * score_mod(s) = log(gelu(s) + 1).  Everything else (routing, clustering,
 * the gate-weighted combine of Eq. (1)) is as in mhlmoe_experts and
 * mhlmoe_layer, with the same workspace sizes (MHLMOE_OP_EXPERTS and
 * MHLMOE_OP_LAYER).
 *
 *   W_in  [n_heads][n_experts][d_ff][d_head]  dtype   (W1's layout)  (in)
 *   W_out [n_heads][n_experts][d_head][d_ff]  dtype   (W2's layout)  (in)
 *
 * Supported: the shapes of mhlmoe_experts / mhlmoe_layer (dtype MHLMOE_BF16
 * or MHLMOE_F32, d_head 64 or 128, the paper's 16 x 64 and 8 x 128 head
 * configurations among them, d_ff a multiple of 32 in [32, 512]); other
 * shapes return MHLMOE_EUNSUPPORTED.  On the GPU Phi is a logistic function
 * of a fitted odd polynomial, Phi(z) ~ 1 / (1 + exp(-z P(z^2))) with P of
 * degree 4 (|Phi error| <= 1.6e-6), below the rounding of the intermediate
 * (bf16) and within the fp32 tolerance.
 */
mhlmoe_status mhlmoe_experts_gelu(const void *X, const int32_t *idx,
                                  const float *gate, const void *W_in,
                                  const void *W_out, int64_t T, int n_heads,
                                  int d_head, int n_experts, int top_k,
                                  int d_ff, mhlmoe_dtype dtype, void *Y,
                                  void *workspace, size_t workspace_bytes,
                                  hipStream_t stream);

mhlmoe_status mhlmoe_layer_gelu(const void *X, const float *W_router,
                                const float *bias, const void *W_in,
                                const void *W_out, int64_t T, int n_heads,
                                int d_head, int n_experts, int top_k, int d_ff,
                                mhlmoe_dtype dtype, void *Y, int32_t *idx,
                                float *gate, int32_t *counts, void *workspace,
                                size_t workspace_bytes, hipStream_t stream);

/*
 * Backward of mhlmoe_layer: Algorithm 2 (routing backward, gradients only
 * for the k selected experts, Sec. 3.3) and the gradient of Eq. (1)-(3) with
 * the SwiGLU expert, recomputing the expert intermediate instead of storing
 * it.  No gradient flows through the selection or to the bias.
 *
 *   X, W_router, W1, W3, W2   forward inputs                  (in)
 *   idx, gate                 the forward's outputs           (in)
 *   dY   [T][n_heads][d_head] dtype                           (in)
 *   dX   [T][n_heads][d_head] dtype                           (out)
 *   dW_router [n_heads][n_experts][d_head] float              (out)
 *   dW1, dW3  [n_heads][n_experts][d_ff][d_head] float        (out)
 *   dW2       [n_heads][n_experts][d_head][d_ff] float        (out)
 * Weight gradients are overwritten, not accumulated into; experts that
 * received no slot get exact zeros.  dtype must be MHLMOE_BF16 (activations,
 * dY, dX and expert weights bf16; MHLMOE_EUNSUPPORTED otherwise); gradients
 * are accumulated in fp32 and the sums are taken in a fixed order, so equal
 * inputs give bitwise equal outputs.  idx entries must lie in
 * [0, n_experts) (the forward guarantees it); other values are not
 * detected.  Same shape limits as mhlmoe_layer.
 */
mhlmoe_status mhlmoe_layer_backward(
    const void *X, const float *W_router, const void *W1, const void *W3,
    const void *W2, const int32_t *idx, const float *gate, const void *dY,
    int64_t T, int n_heads, int d_head, int n_experts, int top_k, int d_ff,
    mhlmoe_dtype dtype, void *dX, float *dW_router, float *dW1, float *dW3,
    float *dW2, void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Backward of mhlmoe_layer_gelu (the two-matrix GELU expert of Sec. 3.4):
 * as mhlmoe_layer_backward with u = gelu(a), a = W_in x, and
 *   da = (g W_out^T dY) * gelu'(a),  gelu'(z) = Phi(z) + z phi(z),
 *   dX_expert = W_in^T da,  dW_in = sum da x^T,  dW_out = sum (g dY) u^T.
 *   dW_in  [n_heads][n_experts][d_ff][d_head] float  (out)
 *   dW_out [n_heads][n_experts][d_head][d_ff] float  (out)
 * dtype MHLMOE_BF16 (fp32 returns MHLMOE_EUNSUPPORTED, as for
 * mhlmoe_layer_backward); d_head in {64, 128}, d_ff a multiple of 32 up to
 * 512.  On the GPU
 * Phi comes from the Abramowitz & Stegun 7.1.26 erf (|error| <= 1.5e-7) and
 * phi from the exponential it already evaluates; the recomputed gelu(a)
 * differs from the forward's by at most 1.6e-6 |a|.  Workspace:
 * MHLMOE_OP_LAYER_BACKWARD.
 */
mhlmoe_status mhlmoe_layer_gelu_backward(
    const void *X, const float *W_router, const void *W_in, const void *W_out,
    const int32_t *idx, const float *gate, const void *dY, int64_t T,
    int n_heads, int d_head, int n_experts, int top_k, int d_ff,
    mhlmoe_dtype dtype, void *dX, float *dW_router, float *dW_in,
    float *dW_out, void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * Separate routing sub-tokens (Sec. 4.4, Eq. (9)): W_in x is split into
 * 2 n_heads sub-tokens, x_{t,i} for the experts and r_{t,i} for the router.
 * The layer routes head h of token t by R[t][h] and computes the experts on
 * X[t][h]; everything else is as in mhlmoe_layer.  W3 == NULL selects the
 * two-matrix GELU expert (W1 = W_in, W2 = W_out, with mhlmoe_layer_gelu's
 * shape limits).  With R == X the outputs equal mhlmoe_layer's (or
 * mhlmoe_layer_gelu's) bit for bit.  Workspace: MHLMOE_OP_LAYER.
 *
 *   R  [T][n_heads][d_head]  dtype  (in)  the routing sub-tokens
 */
mhlmoe_status mhlmoe_layer_routed(const void *X, const void *R,
                                  const float *W_router, const float *bias,
                                  const void *W1, const void *W3,
                                  const void *W2, int64_t T, int n_heads,
                                  int d_head, int n_experts, int top_k,
                                  int d_ff, mhlmoe_dtype dtype, void *Y,
                                  int32_t *idx, float *gate, int32_t *counts,
                                  void *workspace, size_t workspace_bytes,
                                  hipStream_t stream);

/*
 * Backward of mhlmoe_layer_routed (bf16): as mhlmoe_layer_backward (W3 ==
 * NULL: as mhlmoe_layer_gelu_backward, dW3 unused), except that Algorithm
 * 2's router gradients are taken against R: dR receives
 * sum_j dS_j W_router[h][e_j] and dW_router sums dS_j R[t][h], while dX
 * holds the expert input gradient only.
 *
 *   R   [T][n_heads][d_head]  bf16  (in)
 *   dR  [T][n_heads][d_head]  bf16  (out) a buffer distinct from dX; may be
 *                                   NULL only when T == 0.
 * Workspace: MHLMOE_OP_LAYER_BACKWARD.  The expert weight gradients equal
 * mhlmoe_layer_backward's bit for bit at the same (X, idx, gate, dY).
 */
mhlmoe_status mhlmoe_layer_backward_routed(
    const void *X, const void *R, const float *W_router, const void *W1,
    const void *W3, const void *W2, const int32_t *idx, const float *gate,
    const void *dY, int64_t T, int n_heads, int d_head, int n_experts,
    int top_k, int d_ff, mhlmoe_dtype dtype, void *dX, void *dR,
    float *dW_router, float *dW1, float *dW3, float *dW2, void *workspace,
    size_t workspace_bytes, hipStream_t stream);

/*
 * The whole Multi-Head LatentMoE layer with its projections (Eq. (5)-(6),
 * Sec. 3.1), N = n_heads * d_head latent width:
 *
 *   X_lat = W_in x                 [T][N], read as [T][n_heads][d_head]: the
 *                                  split of Eq. (5) is a view, no copy
 *   Y_lat = the per-head MoEs of mhlmoe_layer on X_lat (idx, gate, counts
 *           as there; W3 == NULL selects the two-matrix GELU expert)
 *   out   = W_out concat(Y_lat)    [T][d_model] (Eq. (6))
 *
 * routing_tokens = 1 gives the separate routing sub-tokens of Sec. 4.4,
 * Eq. (9): W_in then has 2N rows, its first N produce X_lat and its last N
 * the routing sub-tokens R_lat, which the router reads instead of X_lat.
 *
 *   x      [T][d_model]                         dtype  (in)
 *   W_in   [(1 + routing_tokens) N][d_model]    dtype  (in)
 *   W_out  [d_model][N]                         dtype  (in)
 *   out    [T][d_model]                         dtype  (out)
 *   X_lat, R_lat, Y_lat [T][n_heads][d_head]    dtype  (out, optional: NULL
 *          keeps them in the workspace; keep X_lat, Y_lat (and R_lat) for
 *          mhlmoe_latent_layer_backward)
 * The projections are hipBLASLt GEMMs with fp32 accumulation, rounded once
 * to dtype; the library creates one hipBLASLt handle per device on first use
 * and caches a GEMM plan per shape (the only host-side allocations of the
 * library besides the timing events).  Their results are reproducible for a
 * given hipBLASLt build and shape.  1 <= d_model <= 65536.  Workspace:
 * MHLMOE_OP_LATENT_LAYER (d_model does not change its size).
 */
mhlmoe_status mhlmoe_latent_layer(const void *x, const void *W_in,
                                  const float *W_router, const float *bias,
                                  const void *W1, const void *W3,
                                  const void *W2, const void *W_out,
                                  int64_t T, int d_model, int n_heads,
                                  int d_head, int n_experts, int top_k,
                                  int d_ff, int routing_tokens,
                                  mhlmoe_dtype dtype, void *out, void *X_lat,
                                  void *R_lat, void *Y_lat, int32_t *idx,
                                  float *gate, int32_t *counts,
                                  void *workspace, size_t workspace_bytes,
                                  hipStream_t stream);

/*
 * Backward of mhlmoe_latent_layer (bf16; W3 == NULL: the GELU expert, dW3
 * unused), given the
 * forward's x, X_lat, (R_lat), Y_lat, idx and gate and the output gradient
 * dout [T][d_model]:
 *
 *   dY_lat = dout W_out;  dW_out = dout^T Y_lat
 *   the heads' backward of mhlmoe_layer_backward (mhlmoe_layer_backward_routed
 *   with routing sub-tokens) on X_lat and dY_lat -> dX_lat (dR_lat) and
 *   dW_router, dW1, dW3, dW2
 *   dW_in = [dX_lat; dR_lat]^T x;  dx = dX_lat W_in_x (+ dR_lat W_in_r)
 *
 *   dx     [T][d_model]                        bf16   (out)
 *   dW_in  [(1 + routing_tokens) N][d_model]   float  (out)
 *   dW_out [d_model][N]                        float  (out)
 *   dW_router, dW1, dW3, dW2 as in mhlmoe_layer_backward (out)
 * dY_lat, dX_lat and dR_lat are rounded to bf16 in the workspace; with
 * routing sub-tokens dx is the bf16 sum of its two products (accumulated by
 * the second GEMM).  Workspace: MHLMOE_OP_LATENT_BACKWARD.
 */
mhlmoe_status mhlmoe_latent_layer_backward(
    const void *x, const void *W_in, const float *W_router, const void *W1,
    const void *W3, const void *W2, const void *W_out, const void *X_lat,
    const void *R_lat, const void *Y_lat, const int32_t *idx,
    const float *gate, const void *dout, int64_t T, int d_model, int n_heads,
    int d_head, int n_experts, int top_k, int d_ff, int routing_tokens,
    mhlmoe_dtype dtype, void *dx, float *dW_in, float *dW_router, float *dW1,
    float *dW3, float *dW2, float *dW_out, void *workspace,
    size_t workspace_bytes, hipStream_t stream);

/*
 * Auxiliary-loss-free load balancing (Sec. 2.2, after the aux-free method it
 * cites): after a batch, every head's routing bias (Algorithm 1's b) moves
 * toward equal expert load by a fixed rate,
 *
 *   bias[h][e] += rate * sign(mean_e' counts[h][e'] - counts[h][e]),
 *
 * with sign(0) = 0, the mean compared exactly in integers and each bias
 * changed by one fp32 addition (round to nearest even).
 *
 *   counts [n_heads][n_experts] int32  (in)  e.g. mhlmoe_layer's counts,
 *                                      summed over the batches of a step
 *   bias   [n_heads][n_experts] float  (in/out, updated in place)
 *   rate   the update rate u, finite and >= 0 (MHLMOE_EINVAL otherwise)
 * 1 <= n_heads <= 1024, 1 <= n_experts <= 1024; no workspace.  The call
 * enqueues one kernel on `stream`; calls that update the same bias must be
 * ordered by the caller.
 */
mhlmoe_status mhlmoe_bias_update(const int32_t *counts, float *bias,
                                 int n_heads, int n_experts, float rate,
                                 hipStream_t stream);

/*
 * The operators around the heads: what stands between the layer and the
 * network it is in.  8 bits are e4m3 (OCP: largest value 448, no infinities)
 * with one float scale per block of 128 values along the contraction; a block
 * of values v is held as
 *
 *   scale = max(max |v| / 448, 2^-126),   q = e4m3(v / scale), nearest even,
 *
 * so q * scale stands for v; the last block of a row may be shorter.  The scale
 * is rounded to fp32, and v / scale is taken in fp32 (within an ulp) on its way
 * to e4m3: a quotient within an fp32 step of a border between two of e4m3's
 * values, as those of bf16 values often are, can count as lying on it.  A block
 * that holds an infinity or a NaN becomes NaN as a whole.
 *
 * Residual sum and root-mean-square norm, per row t of d_model columns c:
 *
 *   h = x + residual, rounded to dtype        (h = x where residual is NULL)
 *   y[c] = h[c] / sqrt(mean_c' h[c']^2 + eps) * weight[c]
 *
 *   x        [T][d_model]  dtype                     (in)
 *   residual [T][d_model]  dtype or NULL             (in)
 *   weight   [d_model]     float                     (in)
 *   sum      [T][d_model]  dtype  h, with residual only (out); may be x or
 *            residual itself
 *   y        [T][d_model]  dtype or NULL             (out); may be x
 *   q        [T][d_model]  e4m3 or NULL              (out) y in 8 bits, with
 *   scales   [T][ceil(d_model / 128)] float          (out) its scales; d_model
 *            must be a multiple of 16
 * y and q may both be asked for; at least one must be.  The norm is that of
 * the rounded h, which mhlmoe_rmsnorm_backward reads.  1 <= d_model <= 65536,
 * T < 2^31, eps finite and > 0.  Sums and the norm are in fp32: where the sum
 * of a row's squares is infinite there, its finite elements become zeros.  No
 * workspace.
 */
mhlmoe_status mhlmoe_rmsnorm(const void *x, const void *residual,
                             const float *weight, int64_t T, int d_model,
                             float eps, mhlmoe_dtype dtype, void *sum, void *y,
                             void *q, float *scales, hipStream_t stream);

/*
 * Its gradient, with rs = 1 / sqrt(mean_c h^2 + eps) and g = dy * weight:
 *
 *   dx[c] = dsum[c] + rs (g[c] - h[c] rs^2 mean_c'(g[c'] h[c']))
 *   dweight[c] = sum_t dy[c] h[c] rs
 *
 *   h       [T][d_model]  dtype  the forward's sum (x without residual) (in)
 *   dy      [T][d_model]  dtype  the gradient of y                      (in)
 *   dsum    [T][d_model]  dtype or NULL  the gradient that reaches h past the
 *           norm (the residual stream's)                                (in)
 *   dx      [T][d_model]  dtype  the gradient of x, and of residual    (out);
 *           may be dy or dsum, not h
 *   dweight [d_model]     float  overwritten; zeros where T = 0        (out)
 * dweight is summed in a fixed order.  Workspace: the size that
 * mhlmoe_rmsnorm_backward_workspace writes to *bytes.
 */
mhlmoe_status mhlmoe_rmsnorm_backward_workspace(int64_t T, int d_model,
                                                size_t *bytes);
mhlmoe_status mhlmoe_rmsnorm_backward(const void *h, const float *weight,
                                      const void *dy, const void *dsum,
                                      int64_t T, int d_model, float eps,
                                      mhlmoe_dtype dtype, void *dx,
                                      float *dweight, void *workspace,
                                      size_t workspace_bytes,
                                      hipStream_t stream);

/*
 * Quantisation of x [rows][cols] (dtype; cols a multiple of 16) in blocks of
 * block_rows x 128: block_rows 1 gives every row its own scales (activations),
 * 128 one scale per tile (weights).
 *
 *   transpose 0:  q [rows][cols] e4m3,
 *                 scales [ceil(rows / block_rows)][ceil(cols / 128)] float
 *   transpose 1:  x^T is quantised, its rows padded with zeros to a multiple
 *                 of 16:  q [cols][rows16], rows16 = 16 ceil(rows / 16),
 *                 scales [ceil(cols / block_rows)][ceil(rows / 128)]
 * The transposed forms serve the gradients of mhlmoe_gemm_scaled: with C = A
 * B^T, dA = dC B contracts over N and dB = dC^T A over M.  A 128 x 128 block's
 * scale is the same either way.  rows, cols < 2^31 and fewer than 2^24 tiles
 * of 128 x 128 (2^32 blocks of 1 x 128).  No workspace.
 */
mhlmoe_status mhlmoe_quantize(const void *x, int64_t rows, int64_t cols,
                              mhlmoe_dtype dtype, int block_rows, int transpose,
                              void *q, float *scales, hipStream_t stream);

/*
 * The 8-bit product C = A B^T with a scale per block of 128, KB = ceil(K / 128):
 *
 *   C[m][n] = sum_b scale_a[m][b] scale_b[n / b_block_rows][b]
 *                   sum_{k = 128 b .. 128 b + 127} A[m][k] B[n][k]
 *
 *   A       [M][K] e4m3,  scale_a [M][KB] float                         (in)
 *   B       [N][K] e4m3,  scale_b [ceil(N / b_block_rows)][KB] float    (in)
 *   C       [M][N] out_dtype                                           (out)
 * b_block_rows is 128 (weights quantised in tiles) or 1 (both operands
 * quantised by rows: the weight gradient).  K must be a multiple of 16; M and
 * N are any sizes (C's rows then need no alignment).
 *
 * A block's sum depends on out_dtype.  MHLMOE_F32: the products are exact and
 * added in fp32.  MHLMOE_BF16: the 8-bit matrix instructions (twice the rate)
 * add eight products of a block at a time and drop of each what lies below
 * 2^-13 of the largest of the eight, then add the groups in fp32.  Besides the
 * roundings of fp32 a result is so off by up to 7 * 2^-13 of the sum of its
 * terms' magnitudes before it is rounded to bf16: nothing next to that rounding
 * where the terms are alike (about 1e-5 of the result for random operands), but
 * products below 2^-13 of others that cancel are lost.  A caller who needs them
 * asks for MHLMOE_F32.
 *
 * A block's two scales are multiplied in fp32 before they meet its sum: the
 * product must not overflow, and below 2^-126 it loses bits, down to zero, even
 * where the block's sum (up to 448 * 448 * 128 < 2^25) would lift the result back.
 * Blocks are added in fp32 in a fixed order; C is rounded once.  K = 0 writes
 * zeros.  M, N < 2^31, K < 2^23, ceil(M / 128) ceil(N / 128) < 2^24.  No workspace.
 */
mhlmoe_status mhlmoe_gemm_scaled(const void *A, const float *scale_a,
                                 const void *B, const float *scale_b, int64_t M,
                                 int64_t N, int64_t K, int b_block_rows,
                                 mhlmoe_dtype out_dtype, void *C,
                                 hipStream_t stream);

/*
 * mhlmoe_latent_layer for serving, behind its norm and with its projections in
 * 8 bits (N = n_heads * d_head):
 *
 *   h     = x + residual (to sum); n = its RMS norm in 8 bits (mhlmoe_rmsnorm)
 *   X_lat = n W_in^T,  R_lat = n W_r^T (W_r NULL: R_lat is X_lat)
 *   Y_lat = the heads on X_lat, routed by R_lat (mhlmoe_layer_routed)
 *   out   = Y_lat, quantised by rows, W_out^T
 *
 * bit for bit what the named calls, mhlmoe_quantize and mhlmoe_gemm_scaled
 * give one by one.  W_in, W_r [N][d_model] and W_out [d_model][N] are e4m3 with
 * scales per 128 x 128 tile (mhlmoe_quantize, block_rows 128); W_r gives the
 * separate routing sub-tokens of Eq. (9).  residual and sum, X_lat, R_lat,
 * Y_lat, idx, gate and counts are optional as in the calls themselves.
 * The products are mhlmoe_gemm_scaled's with out_dtype = dtype: the latent
 * activations, and with them the routing, of a bf16 layer carry its 8-bit sums.
 * d_model must be a multiple of 16 in [16, 65536].  Workspace: the size that
 * mhlmoe_latent_layer_scaled_workspace writes to *bytes, which has room for
 * X_lat, R_lat and Y_lat whether or not the caller passes them.
 */
mhlmoe_status mhlmoe_latent_layer_scaled_workspace(
    int64_t T, int d_model, int n_heads, int d_head, int n_experts, int top_k,
    int d_ff, mhlmoe_dtype dtype, size_t *bytes);
mhlmoe_status mhlmoe_latent_layer_scaled(
    const void *x, const void *residual, const float *norm_weight, float eps,
    const void *W_in, const float *scale_in, const void *W_r,
    const float *scale_r, const float *W_router, const float *bias,
    const void *W1, const void *W3, const void *W2, const void *W_out,
    const float *scale_out, int64_t T, int d_model, int n_heads, int d_head,
    int n_experts, int top_k, int d_ff, mhlmoe_dtype dtype, void *out,
    void *sum, void *X_lat, void *R_lat, void *Y_lat, int32_t *idx, float *gate,
    int32_t *counts, void *workspace, size_t workspace_bytes,
    hipStream_t stream);

/*
 * What a training step has around the layer besides: layer norm, the loss that
 * balances the experts by gradient, and the optimiser's step.
 *
 * Residual sum and layer norm, per row t of d_model columns c:
 *
 *   h = x + residual, rounded to dtype        (h = x where residual is NULL)
 *   y[c] = (h[c] - mu) / sqrt(var + eps) * weight[c] + bias[c],
 *   mu = mean_c' h[c'],  var = mean_c' (h[c'] - mu)^2
 *
 *   bias [d_model] float or NULL (zeros)                               (in)
 * The other arguments, what may be NULL, which of them may be the same tensor, the
 * 8-bit output and the extents are mhlmoe_rmsnorm's.  Sums are in fp32; a row that
 * holds an infinity or a NaN, or whose sums overflow there, becomes NaN or zeros
 * in itself only.  No workspace.
 */
mhlmoe_status mhlmoe_layernorm(const void *x, const void *residual,
                               const float *weight, const float *bias,
                               int64_t T, int d_model, float eps,
                               mhlmoe_dtype dtype, void *sum, void *y, void *q,
                               float *scales, hipStream_t stream);

/*
 * Its gradient, with rs = 1 / sqrt(var + eps), n = (h - mu) rs, g = dy * weight:
 *
 *   dx[c] = dsum[c] + rs (g[c] - mean_c' g[c'] - n[c] mean_c'(g[c'] n[c']))
 *   dweight[c] = sum_t dy[c] n[c],   dbias[c] = sum_t dy[c]
 *
 *   dbias [d_model] float or NULL (not wanted)  overwritten           (out)
 * and the other arguments as in mhlmoe_rmsnorm_backward.  dweight and dbias are
 * summed in a fixed order; zeros where T = 0.
 */
mhlmoe_status mhlmoe_layernorm_backward_workspace(int64_t T, int d_model,
                                                  size_t *bytes);
mhlmoe_status mhlmoe_layernorm_backward(const void *h, const float *weight,
                                        const void *dy, const void *dsum,
                                        int64_t T, int d_model, float eps,
                                        mhlmoe_dtype dtype, void *dx,
                                        float *dweight, float *dbias,
                                        void *workspace, size_t workspace_bytes,
                                        hipStream_t stream);

/*
 * Counts of the tokens that count:
 *
 *   counts[h][e] = #{(t, j): mask[t] != 0, idx[t][h][j] == e}
 *
 *   idx    [T][n_heads][top_k] int32; values outside [0, n_experts) are not
 *          counted                                                     (in)
 *   mask   [T] bytes or NULL (every token counts): 0 for a padded token (in)
 *   counts [n_heads][n_experts] int32, overwritten; zeros where T = 0 (out)
 * 1 <= n_heads, n_experts <= 1024, 1 <= top_k <= 32, T * top_k < 2^31.  No
 * workspace.
 */
mhlmoe_status mhlmoe_expert_counts(const int32_t *idx, const uint8_t *mask,
                                   int64_t T, int n_heads, int n_experts,
                                   int top_k, int32_t *counts,
                                   hipStream_t stream);

/*
 * The loss that balances a head's experts by gradient.  Over the n tokens of mask,
 * with p_t = softmax_e(X[t,h,:] . W_router[h,e,:]) over all experts and
 * f_e = counts[h][e] / sum_e' counts[h][e']:
 *
 *   loss[h] = n_experts sum_e f_e mean_t p_t(e)
 *
 * 1 for an even load or even probabilities, up to n_experts.  0 for a head whose
 * counts are all zero; 1 where they are not and no token counts (n = 0).
 *
 *   X        [T][n_heads][d_head]         dtype                         (in)
 *   W_router [n_heads][n_experts][d_head] float                         (in)
 *   counts   [n_heads][n_experts] int32, e.g. mhlmoe_expert_counts', or these
 *            summed over the batches or ranks of a step                 (in)
 *   mask     [T] bytes or NULL, as above                                (in)
 *   loss     [n_heads] float                                           (out)
 *   stats    [T + 1][n_heads][2] float, for the gradient: log sum_e' exp of the
 *            scores and sum_e p_t(e) (n_experts f_e - 1) of every token (zeros
 *            where it does not count), and 1 / max(n, 1) and 0 as row T (out)
 * X may hold anything at tokens that do not count, NaN and infinities too.
 * Scores are of fp32 accuracy (the paper's FP32 router) and never leave the chip.
 * A token with a score that is not finite makes its head's loss NaN.  |X| must stay
 * below 2^64 (the gradient's intermediate values overflow beyond).
 * d_head 64 or 128, 1 <= n_heads, n_experts <= 1024, (T + 128) * n_heads < 2^31.
 */
mhlmoe_status mhlmoe_balance_loss_workspace(int64_t T, int n_heads, int d_head,
                                            int n_experts, size_t *bytes);
mhlmoe_status mhlmoe_balance_loss(const void *X, const float *W_router,
                                  const int32_t *counts, const uint8_t *mask,
                                  int64_t T, int n_heads, int d_head,
                                  int n_experts, mhlmoe_dtype dtype, float *loss,
                                  float *stats, void *workspace,
                                  size_t workspace_bytes, hipStream_t stream);

/*
 * Its gradient (the counts are no function of the router), added to gradients
 * that are there already, such as mhlmoe_layer_backward's:
 *
 *   ds_t(e) = dloss[h] / n p_t(e) (n_experts f_e - 1 - stats[t][h][1])
 *   dX[t,h,:] = dX_add[t,h,:] + sum_e ds_t(e) W_router[h,e,:]
 *   dW_router[h,e,:] = dW_add[h,e,:] + sum_t ds_t(e) X[t,h,:]
 *
 *   dloss     [n_heads] float                                          (in)
 *   dX_add    [T][n_heads][d_head] dtype or NULL (zeros); may be dX    (in)
 *   dW_add    [n_heads][n_experts][d_head] float or NULL (zeros); may be
 *             dW_router                                                (in)
 *   dX        [T][n_heads][d_head] dtype; tokens that do not count get
 *             dX_add; not X                                           (out)
 *   dW_router [n_heads][n_experts][d_head] float; not W_router        (out)
 * The other arguments are those of the mhlmoe_balance_loss call that wrote
 * stats.  dX_add (dW_add) is added in fp32 before the one rounding of dX.  Products
 * are of fp32 accuracy: off by up to 2^-21 of themselves.  What is far below the largest
 * beside it has fewer bits: a value of X or W_router, here and in the scores, may be off
 * by 2^-39 of the largest of its token's row or of up to 256 experts next to it; and, with
 * D = dloss[h] / n, a term of dX by 2^-37 D R max |W_router[h]|, R = n_experts (max f -
 * min f), and one of dW_router by 2^-70 D.  p_t comes from the fp32 log sum in stats, so it
 * is off by about 2^-22 times the token's largest |score|.
 */
mhlmoe_status mhlmoe_balance_loss_backward_workspace(int64_t T, int n_heads,
                                                     int d_head, int n_experts,
                                                     size_t *bytes);
mhlmoe_status mhlmoe_balance_loss_backward(
    const void *X, const float *W_router, const int32_t *counts,
    const float *stats, const float *dloss, const uint8_t *mask,
    const void *dX_add, const float *dW_add, int64_t T, int n_heads, int d_head,
    int n_experts, mhlmoe_dtype dtype, void *dX, float *dW_router,
    void *workspace, size_t workspace_bytes, hipStream_t stream);

/*
 * One AdamW step over n_tensors tensors, per element in fp32:
 *
 *   g = grad_scale * grad
 *   m = beta1 m + (1 - beta1) g
 *   v = beta2 v + (1 - beta2) g^2
 *   p = p - lr (m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps)
 *               + weight_decay p)
 *
 * p is the fp32 master where there is one (param is then written as p rounded to
 * bf16, and not read), else param itself.
 */
typedef struct mhlmoe_adamw_tensor {
    void *param;   /* [n] param_dtype                               (in/out) */
    float *master; /* [n], with a bf16 param only, or NULL          (in/out) */
    const void *grad; /* [n] grad_dtype                                 (in) */
    void *m;       /* [n] float, or with scales e4m3                (in/out) */
    void *v;       /* [n] float; with scales sqrt(v) in e4m3        (in/out) */
    float *m_scale; /* [ceil(n / 128)], or NULL (32-bit states) ... (in/out) */
    float *v_scale; /* ... together with m_scale                    (in/out) */
    int64_t n;
    float weight_decay; /* finite and >= 0 */
    uint32_t seed;      /* of the 8-bit states' rounding */
    mhlmoe_dtype param_dtype, grad_dtype;
} mhlmoe_adamw_tensor;

typedef struct mhlmoe_adamw_step {
    double lr;           /* finite and >= 0 */
    double beta1, beta2; /* in [0, 1) */
    double eps;          /* finite, > 0 as a float */
    int64_t step;        /* from 1: the number of this step */
    const float *grad_scale; /* one float on the device, or NULL (1) */
} mhlmoe_adamw_step;

/*
 * The structs are read during the call and not kept.  m_scale and v_scale choose
 * 8-bit states: m and sqrt(v) are held in blocks of 128 consecutive elements of
 * the tensor (the last may be shorter) as described above for 8 bits, but each
 * value is rounded up or down at random, up with the probability of the part
 * below the step, and what is not zero of sqrt(v) does not become zero; a scale is
 * the largest magnitude times 1 / 448 (at most an ulp from the quotient).  Zero
 * states may be all zero bytes with any finite scales.  The random numbers are a
 * hash of seed, step and the element's place: the same call gives the same bits.
 * A value that is not finite makes its block of that state NaN.
 *
 * Memory that the step writes must not overlap any other memory of the step
 * (MHLMOE_EINVAL); tensors may share a gradient.  lr and step are the call's: a
 * captured call repeats the same step, and only grad_scale's value is read anew.
 * No workspace; one kernel for every 48 tensors that are not empty.
 */
mhlmoe_status mhlmoe_adamw(const mhlmoe_adamw_tensor *tensors, int n_tensors,
                           const mhlmoe_adamw_step *step, hipStream_t stream);

/*
 * Per-kernel timing (a measurement aid, off by default).  While enabled, each
 * kernel the library launches is bracketed by two HIP events recorded on the
 * caller's stream, so the measured interval is that kernel's execution on
 * the stream it actually runs on.  Kernel names: "route_fwd", "hist",
 * "count_scan", "scatter", "ffn", "combine", "bwd_dx", "bwd_combine",
 * "dw_plan", "bwd_dw", "router_dw", "route_bwd", "bias_update", "proj_in", "proj_out" and
 * "proj_bwd" (the projection GEMMs of the latent layer), "rmsnorm",
 * "rmsnorm_bwd", "rmsnorm_dw", "quantize" and "gemm_scaled"; "layernorm",
 * "layernorm_bwd", "layernorm_dw", "expert_counts", "balance_weights",
 * "balance_loss", "balance_sum", "balance_dx", "balance_dw", "balance_dx_dw" and
 * "adamw".
 *
 * mhlmoe_timing_enable(on)   start (on != 0) or stop recording; records
 *                            already taken are kept.
 * mhlmoe_timing_query(name, total_ms, launches)
 *                            waits for the recorded events of kernel `name`
 *                            and returns the sum of their durations (ms) and
 *                            how many launches were recorded.
 * mhlmoe_timing_reset()      waits for and drops every record.
 * Events are created on first use and reused; enabling timing is the only
 * way the library creates HIP objects.
 */
mhlmoe_status mhlmoe_timing_enable(int on);
mhlmoe_status mhlmoe_timing_query(const char *kernel, double *total_ms,
                                  int64_t *launches);
mhlmoe_status mhlmoe_timing_reset(void);

#ifdef __cplusplus
}
#endif

#endif /* MHLMOE_H */
