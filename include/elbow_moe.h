/*
 * elbow_moe.h - C ABI of the elbow-routed MoE layer for AMD MI355X (gfx950).
 *
 * The layer (Section 2 of "Elbow-based MoE Routing: A Training-Free Inference Time Plugin
 * for Expert Selection"): for each token, router logits l = W_r x, probabilities
 * p = softmax(l), the probabilities sorted in descending order, a Kneedle-style elbow
 * index e on that sorted curve (Appendix A.1, Algorithm 1), the expert count
 * k = min(e + 1, K) capped at the model's top-K (Section 2.1), and the output
 * y = sum_{j<k} w_j FFN_{id_j}(x) over the selected experts, FFN being a bias-free SwiGLU
 * MLP.  Fixed top-K routing (the paper's baseline) runs through the same path.
 *
 * Conventions for every entry point:
 *  - All tensor pointers are DEVICE pointers owned by the caller; row-major, densely packed,
 *    starting at any element boundary (x and weights off a 16-byte boundary run slower kernels).
 *    The library never allocates, frees or synchronises device memory; scratch space
 *    comes only from the caller's workspace, which must be 256-byte aligned (as hipMalloc
 *    and torch allocations are).  Nothing is retained between calls.
 *  - `stream` is a hipStream_t passed as void* (NULL = the null stream).  Kernels are
 *    enqueued on it and the call returns without waiting for them.
 *  - Arguments are validated on the host BEFORE anything is enqueued.  On any error
 *    nothing is launched and nothing is written.  T = 0 is valid and enqueues nothing.
 *  - Return value: ELB_OK (0) or one of the ELB_ERR_* codes below; elb_last_error()
 *    gives a message for the last failing call of the calling thread.
 *  - Calls on the same stream are ordered; concurrent calls on different streams must not
 *    share output or workspace buffers.
 *  - Inputs must be finite, except that -inf logits are allowed when each row has at
 *    least one finite logit.  NaN inputs give unspecified (but in-bounds) results.
 *
 * Data types: ELB_F32 tensors are float; ELB_BF16 tensors are bfloat16 (uint16 storage,
 * round-to-nearest-even).  Router logits, routing weights and all accumulation are fp32.
 */
#ifndef ELBOW_MOE_H
#define ELBOW_MOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ELB_ABI_VERSION 1

/* Largest supported expert count N and cap K (any cap up to N: K = N is the uncapped
   elbow routing). */
#define ELB_MAX_EXPERTS 64
#define ELB_MAX_K 64

typedef enum {
    ELB_OK = 0,
    ELB_ERR_INVALID_ARG = 1, /* null pointer, negative size, K outside [1, N], eps < 0, ... */
    ELB_ERR_UNSUPPORTED = 2, /* a size outside what the kernels implement (e.g. N > 64) */
    ELB_ERR_WORKSPACE = 3,   /* workspace missing, not 256-byte aligned or smaller than
                                elb_*_workspace_bytes */
    ELB_ERR_HIP = 4          /* a HIP launch error (hipGetLastError after the launch) */
} elb_status;

typedef enum { ELB_F32 = 0, ELB_BF16 = 1 } elb_dtype;

typedef enum {
    ELB_MODE_ELBOW = 0, /* k = min(e + 1, K), Algorithm 1 with the cap of Section 2.1 */
    ELB_MODE_TOPK = 1   /* k = K: the fixed top-K routing the method prunes */
} elb_mode;

typedef struct {
    int32_t K;           /* cap: the model's top-K (8 for OLMoE); 1 <= K <= min(N, ELB_MAX_K) */
    float eps;           /* the normaliser's epsilon of Algorithm 1 (default 1e-8); >= 0 */
    int32_t mode;        /* elb_mode */
    int32_t renormalize; /* 0: w_j = p_(j) (full-softmax probability); 1: w_j = p_(j) /
                            sum_{i<k} p_(i) */
} elb_route_params;

/* ABI version (ELB_ABI_VERSION of the built library). */
int elb_abi_version(void);

/* Static description of a status code. */
const char *elb_status_str(int status);

/* Message of the last failing call on the calling thread ("" if none). */
const char *elb_last_error(void);

/*
 * Router logits (Section 2: a learned router produces logits l(x) in R^N per token).
 *   x        [T, d]  dtype            token activations
 *   W_router [N, d]  dtype            router weight (nn.Linear layout, no bias)
 *   logits   [T, N]  float (output)   l = x W_router^T, fp32 accumulation
 * Requirements: 2 <= N <= ELB_MAX_EXPERTS, d >= 1 (d % 32 == 0 for ELB_BF16).
 */
int elb_router_logits(const void *x, const void *W_router, int64_t T, int32_t d, int32_t N,
                      int32_t dtype, float *logits, void *stream);

/*
 * Routing (Section 2 and 2.1; Appendix A.1 Algorithm 1).  Per token:
 *   p = softmax(l); sort p descending (equal logits: lower expert id first);
 *   p'_i = (p_(0) - p_(i)) / (p_(0) - p_(N-1) + eps),  x'_i = i / (N - 1),
 *   D_i = p'_i - x'_i,  e = smallest index maximising D,  k = min(e + 1, K)
 *   (ELB_MODE_TOPK: k = K).
 * The normalised curve runs from (0,0) to (1,1), the orientation of the paper's elbow
 * angle (Section 2.3); D_i is the depth of sorted point i below the chord.
 *   logits [T, N] float   input
 *   k      [T]    int32   output, 1 <= k <= K
 *   ids    [T, K] int32   output, expert ids in descending-probability order; -1 for j >= k
 *   w      [T, K] float   output, weights (see elb_route_params.renormalize); 0 for j >= k
 * Requirements: 2 <= N <= ELB_MAX_EXPERTS; params valid.
 */
int elb_route(const float *logits, int64_t T, int32_t N, const elb_route_params *params,
              int32_t *k, int32_t *ids, float *w, void *stream);

/*
 * Router and routing fused (elb_router_logits followed by elb_route, in one kernel): each
 * block computes the logits of 16 tokens on the matrix cores, keeps them in LDS and routes
 * them there with the routing kernel's own per-token code, so k, ids and w are bit-identical
 * to the two-step path and the logits need not be written to memory.
 *   x, W_router          as elb_router_logits (ELB_BF16 only, d % 32 == 0)
 *   params               as elb_route, with K <= 16
 *   logits_out [T, N]    float output, or NULL to skip writing the logits
 *   k, ids, w            as elb_route
 * Other dtypes or caps: ELB_ERR_UNSUPPORTED (use the two calls).
 */
int elb_router_route(const void *x, const void *W_router, int64_t T, int32_t d, int32_t N,
                     int32_t dtype, const elb_route_params *params, float *logits_out,
                     int32_t *k, int32_t *ids, float *w, void *stream);

/*
 * Tail randomisation (Section 2.2): the elbow's k = min(e + 1, K) experts, as elb_route
 * selects them, followed by K - k further experts drawn uniformly without replacement from
 * the N - k experts outside that selection, so every token uses exactly K experts.  The draw
 * is the caller's: `rand[t, c]` is a uniform sample for expert c of token t, and the tail is
 * the K - k unselected experts with the smallest draws, in increasing draw order (equal
 * draws: lower expert id first).  With i.i.d. uniform draws this is a uniform draw without
 * replacement; the caller owns the random stream, so results are reproducible.
 *   logits  [T, N] float   input
 *   rand    [T, N] float   input, the draws (any finite values; only their order matters)
 *   k_elbow [T]    int32   output, the elbow's k (1 <= k <= K)
 *   ids     [T, K] int32   output, the elbow's experts in descending-probability order,
 *                          then the tail in increasing draw order; never -1
 *   w       [T, K] float   output, each expert's own full-softmax probability, or with
 *                          params->renormalize the probability over the K selected experts
 * Requirements as elb_route; params->mode = ELB_MODE_TOPK gives k = K and no tail.
 */
int elb_route_tail_random(const float *logits, const float *rand, int64_t T, int32_t N,
                          const elb_route_params *params, int32_t *k_elbow, int32_t *ids,
                          float *w, void *stream);

/*
 * Elbow angle (Section 2.3): the angle at the elbow point P_e = (x'_e, p'_e) of the
 * normalised sorted curve between the vectors to its ends (0,0) and (1,1),
 *   theta = arccos(v1 . v2 / (|v1| |v2|)),  v1 = -P_e,  v2 = (1,1) - P_e,
 * in degrees; small angles mark sharp elbows (confident routing), angles near 180 a curve
 * close to the chord.  e is the uncapped elbow index of elb_route (before min(e + 1, K));
 * when no point has D_i > 0, e = 0 and theta is taken as 180 (a straight curve).
 * Every elbow point lies in the unit square, inside the circle whose diameter is the chord
 * from (0,0) to (1,1), so 90 <= theta <= 180.
 *   logits [T, N] float   input
 *   e      [T]    int32   output, 0 <= e <= N - 1 (may be NULL)
 *   theta  [T]    float   output, degrees (may be NULL)
 * Requirements: 2 <= N <= ELB_MAX_EXPERTS; eps >= 0 and finite.
 */
int elb_elbow_angle(const float *logits, int64_t T, int32_t N, float eps, int32_t *e,
                    float *theta, void *stream);

/*
 * Variable-k dispatch: expert-major token lists built from a routing (deterministic:
 * within an expert, rows are in increasing token order).
 *   k, ids            [T], [T, K]   a routing as written by elb_route
 *   counts    [N]     int32 output  assignments per expert, sum = sum_t k_t
 *   offsets   [N + 1] int32 output  exclusive prefix sum of counts (offsets[N] = sum k)
 *   row_token [T * K] int32 output  row r of the expert-major order holds token
 *                                   row_token[r]; rows >= offsets[N] are left untouched
 *   inv       [T, K]  int32 output  row of (t, j) for j < k_t, -1 otherwise
 *   workspace          device scratch of at least elb_dispatch_workspace_bytes(T, N) bytes
 */
size_t elb_dispatch_workspace_bytes(int64_t T, int32_t N);
int elb_dispatch(const int32_t *k, const int32_t *ids, int64_t T, int32_t N, int32_t K,
                 int32_t *counts, int32_t *offsets, int32_t *row_token, int32_t *inv,
                 void *workspace, size_t workspace_bytes, void *stream);

/*
 * Expert part of the layer for a given routing: dispatch, the grouped SwiGLU expert
 * GEMMs and the weighted combine, in rank order with fp32 accumulation:
 *   y_t = [residual_t +] sum_{j<k_t} w_tj FFN_{ids_tj}(x_t),
 *   FFN_e(x) = W_down[e] (silu(W_gate[e] x) * (W_up[e] x)),  silu(z) = z / (1 + e^-z).
 *   x         [T, d]      dtype
 *   W_gate_up [N, 2m, d]  dtype   rows [0, m) = W_gate[e], rows [m, 2m) = W_up[e]
 *   W_down    [N, d, m]   dtype
 *   k, ids, w             a routing ([T], [T, K], [T, K]) as written by elb_route
 *   residual  [T, d]      dtype   optional (NULL: none)
 *   y         [T, d]      dtype   output; may alias residual, must not alias x
 *   workspace             at least elb_moe_workspace_bytes(T, d, N, m, K, dtype) bytes
 * Requirements: 2 <= N <= ELB_MAX_EXPERTS; 1 <= K <= min(N, ELB_MAX_K);
 * ELB_BF16: d % 64 == 0 and m % 64 == 0; ELB_F32: d % 16 == 0 and m % 16 == 0.
 */
size_t elb_moe_workspace_bytes(int64_t T, int32_t d, int32_t N, int32_t m, int32_t K,
                               int32_t dtype);
int elb_moe_experts(const void *x, const void *W_gate_up, const void *W_down,
                    const int32_t *k, const int32_t *ids, const float *w, const void *residual,
                    int64_t T, int32_t d, int32_t N, int32_t m, int32_t K, int32_t dtype,
                    void *y, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The whole layer: elb_router_logits and elb_route (fused as in elb_router_route for bf16 and
 * K <= 16: one launch up to 4096 tokens; above, two launches when N = 64 and d % 256 == 0, the
 * router's contraction in four quarters whose partial logits are summed in a fixed order
 * before the routing, else one; every form gives the same bits), then
 * elb_moe_experts, on one stream, with no host round trip.  Arguments as above; the optional debug outputs (NULL to
 * skip) receive the intermediate results of this call:
 *   logits_out [T, N] float, k_out [T], ids_out [T, K], w_out [T, K],
 *   counts_out [N] int32 (assignments per expert).
 * With T = 0 nothing is launched and no output (counts_out included) is written.
 */
int elb_moe_forward(const void *x, const void *W_router, const void *W_gate_up,
                    const void *W_down, const void *residual, int64_t T, int32_t d, int32_t N,
                    int32_t m, int32_t dtype, const elb_route_params *params, void *y,
                    void *workspace, size_t workspace_bytes, float *logits_out,
                    int32_t *k_out, int32_t *ids_out, float *w_out, int32_t *counts_out,
                    void *stream);

/*
 * The whole layer (elb_moe_forward) without a caller workspace and without any allocation,
 * for callers that cannot allocate device memory: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Scratch comes from a static device array of
 * ELB_NOALLOC_SCRATCH_BYTES per GPU (256 MiB, held by every GPU the library runs on until the
 * process ends; its address is looked up once per device, on the first call there, with the
 * stream's device current).  The caller still passes inputs and outputs, as for
 * elb_moe_forward, whose kernels and results (bit for bit) this call shares.
 * Limits and behaviour:
 *  - a problem whose elb_moe_workspace_bytes(T, d, N, m, K, dtype) exceeds
 *    ELB_NOALLOC_SCRATCH_BYTES is rejected with ELB_ERR_UNSUPPORTED before anything is
 *    enqueued (the OLMoE-shaped layer, d = 2048, N = 64, m = 1024, K = 8, fits up to 5307
 *    tokens);
 *  - nothing in the scratch has to start at zero, and nothing is cleared;
 *  - every call on one GPU uses that GPU's one array, so calls that overlap in time on one
 *    GPU (different streams, or different host threads) race and must be serialised by the
 *    caller; calls in order on one stream are safe;
 *  - with elb_profile_enable(1) the library creates timing events; leave profiling off where
 *    no allocation of any kind is allowed.
 */
#define ELB_NOALLOC_SCRATCH_BYTES ((size_t)256 << 20)
int elb_moe_forward_noalloc(const void *x, const void *W_router, const void *W_gate_up,
                            const void *W_down, const void *residual, int64_t T, int32_t d,
                            int32_t N, int32_t m, int32_t dtype, const elb_route_params *params,
                            void *y, float *logits_out, int32_t *k_out, int32_t *ids_out,
                            float *w_out, int32_t *counts_out, void *stream);

/*
 * Packed expert weights.  elb_pack_expert_weights writes a copy of W_gate_up and W_down in
 * MFMA operand order (per 64-row task, 64-deep stage, 32-deep half and 16-row fragment the 64
 * lanes' 16-byte pieces contiguous): the order an operand-streaming kernel loads in.  The
 * packed copy has the size of the two weight tensors together (elb_packed_expert_bytes) and
 * is bf16 only (d % 64 == 0, m % 64 == 0).
 *   W_gate_up [N, 2m, d], W_down [N, d, m]   bf16 input (as for elb_moe_experts)
 *   packed                                   device output, elb_packed_expert_bytes bytes
 * elb_moe_experts_packed / elb_moe_forward_packed are elb_moe_experts / elb_moe_forward with
 * that copy (or NULL) as an extra argument, kept for compatibility: the decode-sized kernels
 * stream the row-major weights at the rate they once needed the copy for, so every path reads
 * W_gate_up and W_down (both are required, as before) and the copy is not read.  Results are
 * bit-identical to the unpacked calls, and a program can save the copy's memory.
 */
size_t elb_packed_expert_bytes(int32_t N, int32_t d, int32_t m);
int elb_pack_expert_weights(const void *W_gate_up, const void *W_down, int32_t N, int32_t d,
                            int32_t m, int32_t dtype, void *packed, void *stream);
int elb_moe_experts_packed(const void *x, const void *W_gate_up, const void *W_down,
                           const void *packed, const int32_t *k, const int32_t *ids,
                           const float *w, const void *residual, int64_t T, int32_t d,
                           int32_t N, int32_t m, int32_t K, int32_t dtype, void *y,
                           void *workspace, size_t workspace_bytes, void *stream);
int elb_moe_forward_packed(const void *x, const void *W_router, const void *W_gate_up,
                           const void *W_down, const void *packed, const void *residual,
                           int64_t T, int32_t d, int32_t N, int32_t m, int32_t dtype,
                           const elb_route_params *params, void *y, void *workspace,
                           size_t workspace_bytes, float *logits_out, int32_t *k_out,
                           int32_t *ids_out, float *w_out, int32_t *counts_out, void *stream);

/*
 * The dense gated feed-forward block: the bias-free SwiGLU MLP of elb_moe_experts as a block that
 * every token goes through (a shared expert beside the routed ones, whose output is then the
 * residual here; or a dense layer of its own).
 *   y_t = [residual_t +] W_down h_t,  h_t = silu(W_gate x_t) * (W_up x_t)
 *   x         [T, d]   dtype
 *   W_gate_up [2m, d]  dtype   rows [0, m) = W_gate, rows [m, 2m) = W_up
 *   W_down    [d, m]   dtype
 *   residual  [T, d]   dtype   optional (NULL: none)
 *   y         [T, d]   dtype   output; may be residual, and may share memory with x (which is read
 *                              before y is written), with no other tensor of the call
 *   gate_up   [T, 2m]  float   optional output (NULL: not written): W_gate x_t and W_up x_t, for
 *                              elb_ffn_backward; shares memory with no other tensor
 *   workspace          at least elb_ffn_workspace_bytes(T, d, m, dtype) bytes
 * Sums are fp32; for ELB_BF16 h is rounded to bf16 before the second product and y at the end.
 * Requirements: d and m positive multiples of 16, at most 2^20; T < 2^31, T d and T m at most 2^38
 * (as for the entry points below).
 * An output that shares memory where it may not is refused with ELB_ERR_INVALID_ARG, here and below.
 * The workspace sizes of this and the entry points below never fall as T grows: a workspace for
 * a batch serves every smaller one too.
 */
size_t elb_ffn_workspace_bytes(int64_t T, int32_t d, int32_t m, int32_t dtype);
int elb_ffn_forward(const void *x, const void *W_gate_up, const void *W_down,
                    const void *residual, int64_t T, int32_t d, int32_t m, int32_t dtype, void *y,
                    float *gate_up, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Gradients of the block from dy, the gradient of y (that of residual is dy itself):
 *   dh = dy W_down,  s = 1 / (1 + e^-g),  dg = dh u s (1 + g (1 - s)),  du = dh g s,
 *   dx = dg W_gate + du W_up,  dW_gate = dg^T x,  dW_up = du^T x,  dW_down = dy^T h
 *   dy         [T, d]   dtype   gradient of y
 *   x, W_gate_up, W_down        as given to elb_ffn_forward
 *   gate_up    [T, 2m]  float   as written by elb_ffn_forward (g and u)
 *   dx         [T, d]   dtype   output, or NULL: not computed
 *   dW_gate_up [2m, d]  dtype   output, or NULL: not computed
 *   dW_down    [d, m]   dtype   output, or NULL: not computed
 *   workspace           at least elb_ffn_backward_workspace_bytes(T, d, m, dtype) bytes
 * Outputs are overwritten, not added to, and share memory with no other tensor of the call.  Sums are fp32 in a fixed
 * order (the same bits on every call); for ELB_BF16 dg, du and h are rounded to bf16 before the
 * products they enter.  With T = 0 the weight gradients are sums over no token: they are
 * written as zeros (the one case in which T = 0 enqueues work).  Requirements as elb_ffn_forward.
 */
size_t elb_ffn_backward_workspace_bytes(int64_t T, int32_t d, int32_t m, int32_t dtype);
int elb_ffn_backward(const void *dy, const void *x, const void *W_gate_up, const void *W_down,
                     const float *gate_up, int64_t T, int32_t d, int32_t m, int32_t dtype,
                     void *dx, void *dW_gate_up, void *dW_down, void *workspace,
                     size_t workspace_bytes, void *stream);

/*
 * Rows to 8-bit integers with one scale per row (symmetric):
 *   scale_t = fl32(max_i |x_ti| / 127),  q_ti = the whole number nearest to x_ti / scale_t (of the
 *   exact quotient; ties to even), at most 127 in magnitude; 0 where scale_t = 0
 *   A row that holds a NaN has scale NaN, one that holds an infinity (and no NaN) an infinite
 *   scale; the products of both are NaN.
 *   x     [T, d]  dtype
 *   q     [T, d]  int8 output
 *   scale [T]     float output: q_ti scale_t stands for x_ti; x, q and scale share no memory
 * Quantises tokens for elb_gemm_i8, and weights too (rows = output channels).
 * Requirements: d a positive multiple of 16, at most 2^20; T < 2^31.
 */
int elb_quantize_rows(const void *x, int64_t T, int32_t d, int32_t dtype, int8_t *q, float *scale,
                      void *stream);

/*
 * Product of 8-bit integers with a scale per token and per output channel:
 *   y_tn = [residual_tn +] (sum_i q_ti W_ni) scale_t W_scale_n
 *   q        [T, k]  int8, scale [T] float     tokens (elb_quantize_rows)
 *   W        [n, k]  int8, W_scale [n] float   weights
 *   residual [T, n]  dtype   optional (NULL: none)
 *   y        [T, n]  dtype   output; may be residual, shares memory with no other input
 * The sum is exact (int32); its scaling and the residual are fp32, rounded to dtype once.
 * Requirements: n and k positive multiples of 16, n at most 2^20, k at most 131071; T < 2^31.
 */
int elb_gemm_i8(const int8_t *q, const float *scale, const int8_t *W, const float *W_scale,
                const void *residual, int64_t T, int32_t n, int32_t k, int32_t dtype, void *y,
                void *stream);

/*
 * elb_quantize_rows and elb_gemm_i8 in one call, for activations x [T, k] of dtype.
 *   workspace  at least elb_linear_i8_workspace_bytes(T, n, k) bytes
 *   y may be residual and shares memory with no other input (x is read while y is written)
 */
size_t elb_linear_i8_workspace_bytes(int64_t T, int32_t n, int32_t k);
int elb_linear_i8(const void *x, const int8_t *W, const float *W_scale, const void *residual,
                  int64_t T, int32_t n, int32_t k, int32_t dtype, void *y, void *workspace,
                  size_t workspace_bytes, void *stream);

/*
 * The dense gated feed-forward block with 8-bit weights (and activations quantised on the way):
 * x is quantised by rows, g and u are its 8-bit products with W_gate_up, h = silu(g) u is kept in
 * fp32 and quantised by rows, and y = [residual +] the 8-bit product of that with W_down.
 *   x [T, d], residual [T, d] (or NULL), y [T, d]   dtype; y may be residual, and may share memory
 *                                                   with x, with no other input
 *   W_gate_up [2m, d] int8, gate_up_scale [2m] float; W_down [d, m] int8, down_scale [d] float
 *   workspace  at least elb_ffn_i8_workspace_bytes(T, d, m) bytes
 * Requirements: d and m positive multiples of 16, at most 131071; T < 2^31.
 */
size_t elb_ffn_i8_workspace_bytes(int64_t T, int32_t d, int32_t m);
int elb_ffn_forward_i8(const void *x, const int8_t *W_gate_up, const float *gate_up_scale,
                       const int8_t *W_down, const float *down_scale, const void *residual,
                       int64_t T, int32_t d, int32_t m, int32_t dtype, void *y, void *workspace,
                       size_t workspace_bytes, void *stream);

/*
 * Norms before and after a block, fused with its gate and the residual stream (an RMS norm has
 * no mean and no bias).  Per token:
 *   r_post = 1 / sqrt(mean(block^2) + eps),  p = w_post * block r_post     (w_post NULL: p = block)
 *   sum    = residual_scale residual + block_scale gate * p
 *   r_pre  = 1 / sqrt(mean(sum^2) + eps),    normed = w_pre * sum r_pre
 * `block` is a block's output, `sum` the residual stream after it and `normed` the next block's
 * input.  Without a block the call is a pre-norm alone, without w_pre the end of a block alone.
 *   residual [T, d] dtype   or NULL: none (then block is required)
 *   block    [T, d] dtype   or NULL: none (then gate and w_post have to be NULL too)
 *   gate            dtype   by gate_kind: NULL, [d], [T] or [T, d]
 *   w_post   [d]    dtype   or NULL: the block's output is not normalised
 *   w_pre    [d]    dtype   or NULL: normed is not computed
 *   eps                     finite, > 0
 * Sums are fp32; sum and normed are each rounded once (normed from the unrounded sum).
 * Requirements: d a positive multiple of 16, at most ELB_NORM_MAX_DIM; T < 2^31.
 */
#define ELB_NORM_MAX_DIM 16384
typedef enum {
    ELB_GATE_NONE = 0,
    ELB_GATE_CHANNEL = 1, /* [d], the same for every token */
    ELB_GATE_TOKEN = 2,   /* [T], the same for every channel */
    ELB_GATE_FULL = 3     /* [T, d] */
} elb_gate;

typedef struct {
    const void *residual, *block, *gate, *w_post, *w_pre;
    int64_t T;
    int32_t d;
    int32_t gate_kind; /* elb_gate */
    int32_t dtype;     /* elb_dtype */
    float residual_scale, block_scale, eps;
} elb_norm;

/*
 *   sum    [T, d] dtype  output, or NULL: not written; may be residual
 *   normed [T, d] dtype  output; NULL exactly where w_pre is
 *   r_post [T], r_pre [T] float  optional outputs (NULL: not written), for elb_norm_backward; r_post
 *                        is written only with w_post, r_pre only with w_pre.  Of a root mean square
 *                        above 2^126 they are subnormal numbers, with digits to 2^-149
 * Apart from sum and residual, outputs share memory with no other tensor.  A call with neither sum nor
 * normed asks for nothing: it enqueues nothing and writes no r_post either.
 */
int elb_norm_forward(const elb_norm *op, void *sum, void *normed, float *r_post, float *r_pre,
                     void *stream);

/*
 * Gradients of elb_norm_forward from those of sum (as what comes later uses it) and normed:
 *   s^ = sum r_pre,   S = d_sum + r_pre (w_pre * d_normed - s^ mean(s^ * w_pre * d_normed))
 *   b^ = block r_post, q = block_scale S, d_p = q * gate
 *   d_residual = residual_scale S,  d_block = r_post (w_post * d_p - b^ mean(b^ * w_post * d_p))
 *   d_gate = q * p, d_w_post = d_p * b^, d_w_pre = d_normed * s^, the last three summed over what
 *   the tensor is broadcast to
 *   op                 as given to elb_norm_forward (residual is not read)
 *   d_sum, d_normed    [T, d] dtype, either may be NULL (zero); d_normed needs w_pre, sum and r_pre
 *   sum                [T, d] dtype as written by elb_norm_forward (for a pre-norm alone with
 *                      residual_scale 1: the residual); read only with d_normed
 *   r_post, r_pre      as written by elb_norm_forward
 *   d_residual, d_block, d_gate, d_w_post, d_w_pre   outputs of dtype in the shapes of their tensors,
 *                      each NULL: not computed; d_block, d_gate and d_w_post need the block
 *   workspace          at least elb_norm_backward_workspace_bytes(T, d) bytes
 * Outputs are overwritten and share memory with no other tensor of the call.  Sums are fp32 in a
 * fixed order.  With T = 0 the gradients of w_post, w_pre and a gate per channel are written as zeros.
 */
size_t elb_norm_backward_workspace_bytes(int64_t T, int32_t d);
int elb_norm_backward(const elb_norm *op, const void *d_sum, const void *d_normed, const void *sum,
                      const float *r_post, const float *r_pre, void *d_residual, void *d_block,
                      void *d_gate, void *d_w_post, void *d_w_pre, void *workspace,
                      size_t workspace_bytes, void *stream);

/*
 * Rows to 4-bit values with a power-of-two scale for every 32 along the row (the layout of the 4-bit
 * weights below):
 *   a value is e2m1: code c in 0 .. 7 stands for 0, 0.5, 1, 1.5, 2, 3, 4, 6, c + 8 for its negative;
 *   the byte at column i / 2 holds value i (even) in its low half and value i + 1 in its high half
 *   a scale byte b stands for 2^(b - 127) (255: NaN)
 * b is the least from 2 to 252 for which the group's largest magnitude is at most 6 2^(b - 127)
 * (larger ones saturate), 255 for a group with an infinity or a NaN; values are rounded to the nearest
 * of the eight, ties to the even code.
 *   x     [rows, d]       dtype
 *   q     [rows, d / 2]   uint8 output
 *   scale [rows, d / 32]  uint8 output; x, q and scale share no memory
 * Requirements: d a positive multiple of 32, at most 2^20; rows < 2^31.
 */
int elb_quantize_f4(const void *x, int64_t rows, int32_t d, int32_t dtype, uint8_t *q,
                    uint8_t *scale, void *stream);

/*
 * A projection with 4-bit weights: y_tn = [residual_tn +] sum_i x_ti W_ni, W_ni the value of code
 * (n, i) times its group's scale.
 *   x        [T, k]       dtype
 *   W        [n, k / 2]   uint8, W_scale [n, k / 32] uint8   as elb_quantize_f4 lays them out, with any
 *                         scale byte: a zero is one at every scale but 255, which makes the row's products
 *                         NaN; values of 2^128 and more (bytes 253, 254) make them infinite or NaN
 *   residual [T, n]       dtype   optional (NULL: none)
 *   y        [T, n]       dtype   output; may be residual, shares memory with no other input
 *   workspace             at least elb_linear_f4_workspace_bytes(T, n, k, dtype) bytes (may be 0)
 * Products are exact (of an fp32 x below 2^-100 in magnitude: x is taken to within 2^-124), sums fp32, y
 * is rounded once.  An infinity in x gives an infinity or a NaN.
 * Requirements: n a positive multiple of 16, k of 32, both at most 2^20; T < 2^31.
 */
size_t elb_linear_f4_workspace_bytes(int64_t T, int32_t n, int32_t k, int32_t dtype);
int elb_linear_f4(const void *x, const uint8_t *W, const uint8_t *W_scale, const void *residual,
                  int64_t T, int32_t n, int32_t k, int32_t dtype, void *y, void *workspace,
                  size_t workspace_bytes, void *stream);

/*
 * The dense gated feed-forward block (elb_ffn_forward) with 4-bit weights.
 *   x [T, d], residual [T, d] (or NULL), y [T, d]   dtype; y may be residual, and may share memory
 *                                                   with x, with no other input
 *   W_gate_up [2m, d / 2], gate_up_scale [2m, d / 32], W_down [d, m / 2], down_scale [d, m / 32]
 *                                                   uint8, as for elb_linear_f4
 *   workspace  at least elb_ffn_f4_workspace_bytes(T, d, m, dtype) bytes
 * For ELB_BF16 h is rounded to bf16 before the second product, as in elb_ffn_forward.
 * Requirements: d and m positive multiples of 32, at most 2^20; T < 2^31.
 */
size_t elb_ffn_f4_workspace_bytes(int64_t T, int32_t d, int32_t m, int32_t dtype);
int elb_ffn_forward_f4(const void *x, const uint8_t *W_gate_up, const uint8_t *gate_up_scale,
                       const uint8_t *W_down, const uint8_t *down_scale, const void *residual,
                       int64_t T, int32_t d, int32_t m, int32_t dtype, void *y, void *workspace,
                       size_t workspace_bytes, void *stream);

/*
 * The whole layer for at most ELB_FEW_TOKENS tokens in two launches, with experts in bf16 or in 4
 * bits: routing as elb_moe_forward (the same bits of k, ids and w), then
 *   y_t = [residual_t +] sum_{j<k_t} W_down[ids_tj] h_tj,
 *   h_tj = w_tj silu(W_gate[ids_tj] x_t) * (W_up[ids_tj] x_t)
 * with fp32 sums; h is rounded to bf16, y once at the end.
 *   x [T, d], W_router [N, d], residual [T, d] (or NULL)   bf16
 *   y [T, d]             bf16 output; may be residual or x, shares memory with no other tensor
 *   gate_up_scale, down_scale   both NULL: W_gate_up [N, 2m, d] and W_down [N, d, m] are bf16;
 *                        otherwise uint8 [N, 2m, d / 32] and [N, d, m / 32], and the weights uint8
 *                        [N, 2m, d / 2] and [N, d, m / 2], as for elb_linear_f4
 *   workspace            at least elb_moe_few_workspace_bytes(T, d, N, m, K) bytes
 *   k_out [T], ids_out [T, K], w_out [T, K]   optional outputs (NULL: not written), as elb_route
 * Requirements: T <= ELB_FEW_TOKENS (more: ELB_ERR_UNSUPPORTED), d and m positive multiples of 64, at
 * most 2^20; 2 <= N <= ELB_MAX_EXPERTS, K <= 16 (a larger cap: ELB_ERR_UNSUPPORTED).
 */
#define ELB_FEW_TOKENS 16
size_t elb_moe_few_workspace_bytes(int64_t T, int32_t d, int32_t N, int32_t m, int32_t K);
int elb_moe_forward_few(const void *x, const void *W_router, const void *W_gate_up,
                        const uint8_t *gate_up_scale, const void *W_down, const uint8_t *down_scale,
                        const void *residual, int64_t T, int32_t d, int32_t N, int32_t m,
                        const elb_route_params *params, void *y, void *workspace,
                        size_t workspace_bytes, int32_t *k_out, int32_t *ids_out, float *w_out,
                        void *stream);

/*
 * Calibration of the matrix-core roofline (a measurement aid, not part of the layer): a
 * kernel of `blocks` blocks of 4 waves, each wave issuing iters x 8 back-to-back
 * v_mfma_f32_32x32x16_bf16 instructions (32 x 32 x 16 multiply-adds each) on register
 * operands, with no memory traffic.  Timing it gives the bf16 MFMA rate the chip sustains,
 * clock and power included.
 *   out [blocks * 4] float   device output (one sum per wave, so the work is kept)
 * Returns the number of MFMA instructions enqueued (> 0), or a negative elb_status.
 */
int64_t elb_calibrate_mfma_bf16(int32_t blocks, int32_t iters, float *out, void *stream);

/*
 * Calibration of the HBM read roofline (a measurement aid, not part of the layer): `blocks`
 * blocks of 4 waves read the whole of buf once, each block its own contiguous share, with
 * coalesced non-temporal 16-byte loads (sixteen in flight per lane), and fold the words into
 * one per wave.
 * Timing it over a buffer larger than the last-level cache gives the read rate the chip
 * sustains.
 *   buf   [bytes] device memory, 16-byte aligned; bytes a positive multiple of 16 (read only)
 *   out   [blocks * 4] uint32 device output (one word per wave, so the reads are kept)
 * Returns ELB_OK or an elb_status; nothing is allocated.
 */
int elb_calibrate_read_stream(const void *buf, int64_t bytes, int32_t blocks, uint32_t *out,
                              void *stream);

/*
 * Per-kernel timing (hipEvents attached to each launch the library makes).
 * elb_profile_enable(1) starts recording on the calling process for every launch,
 * elb_profile_enable(2) for the grouped expert GEMMs only, elb_profile_enable(0) stops; a
 * recorded launch carries a start/stop event pair in its own dispatch
 * (hipExtLaunchKernelGGL).  Timed launches run measurably slower than untimed back-to-back
 * ones (on MI355X the large expert GEMMs by about 10 %), so per-kernel figures from this
 * are upper bounds.  elb_profile_read() synchronises on the
 * recorded events, fills up to `cap` entries of names (static strings), total
 * milliseconds and launch counts per kernel, clears the records and returns the number
 * of kernels (or a negative elb_status).  Not for use under graph capture.
 */
int elb_profile_enable(int on);
int elb_profile_read(const char **names, double *total_ms, int64_t *launches, int cap);

#ifdef __cplusplus
}
#endif

#endif /* ELBOW_MOE_H */
