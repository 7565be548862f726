/*
 * modse.h - C ABI of the MI355X (gfx950) library for one Mixture-of-Diverse-
 * Size-Experts (MoDSE) FFN layer, arXiv 2409.12210.
 *
 * The layer (Sec. 2 Eq. 1-3 and Sec. 3.1 of the paper):
 *     logits  H(x)_i = (x W_gate)_i (+ logit_bias_i)
 *     gate    G(x)   = Softmax(KeepTopK(H(x), top_k))         (Eq. 2, Eq. 3)
 *     output  y      = sum_i G_i(x) E_i(x)                     (Eq. 1; Sec. 3.1)
 *     expert  E_i(x) = W2_i ( silu(W1_i x) * (W3_i x) ),  W1_i,W3_i in R^{d_ff[i] x d},
 *                      W2_i in R^{d x d_ff[i]}                 (Llama-2 FFN, Sec. 4.1)
 * Each expert has its own hidden width d_ff[i] (Sec. 3.1).  Ties in top-k go to
 * the lower expert index; no token is ever dropped.
 *
 * Conventions for every call
 *  - "HOST" / "DEVICE" says where a pointer must point.  The library allocates
 *    and frees nothing: all buffers, workspace included, belong to the caller.
 *  - Calls only enqueue work on `hip_stream` (a hipStream_t passed as void*,
 *    NULL = the default stream).  They never synchronise and never read device
 *    memory from the host.
 *  - All argument checks run before the first enqueue and need no GPU.
 *    Errors are reported through the return code only.
 *  - T == 0 is valid and does nothing (pointers are then not examined).
 *  - NaN/Inf inputs: behaviour unspecified.
 *
 * Layouts (row-major everywhere, element type = desc.dtype unless said):
 *    x, y, dY, dX   [T, d_model]
 *    W_gate         [d_model, n_experts]
 *    W1, W3         one [F, d_model] matrix, F = sum d_ff; expert e owns rows
 *                   foff[e] .. foff[e+1]-1, foff[e] = sum_{e'<e} d_ff[e']
 *    W2             expert e starts at element d_model*foff[e] and is a
 *                   [d_model, d_ff[e]] matrix
 *    dW_gate, dW1, dW3, dW2   float32, same shapes as the weights
 */
#ifndef MODSE_H_
#define MODSE_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MODSE_OK = 0,
  MODSE_ERR_INVALID_ARG = 1, /* null pointer, negative size, bad d_ff, ... */
  MODSE_ERR_UNSUPPORTED = 2, /* top_k not in {1,2}, n_experts > 64, unknown dtype */
  MODSE_ERR_WORKSPACE = 3,   /* ws_bytes too small, see modse_workspace_size() */
  MODSE_ERR_HIP = 4          /* a HIP launch failed */
} modse_status;

typedef enum { MODSE_F32 = 0, MODSE_BF16 = 1 } modse_dtype;

/* Layer description.  Plain HOST struct, read during the call only. */
typedef struct {
  int32_t d_model;      /* multiple of 32 */
  int32_t n_experts;    /* N, 1..64 */
  int32_t top_k;        /* 1 or 2, <= N */
  const int32_t* d_ff;  /* HOST array [n_experts]; each > 0 and a multiple of 32;
                           any order, pairs are not assumed (Sec. 3.1 pair
                           constraint is the caller's business) */
  modse_dtype dtype;    /* element type of x, weights, y, dY, dX */
} modse_desc;

/* Routing artefacts, all DEVICE pointers, caller-allocated.  Permuted row r of
 * expert e lies in offsets[e] <= r < offsets[e+1]; inside an expert rows keep
 * ascending token order. */
typedef struct {
  int32_t* topk_idx;       /* [T, top_k] expert ids, slot 0 = largest logit */
  float* topk_w;           /* [T, top_k] gate weights (Eq. 2), sum to 1 per token */
  int32_t* counts;         /* [N] tokens*slots per expert */
  int32_t* offsets;        /* [N+1] exclusive prefix sum of counts */
  int32_t* row_of;         /* [T, top_k] (token, slot) -> permuted row */
  int32_t* src_of;         /* [T*top_k] permuted row -> token*top_k + slot */
  int32_t* near_tie_count; /* [1] tokens with a gap < 1e-6 between two neighbouring
                              logits among their top_k+1 largest */
} modse_routing;

/* Bytes of DEVICE workspace `ws` that serve a call for T tokens or fewer.
 * `which`: MODSE_WS_FWD for modse_route and for modse_layer_fwd without `saved`,
 * MODSE_WS_BWD for modse_layer_bwd, MODSE_WS_FWD_SAVED for modse_layer_fwd
 * with `saved` (the permuted rows, hidden activations and expert outputs then
 * live in `saved`, and the workspace holds routing scratch, tile plans and
 * float32 partial sums; a MODSE_WS_FWD workspace also serves that call).  Any
 * other value: MODSE_ERR_INVALID_ARG.
 * Results do not depend on ws_bytes as long as it is at least the size for the
 * call's T, so one workspace, sized for a program's largest batch, does for all.
 * A smaller one is refused, unless all that it lacks is room for the partial sums
 * of a product that small batches split: the product is then not split, which
 * is slower and adds in another order.  modse_route refuses only what does not
 * hold its scratch; a bfloat16 call of more than 16 experts that finds no room
 * behind it for W_gate's n_experts * d_model elements may take a slower router
 * that adds in another order, which can change the last bit of a gate weight. */
#define MODSE_WS_FWD 0
#define MODSE_WS_BWD 1
#define MODSE_WS_FWD_SAVED 2
modse_status modse_workspace_size(const modse_desc* desc, int64_t T, int which, size_t* bytes);

/* Bytes of the DEVICE buffer `saved` that carries activations from
 * modse_layer_fwd to modse_layer_bwd (the derivatives of the SwiGLU hidden
 * activation by its two pre-activations W1 x and W3 x, the hidden activations,
 * the expert outputs and the permuted token rows, all in permuted row order).
 * Its layout is private. */
modse_status modse_saved_size(const modse_desc* desc, int64_t T, size_t* bytes);

/* Router only: logits, top-k, gate weights (Eq. 2-3) and the stable permutation
 * by expert.  x [T,d] DEVICE, W_gate [d,N] DEVICE, logit_bias [N] float32
 * DEVICE or NULL.  Fills every field of *out. */
modse_status modse_route(const modse_desc* desc, int64_t T, const void* x, const void* W_gate,
                         const float* logit_bias, const modse_routing* out, void* ws, size_t ws_bytes,
                         void* hip_stream);

/* modse_route for callers that cannot allocate or pass a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * The router's scratch (per-block histograms, near-tie flags) is a device
 * array inside the library, MODSE_ROUTE_STATIC_SCRATCH_BYTES per GPU and 4 MiB
 * for W_gate's columns, held until the process ends; the call allocates and
 * frees nothing.  Same
 * arguments, results and checks as modse_route otherwise.  The need is about
 * T * (4 + (n_experts + 1) / 8) bytes, so the array serves 65536 tokens at
 * any expert count that is a power of two (other counts also keep a padded
 * copy of W_gate there, 2 * d_model * 64 elements at most); a call whose
 * scratch does not fit returns MODSE_ERR_WORKSPACE before anything is
 * launched.  All calls on one GPU share the array: calls that
 * overlap in time on one GPU (different streams) race. */
#define MODSE_ROUTE_STATIC_SCRATCH_BYTES (1u << 20)
modse_status modse_route_static(const modse_desc* desc, int64_t T, const void* x, const void* W_gate,
                                const float* logit_bias, const modse_routing* out, void* hip_stream);

/* Forward pass of the layer (Eq. 1 with diverse-size experts, Sec. 3.1):
 * route, permute, grouped up-projection with SwiGLU, grouped down-projection,
 * gate-weighted combine.  y [T,d] DEVICE out.  routing_out may be NULL unless
 * a backward pass follows; saved may be NULL unless a backward pass follows. */
modse_status modse_layer_fwd(const modse_desc* desc, int64_t T, const void* x, const void* W_gate,
                             const float* logit_bias, const void* W1, const void* W3, const void* W2, void* y,
                             const modse_routing* routing_out, void* saved, void* ws, size_t ws_bytes,
                             void* hip_stream);

/* Backward pass (chain rule through Eq. 1-3; logits outside the kept set get
 * zero gradient).  routing and saved are the ones modse_layer_fwd filled for
 * the same inputs.  dY [T,d] DEVICE in.  Outputs: dX [T,d] (desc.dtype),
 * dW_gate [d,N], dW1 [F,d], dW3 [F,d], dW2 (packed like W2), all float32.
 * accumulate = 0 overwrites the weight gradients, 1 adds to them (fp32
 * gradient accumulation); dX is always overwritten, and may lie in the buffer of
 * dY or of x (which then no longer holds the layer's input). */
modse_status modse_layer_bwd(const modse_desc* desc, int64_t T, const void* x, const void* W_gate, const void* W1,
                             const void* W3, const void* W2, const modse_routing* routing, const void* saved,
                             const void* dY, void* dX, float* dW_gate, float* dW1, float* dW3, float* dW2,
                             int accumulate, void* ws, size_t ws_bytes, void* hip_stream);

/* ---------------------------------------------------------------- optional parts of the gate
 * One struct switches on the two parts of the paper's gate that the plain
 * entry points leave out.  All pointers are DEVICE pointers owned by the
 * caller; the forward call fills the outputs, the backward call reads them.
 *
 * Noise term (second term of H(x) in Sec. 2, with Eq. 4 RMSNorm and Eq. 5
 * Softplus): H(x)_i += gamma * s_i / sqrt(mean_j s_j^2 + eps), s = Softplus(x
 * W_noise), the norm taken over the N per-expert values of one token.  It has
 * no random factor, so it is a function of x.  On when W_noise != NULL; then
 * gamma and noise_pre are required.
 *
 * Auxiliary load-balance loss (Sec. 3.2 Eq. 9-12): p(x) = softmax of H(x) over
 * all N experts, f_i = share of tokens whose largest probability is expert i
 * (ties to the lower index), P_i = mean of p_i, L_a = aux_alpha N sum_i f_i
 * P_i.  On when probs != NULL; then aux_f, aux_P and aux_loss are required. */
typedef struct {
  const void* W_noise; /* [d,N], desc.dtype, or NULL */
  const float* gamma;  /* [1] RMSNorm gain */
  float eps;           /* RMSNorm epsilon, >= 0 */
  float* noise_pre;    /* [T,N] x W_noise: written by forward, read by backward */
  float aux_alpha;     /* alpha of Eq. 9 */
  float* probs;        /* [T,N] p(x): written by forward, read by backward; or NULL */
  float* aux_f;        /* [N] f_i: written by forward, read by backward */
  float* aux_P;        /* [N] P_i */
  float* aux_loss;     /* [1] L_a */
} modse_gate_ext;

/* modse_route / modse_layer_fwd with the optional gate parts; ext == NULL is
 * the plain call.  Same workspace sizes.  An incomplete ext (a switched-on
 * part with a missing pointer, eps < 0) returns MODSE_ERR_INVALID_ARG. */
modse_status modse_route_ext(const modse_desc* desc, int64_t T, const void* x, const void* W_gate,
                             const float* logit_bias, const modse_gate_ext* ext, const modse_routing* out, void* ws,
                             size_t ws_bytes, void* hip_stream);
modse_status modse_layer_fwd_ext(const modse_desc* desc, int64_t T, const void* x, const void* W_gate,
                                 const float* logit_bias, const modse_gate_ext* ext, const void* W1, const void* W3,
                                 const void* W2, void* y, const modse_routing* routing_out, void* saved, void* ws,
                                 size_t ws_bytes, void* hip_stream);

/* Backward pass of loss = <dY, y> + aux_grad * L_a through the gate with its
 * optional parts: adds aux_grad * dL_a/dH (f_i held constant, as it is
 * piecewise constant) to the gradient of the logits, and, when the noise term
 * is on, also returns dW_noise [d,N] float32 and dgamma [1] float32 (both
 * follow `accumulate`) and adds the term's share to dX.  ext must hold the
 * buffers the forward call filled. */
modse_status modse_layer_bwd_ext(const modse_desc* desc, int64_t T, const void* x, const void* W_gate,
                                 const modse_gate_ext* ext, float aux_grad, const void* W1, const void* W3,
                                 const void* W2, const modse_routing* routing, const void* saved, const void* dY,
                                 void* dX, float* dW_gate, float* dW_noise, float* dgamma, float* dW1, float* dW3,
                                 float* dW2, int accumulate, void* ws, size_t ws_bytes, void* hip_stream);

/* Routing statistics in the shape of the paper's Appendix A tables, from
 * routing->topk_idx: slot_counts [top_k,N] int32 DEVICE out (tokens whose j-th
 * choice is expert i); summary [top_k+2] float32 DEVICE out: max/min of each
 * slot's counts, max/min of the per-expert totals, and the average hidden
 * width of the chosen experts (the workload measure of Sec. 4.3).  A ratio
 * whose minimum is 0 reads +inf. */
modse_status modse_routing_stats(const modse_desc* desc, int64_t T, const modse_routing* routing,
                                 int32_t* slot_counts, float* summary, void* hip_stream);

/* ---------------------------------------------------------------- the operators around the layer
 * The norm in front of a layer, the log probabilities that a model of such
 * layers is trained, scored and sampled by, and the orthogonalised update of its
 * expert matrices.  The conventions above hold; where infinities and NaN are
 * defined, it is said.  An output may lie in the buffer of an input only where
 * that is said.  Pointers need the alignment of their elements only, workspaces
 * 16 bytes (modse_orthogonalize: 256). */

/* h = x + residual, y = gamma h / sqrt(mean(h^2) + eps) over the rows of
 * [T, d_model] (d_model 1..16384, any value).  Sums and y are float32 and come
 * from the unrounded h.
 *   x, residual  [T, d_model] of `dtype`; residual may be NULL (h = x)
 *   gamma        [d_model] of `dtype`
 *   y, h         [T, d_model] of `dtype` out, either may be NULL; each may lie in the
 *                buffer of x or of residual
 *   rstd         [T] float32 out or NULL: 1 / sqrt(mean(h^2) + eps), for the backward pass
 *   q, scale     y in 8 bits (e4m3: 4 exponent bits, bias 7, largest 448, no infinity),
 *                [T, d_model], and float32 scales: y is about q * scale, scale = max|y| / 448
 *                (2^-126 at least) of a row (group 0: [T]) or of every `group` columns
 *                (group 32, 64 or 128: [T, ceil(d_model / group)]).  Both or neither. */
modse_status modse_norm_fwd(int64_t T, int32_t d_model, modse_dtype dtype, const void* x, const void* residual,
                            const void* gamma, float eps, void* y, void* h, float* rstd, void* q, float* scale,
                            int32_t group, void* hip_stream);

/* Bytes of workspace of modse_norm_bwd for T tokens or fewer. */
modse_status modse_norm_bwd_workspace_size(int64_t T, int32_t d_model, modse_dtype dtype, size_t* bytes);

/* Backward pass: h and rstd as modse_norm_fwd left them (h = x where there was no
 * residual), dY the gradient of y, dH the gradient that arrives along h itself (or
 * NULL).  dX [T, d_model] out = the gradient of h, which is that of x and of
 * residual; it may lie in the buffer of dY, dH or h.  dgamma [d_model] float32,
 * overwritten, or added to with accumulate = 1.  Sums run in an order that T and
 * d_model alone fix.  T == 0 leaves dgamma as it is. */
modse_status modse_norm_bwd(int64_t T, int32_t d_model, modse_dtype dtype, const void* h, const void* gamma,
                            const float* rstd, const void* dY, const void* dH, void* dX, float* dgamma, int accumulate,
                            void* ws, size_t ws_bytes, void* hip_stream);

/* Log probabilities of given tokens, entropy and the most probable entries of
 * softmax over rows of `vocab` logits.
 *   logits     T rows of `dtype`, row t at element t * ld_logits (ld_logits >= vocab)
 *   targets    [T] int32 or NULL.  Negative: no target, logp 0 and no gradient.  One
 *              that is not below vocab: logp (and the row's gradient) NaN
 *   logp       [T] float32 out, or NULL with targets: log softmax(logits)[target]
 *   stats      [T, 2] float32 out or NULL, for the backward pass
 *   entropy    [T] float32 out or NULL: -sum p log p
 *   top        0..64: top_idx [T, top] int32 and top_logp [T, top] float32 out, by falling
 *              logit, ties to the lower index
 * A logit of -inf is a masked entry: probability 0, never among the top (-1 and
 * -inf stand in the place of an entry that there is not), logp -inf where it is the
 * target.  A row of nothing else has no distribution: logp -inf, entropy 0 and no
 * gradient.  NaN or +inf in a row makes its logp and entropy NaN.  Which outputs
 * are asked for does not change the others, but few long rows are cut into
 * segments by T and by top (as one for top up to 8), and other cuts are other
 * roundings. */
#define MODSE_LOGPROBS_MAX_TOP 64
modse_status modse_logprobs_workspace_size(int64_t T, int32_t vocab, modse_dtype dtype, int32_t top, size_t* bytes);
modse_status modse_logprobs_fwd(int64_t T, int32_t vocab, modse_dtype dtype, const void* logits, int64_t ld_logits,
                                const int32_t* targets, float* logp, float* stats, float* entropy, int32_t top,
                                int32_t* top_idx, float* top_logp, void* ws, size_t ws_bytes, void* hip_stream);

/* Gradient of the logits of loss = sum_t d_logp[t] logp[t] + d_entropy[t]
 * entropy[t].  stats, entropy as modse_logprobs_fwd left them (entropy may be
 * NULL where d_entropy is).  targets and d_logp may be NULL together.  d_logits:
 * rows of `dtype` at ld_d_logits, vocab columns of each are written; it may lie in
 * the buffer of logits, with the same row distance. */
modse_status modse_logprobs_bwd(int64_t T, int32_t vocab, modse_dtype dtype, const void* logits, int64_t ld_logits,
                                const int32_t* targets, const float* stats, const float* entropy, const float* d_logp,
                                const float* d_entropy, void* d_logits, int64_t ld_d_logits, void* hip_stream);

/* A set of matrices, as the expert matrices of a layer are one.  Plain HOST
 * struct with HOST arrays, read during the call only. */
typedef struct {
  int32_t n_matrices;     /* 0..4096 */
  const int32_t* rows;    /* [n] each 1..65536 */
  const int32_t* cols;    /* [n] each 1..65536 */
  const float* const* G;  /* [n] DEVICE, row-major [rows, cols], float32 */
  void* const* U;         /* [n] DEVICE, row-major [rows, cols], of `dtype`; U[i] may be G[i] (float32) */
  modse_dtype dtype;
} modse_matrix_set;

/* U = X after `steps` (1..32) steps X <- a X + (b A + c A^2) X with A = X X^T, from
 * X = G / (|G| + eps), |G| the Frobenius norm.  coeffs: HOST array [steps][3] of
 * (a, b, c).  Products are those of values of 22 bits (pairs of float16) summed in
 * float32, and as near as float32 products where the steps keep singular values
 * within a few powers of two of the most that values up to 1 can come to.  Sets of
 * large products (sum of m m n from 6e8 on and 1.4 times that of m^3, m the shorter
 * side) take several steps together.  Float32 results are then within about three
 * times the error of float32 products.  Where U is bfloat16 more steps go together,
 * and results are off by up to about 1e-3 of |U| (1e-5 to 2e-4 as a rule) before they
 * are rounded, which is 1.7e-3 of |U|: ask for float32 results where that counts.
 * Coefficients that let a singular value of at most 1 grow beyond 2^40, or that are
 * not finite, are unsupported.  A matrix of zeros stays one; NaN or infinities in a
 * matrix make the whole of it NaN and leave the others alone. */
modse_status modse_orthogonalize_workspace_size(const modse_matrix_set* set, size_t* bytes);
modse_status modse_orthogonalize(const modse_matrix_set* set, const float* coeffs, int32_t steps, float eps, void* ws,
                                 size_t ws_bytes, void* hip_stream);

/* ---------------------------------------------------------------- both ends of a model
 * The embedding in front of the first layer, the dropout on the stream, and the
 * log probabilities behind the last layer, with their gradients. */

/* Lookup: x_t = scale E[token_t], rounded once.
 *   tokens  [T] int32.  Negative: no token, a row of zeros.  One that is not below
 *           vocab: a row of NaN
 *   E       [vocab, d_model] of `dtype` (vocab 1..2^20, d_model 1..16384, any value)
 *   x       [T, d_model] of `dtype` out */
modse_status modse_embed_fwd(int64_t T, int32_t d_model, int32_t vocab, modse_dtype dtype, const int32_t* tokens, const void* E,
                             float scale, void* x, void* hip_stream);

/* Its gradient: dE_v = scale sum of dX_t over the tokens t that are v, summed in
 * float32 in an order that the tokens alone fix.
 *   dX  [T, d_model] of `dtype`; rows of no token, or of one beyond vocab, are not read
 *   dE  [vocab, d_model] float32 out.  accumulate = 0: overwritten, rows that do not
 *       occur with zeros; 1: added to, and rows that do not occur stay untouched (tied
 *       matrices: with 1 behind modse_head_bwd, or before it with 1 there).
 * T == 0 leaves dE as it is.  T ceil(d_model / 256) up to 2^29. */
modse_status modse_embed_bwd_workspace_size(int64_t T, int32_t d_model, int32_t vocab, modse_dtype dtype, size_t* bytes);
modse_status modse_embed_bwd(int64_t T, int32_t d_model, int32_t vocab, modse_dtype dtype, const int32_t* tokens, const void* dX,
                             float scale, float* dE, int accumulate, void* ws, size_t ws_bytes, void* hip_stream);

/* Log probabilities from the last hidden rows: logits l = x W^T, of which a
 * workspace holds a piece at a time: it stops growing with T (at 3 to 10 GiB for gradients).
 *   x        [T, d_model] of `dtype` (d_model a multiple of 32 up to 16384; T up to 2^24)
 *   W        [vocab, d_model] of `dtype`, the output matrix (vocab 1..2^20)
 *   targets  [T] int32.  Negative: no target, logp 0 and no gradient, whatever stands in
 *            that row of x and d_logp.  One that is not below vocab: logp NaN, and so
 *            are its row of dX and all of dW
 *   logp     [T] float32 out: log softmax(l_t)[target_t]
 *   log_z    [T] float32 out: log sum_v e^l_tv.  modse_head_fwd: either may be NULL
 * x, W, dX, dW and the workspace lie at addresses that are multiples of 16.
 * Float32 with more rows than a few hundred (as many as make that the faster way), and
 * vocab d_model up to 2^28: x and W are held in 22 bits each, x down to 2^-39 of the
 * largest value of its row, W down to 2^-39 of its largest; what is smaller may be lost.
 * Where that would be more than some values near 0 (more than 1 of 256 values of W other
 * than 0 below 2^-20 of the largest, more than 1 of 16384 below 2^-30, or not all finite)
 * the products with W are in float32, which takes longer.  The workspace of such calls
 * also holds the parts of W, 4 vocab d_model bytes.
 * An infinity or NaN in a row of x makes that row's logp NaN (and its row of dX, and dW).
 * With infinities in W logits go by the products: one of -infinity has probability 0 (its
 * row of W then makes dX NaN), one of +infinity or NaN makes its row's logp NaN. */
modse_status modse_head_workspace_size(int64_t T, int32_t d_model, int32_t vocab, modse_dtype dtype, int which, size_t* bytes);
modse_status modse_head_fwd(int64_t T, int32_t d_model, int32_t vocab, modse_dtype dtype, const void* x, const void* W,
                            const int32_t* targets, float* logp, float* log_z, void* ws, size_t ws_bytes, void* hip_stream);

/* The log probabilities and, in the same call (it needs no modse_head_fwd before it),
 * the gradients of loss = sum_t d_logp[t] logp[t].
 *   d_logp  [T] float32
 *   logp    [T] float32 out or NULL
 *   dX      [T, d_model] of `dtype` out, or NULL; it may lie in the buffer of x
 *   dW      [vocab, d_model] float32 out, or NULL: overwritten, or added to with
 *           accumulate = 1
 * In bf16 the gradient of the logits is held in 16 bits for dX.  For dW, and in float32
 * where x and W are held in 22 bits, it is held in 22 bits, down to 2^-39 of the row's
 * largest, |d_logp_t| (1 - p_t) of its target's p_t; what is smaller may be lost.  In the
 * sums of dW a row counts down to 2^-39 of the largest |d_logp_t| (1 - p_t) max|x_t| of
 * all rows with a target.  No row of logp or dX depends on another row.
 * Workspace sizes: MODSE_WS_FWD and MODSE_WS_BWD for the two calls.  Sums run in an
 * order that the sizes alone fix, the two calls' in orders of their own.  T == 0
 * leaves dW as it is. */
modse_status modse_head_bwd(int64_t T, int32_t d_model, int32_t vocab, modse_dtype dtype, const void* x, const void* W,
                            const int32_t* targets, const float* d_logp, float* logp, void* dX, float* dW, int accumulate, void* ws,
                            size_t ws_bytes, void* hip_stream);

/* Dropout: y = residual + keep x / (1 - p), elementwise over [T, d_model].
 *   residual  of `dtype` or NULL (0)
 *   p         0..1, rounded to a multiple of 2^-16; at 1 everything is dropped
 *   rng       [2] uint64 DEVICE: seed and offset.  Read by the kernel, so that a captured
 *             graph makes another mask when they are changed between its replays
 *   call      tells several calls with one seed and offset apart (one per layer)
 *   y         of `dtype` out; may lie in the buffer of x or of residual
 * Random bits: Philox-4x32 with seven rounds, key = seed (low word first), counter =
 * (i / 8, call, offset low, offset high) for element i = t d_model + column; it gives 16
 * bits to each of eight elements, the low half of word w to that of i % 8 = 2 w.  Kept
 * where they are at least 65536 p.  What is dropped does not count, infinities and NaN
 * included.  T d_model below 2^35.
 * modse_dropout_bwd: dX = keep dY / (1 - p) with the same rng and call (the gradient of
 * residual is dY); dX may lie in the buffer of dY. */
modse_status modse_dropout_fwd(int64_t T, int32_t d_model, modse_dtype dtype, const void* x, const void* residual, double p,
                               const uint64_t* rng, uint32_t call, void* y, void* hip_stream);
modse_status modse_dropout_bwd(int64_t T, int32_t d_model, modse_dtype dtype, const void* dY, double p, const uint64_t* rng,
                               uint32_t call, void* dX, void* hip_stream);

/* Per-stage timing for benchmarks.  When enabled, modse_layer_fwd/bwd record
 * HIP events between their stages on the caller's stream; modse_stage_times
 * waits for the last recorded call and returns milliseconds per stage
 * (HOST array of MODSE_N_STAGES floats; stages not run read 0). */
enum {
  MODSE_STAGE_ROUTE = 0,    /* router GEMM + top-k + gate (+ auxiliary loss) */
  MODSE_STAGE_PERMUTE = 1,  /* histogram, scan over blocks (+ the tile plans of the forward GEMMs), stable row scatter */
  MODSE_STAGE_UP = 2,       /* grouped W1/W3 GEMM + SwiGLU */
  MODSE_STAGE_DOWN = 3,     /* grouped W2 GEMM */
  MODSE_STAGE_COMBINE = 4,  /* gate-weighted unpermute */
  MODSE_STAGE_BWD_PREP = 5, /* dO = g dY, d gate = <dY, O>, tile plans */
  MODSE_STAGE_BWD_DGRAD = 6,/* dH (+SwiGLU backward) and dX_permuted GEMMs */
  MODSE_STAGE_BWD_WGRAD = 7,/* dW1, dW3, dW2 GEMMs; layers of small tiles, where one
                               launch makes them and dX_permuted, count them as
                               BWD_DGRAD, and this stage reads 0 */
  MODSE_STAGE_BWD_ROUTER = 8,/* dX gather, d logits, dW_gate (whose shares may be
                                made beside dX_permuted) */
  MODSE_N_STAGES = 9
};
modse_status modse_stage_timing_enable(int on);
modse_status modse_stage_times(float* ms);

const char* modse_status_string(modse_status s);

#ifdef __cplusplus
}
#endif
#endif /* MODSE_H_ */
