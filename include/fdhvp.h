/*
 * fdhvp.h - finite-difference Hessian-vector products, Lanczos and stochastic
 * Lanczos quadrature for decoder-only language-model losses on AMD MI355X
 * (gfx950).  C ABI: plain pointers and sizes, no framework types.
 *
 * The operation (section 3.1, Eq. grad-fd-hvp; Algorithm 1): for parameters
 * theta, a direction v and a step eps,
 *     Hv ~= (grad L(theta + eps v) - grad L(theta - eps v)) / (2 eps),
 * where L is the mean next-token cross-entropy of the model over one token
 * batch.  Lanczos (section 4; Appendix C) drives it to build the tridiagonal
 * T_m = (alpha, beta); SLQ (section 4) turns T_m into Gauss quadrature nodes
 * (Ritz values) and weights.
 *
 * Conventions shared by every call
 *  - Ownership: the caller owns every buffer.  Device pointers: parameters,
 *    directions, outputs, tokens and the workspace.  Host pointers: alpha,
 *    beta, nodes, weights, statistics.  The library never allocates device
 *    memory; it carves all scratch from the workspace given to
 *    fdh_set_workspace.
 *  - Parameter vector: one flat array in the order reported by
 *    fdh_param_layout (per-layer blocks contiguous).  Element type float32
 *    (dtype FDH_F32) or bfloat16 bit patterns, uint16 (FDH_BF16).  Directions
 *    v and products Hv are always float32 of length fdh_num_params().
 *  - Tokens: int32 [B, S] row-major, values in [0, vocab); a token outside
 *    that range is an FDH_ERR_INVALID_ARG (never clamped into a wrong answer).
 *  - Streams: all device work is enqueued on the stream given to fdh_create,
 *    in call order.  fdh_hvp and fdh_hvp_bound wait for the stream at their
 *    end, to report non-finite values and bad tokens; so do the calls that
 *    return host results (lanczos, slq_density, block_stats, last_losses,
 *    the binds, cg_solve, block_diagonal).
 *  - Errors: every call returns an fdh_status; negative values are errors and
 *    leave outputs unspecified; fdh_last_error gives a message.  No call
 *    throws.  One context per host thread.
 *  - theta is never written: the perturbed points are formed on the fly.
 */
#ifndef FDHVP_H
#define FDHVP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define FDH_API_VERSION 1

typedef enum fdh_status {
  FDH_OK = 0,
  FDH_BREAKDOWN = 1,          /* warning: Lanczos stopped early, see steps_done */
  FDH_ERR_INVALID_ARG = -1,   /* null pointer, bad size/shape, eps <= 0 or not finite, m < 1 */
  FDH_ERR_WORKSPACE = -2,     /* no workspace, or smaller than fdh_workspace_bytes */
  FDH_ERR_HIP = -3,           /* a HIP runtime call failed */
  FDH_ERR_NONFINITE = -4,     /* NaN/Inf found in an input direction or in a product */
  FDH_ERR_STATE = -5,         /* call order (e.g. lanczos before bind) */
  FDH_ERR_UNSUPPORTED = -6    /* configuration outside what the kernels support */
} fdh_status;

typedef enum fdh_family {
  FDH_FAMILY_GPT2 = 0,        /* LayerNorm, learned positions, GELU(tanh) MLP, biases, tied head */
  FDH_FAMILY_LLAMA = 1,       /* RMSNorm, RoPE, SwiGLU MLP, GQA, no biases, untied head */
  FDH_FAMILY_QUAD_DIAG = 2    /* L(theta) = 1/2 sum_i d_i theta_i^2 (test operator, Hv = d*v) */
} fdh_family;

typedef enum fdh_dtype { FDH_F32 = 0, FDH_BF16 = 1 } fdh_dtype;
typedef enum fdh_reorth { FDH_REORTH_NONE = 0, FDH_REORTH_FULL = 1, FDH_REORTH_WINDOW = 2 } fdh_reorth;
typedef enum fdh_token_dist { FDH_TOKENS_UNIFORM = 0, FDH_TOKENS_ZIPF = 1 } fdh_token_dist;
typedef enum fdh_vec_kind { FDH_VEC_RADEMACHER = 0, FDH_VEC_GAUSSIAN = 1 } fdh_vec_kind;
typedef enum fdh_param_kind { FDH_PARAM_MATRIX = 0, FDH_PARAM_GAIN = 1, FDH_PARAM_BIAS = 2 } fdh_param_kind;

/* Model description.  For FDH_FAMILY_QUAD_DIAG only quad_n and dtype are read. */
typedef struct fdh_model_config {
  int32_t family;       /* fdh_family */
  int32_t n_layers;
  int32_t d_model;
  int32_t n_heads;
  int32_t n_kv_heads;   /* must divide n_heads */
  int32_t d_ff;
  int32_t vocab;
  int32_t max_seq;      /* learned-position rows (GPT-2) and upper bound on S */
  int32_t dtype;        /* fdh_dtype of the parameter vector and of the GEMM operands */
  float norm_eps;       /* LayerNorm / RMSNorm epsilon */
  float rope_base;      /* RoPE base (Llama family) */
  int32_t reserved;
  int64_t quad_n;       /* QUAD_DIAG dimension */
} fdh_model_config;

typedef struct fdh_lanczos_opts {
  int32_t reorth;       /* fdh_reorth */
  int32_t window;       /* WINDOW: number of most recent Lanczos vectors kept (>= 1) */
  int32_t basis_dtype;  /* fdh_dtype of the stored Krylov basis */
  float breakdown_tol;  /* stop when beta_{k+1} <= tol * max_j |alpha_j|; 0 selects 1e-5 */
} fdh_lanczos_opts;

/* Reduction of the per-target losses over a bound dataset. */
typedef enum fdh_reduction {
  FDH_REDUCE_MEAN = 0,        /* token-weighted mean over every kept target of every batch */
  FDH_REDUCE_SUM = 1          /* their sum (the solution-token objective of section 7) */
} fdh_reduction;

/* One batch of a dataset (Algorithm 1's dataloader): device pointers, caller-owned. */
typedef struct fdh_batch {
  const int32_t* tokens;  /* int32 [B, S] input tokens */
  const int32_t* labels;  /* int32 [B, S] aligned with the tokens: the logits at position t
                           * are scored against labels[t + 1]; -100 drops that target
                           * (padding, masked prompt).  NULL: the next token is the target. */
  int32_t B, S;
} fdh_batch;

typedef struct fdh_block {
  char name[48];        /* e.g. "h3.wqkv" */
  int64_t offset;       /* element offset in the flat vector */
  int64_t numel;
  int64_t rows, cols;   /* matrix shape (cols = 1 for vectors) */
  int32_t layer;        /* transformer layer, -1 for embeddings / final norm / head */
  int32_t kind;         /* fdh_param_kind */
} fdh_block;

/* Queries and keys of a Llama-family model between their projection and
 * attention.  norm: RMSNorm of every query and key head over its head_dim
 * elements (epsilon norm_eps) before the rotation, with one gain vector for the
 * queries and one for the keys of a layer; they are parameters of the layer
 * ("h0.qnorm.g", "h0.knorm.g", behind its wqkv).  n_axes: position axes of the
 * rotation (time, height, width, ...).  Pair i of a head (elements i and
 * i + head_dim/2) turns by rope_base^(-2i/head_dim) times the token's position
 * along the pair's axis; sections[a] pairs belong to axis a (their sum is
 * head_dim / 2), axis after axis or, interleaved, pairs a, a + n_axes, ... to
 * axis a >= 1 and the others to axis 0.  n_axes 0 is one axis (sections unread). */
#define FDH_MAX_AXES 4
typedef struct fdh_qk_config {
  int32_t norm;                     /* 0 or 1 */
  int32_t n_axes;                   /* 0 .. FDH_MAX_AXES */
  int32_t sections[FDH_MAX_AXES];
  int32_t interleaved;              /* 0 or 1 */
  int32_t reserved;                 /* 0 */
} fdh_qk_config;

/* The gains of one layer's query and key norm (device pointers). */
typedef struct fdh_qk_gains {
  const void *q, *k;        /* [head_dim] of the context's dtype */
  const float *v_q, *v_k;   /* [head_dim] directions; NULL: the same gain at both points */
  double eps;               /* the points are q + eps v_q and q - eps v_q; positive, finite */
} fdh_qk_gains;

/* The tables of the token embedding (device pointers). */
typedef struct fdh_embed_tables {
  const void* e;            /* [vocab][d_model] of the context's dtype */
  const float* v_e;         /* its direction; NULL: the same table at both points */
  const void* p;            /* GPT-2 family: [>= S][d_model] learned positions; Llama family: NULL */
  const float* v_p;         /* their direction or NULL */
  double eps;               /* the points are e + eps v_e and e - eps v_e; positive, finite */
} fdh_embed_tables;

/* Inputs of the loss over the vocabulary (device pointers): logits x w^T at the points
 * x_m +- x_d and w_m +- w_d, one target per row. */
typedef struct fdh_head_inputs {
  const void *x_m, *x_d;    /* [T] rows of d_model elements of the context's dtype, ldx elements apart */
  int64_t ldx;
  const void *w_m, *w_d;    /* [vocab][d_model] of the context's dtype (w_d: eps v in that dtype) */
  const int32_t* targets;   /* [T], -100: the row has none */
  int32_t T;                /* rows, 0 .. 2^20 */
  int32_t piece;            /* columns of the vocabulary handled at a time (rounded up to 256); 0: chosen */
  int32_t reserved;         /* 0 */
} fdh_head_inputs;

/* Gradients of the loss (device pointers). */
typedef struct fdh_head_grads {
  void *dx_m, *dx_d;        /* [T] rows of d_model elements, lddx apart: the gradient of x, a pair */
  int64_t lddx;
  void* dw;                 /* [vocab][d_model]: the half difference of the gradient of w over eps (Hv's entries) */
  double scale;             /* weight of every row's loss, e.g. 1 / targets; it and scale / eps finite in float32 */
  double eps;               /* positive, finite */
  int32_t dtype;            /* of dx and dw: FDH_F32 or the context's dtype */
  int32_t accumulate;       /* != 0: dw is added to what is there (FDH_F32) */
} fdh_head_grads;

typedef struct fdh_ctx fdh_ctx;

/* Create a context for one model on the current HIP device; hip_stream is a
 * hipStream_t (NULL = default stream).  *out receives the context. */
fdh_status fdh_create(const fdh_model_config* cfg, void* hip_stream, fdh_ctx** out);
/* fdh_create with a per-head norm of queries and keys and position axes (Llama
 * family, head_dim <= 256, n_heads <= 65536: FDH_ERR_UNSUPPORTED otherwise; FDH_ERR_INVALID_ARG
 * for sections that do not divide the pairs).  qk NULL or all zero is fdh_create. */
fdh_status fdh_create_qk(const fdh_model_config* cfg, const fdh_qk_config* qk, void* hip_stream, fdh_ctx** out);
void fdh_destroy(fdh_ctx* ctx);
int32_t fdh_api_version(void);

/* Number of parameters P (the length of theta, v and Hv). */
int64_t fdh_num_params(const fdh_ctx* ctx);

/* Parameter layout: up to cap entries into out; *n receives the total count. */
fdh_status fdh_param_layout(const fdh_ctx* ctx, fdh_block* out, int32_t cap, int32_t* n);

/* Workspace needed for token batches up to [B, S] and Lanczos runs up to m steps
 * with options o (o may be NULL and m 0 when only fdh_hvp is used). */
fdh_status fdh_workspace_bytes(const fdh_ctx* ctx, int32_t B, int32_t S, int32_t m,
                               const fdh_lanczos_opts* o, size_t* bytes);
/* Hand the library a device buffer of at least the queried size, 256-byte aligned.
 * The caller keeps ownership and must keep it alive while the context uses it.
 * On an error the workspace and carve already in use stay in force.  dev = NULL
 * with bytes = 0 detaches the workspace (the other arguments are ignored): the
 * context then holds no pointer into caller memory until the next call. */
fdh_status fdh_set_workspace(fdh_ctx* ctx, void* dev, size_t bytes, int32_t B, int32_t S,
                             int32_t m, const fdh_lanczos_opts* o);

/* Activation recomputation (gradient checkpointing, an option of the
 * fine-tuning runs of section 6): with on != 0 the workspace keeps, per
 * decoder layer, only the fp32 input pair of the layer (mean and
 * half-difference channels) plus one set of the layer's other activations
 * that all layers share.  Before each layer's backward the HVP runs that
 * layer's forward again from its stored input, up to the MLP activation, so
 * one HVP executes every decoder layer but the last one's forward twice (about
 * a quarter more GEMM work) and needs L - 1 fewer activation sets.  Results are the
 * same bits as without.  Takes effect for the following fdh_workspace_bytes /
 * fdh_set_workspace; the carve in use keeps its mode until then.  Off by
 * default; no effect for QUAD_DIAG. */
fdh_status fdh_set_recompute(fdh_ctx* ctx, int32_t on);

/* The head of the HVP in pieces of the vocabulary: with columns > 0 the logits are formed
 * `columns` (rounded up to 256) at a time by the kernels of fdh_head_grad and never kept, so the
 * workspace holds 4 bytes (bf16) or 8 (fp32) per token and column of one piece in place of 12 or
 * 16 per token and word of the vocabulary; the logits are formed twice (3 to 5 more products of the
 * head's size, where it has 8), unless one piece holds the vocabulary (bf16: 12 bytes then).  0 keeps
 * whole logits (the default).  Results agree to the rounding of the context's dtype: in bf16 the sums of
 * exponentials are fp32 (fp64 with whole logits), and the rows' weight is outside the rounding of the logits'
 * gradient.  As with whole logits, products of two half differences (of second order in the step) are left
 * out of the means, but for batches of up to 32 tokens and where the fp32 kernels have them.  The half differences of the
 * logits may reach 30 (bf16) or 300 (fp32): beyond, where whole logits hold longer steps, the product may be
 * FDH_ERR_NONFINITE.  Takes effect for the following fdh_workspace_bytes / fdh_set_workspace;
 * the carve in use keeps its mode until then. */
fdh_status fdh_set_vocab_piece(fdh_ctx* ctx, int32_t columns);

/* Synthetic inputs (the SplitMix64 counter generator of Steele, Lea and Flood,
 * OOPSLA 2014, in counter form): theta with N(0, 0.02) matrices, unit gains, zero biases (bf16 by
 * round-to-nearest-even); tokens uniform or Zipf(1.1); unit vectors. */
fdh_status fdh_init_params(fdh_ctx* ctx, void* params_dev, uint64_t seed);
fdh_status fdh_make_tokens(fdh_ctx* ctx, int32_t* tokens_dev, int32_t B, int32_t S,
                           uint64_t seed, int32_t dist);
fdh_status fdh_random_vector(fdh_ctx* ctx, float* out_dev, uint64_t seed, int32_t kind);

/* QUAD_DIAG only: the diagonal d (float32, length P, device, caller-owned). */
fdh_status fdh_set_quad_diag(fdh_ctx* ctx, const float* diag_dev);

/* Hv ~= (grad L(theta + eps v) - grad L(theta - eps v)) / (2 eps) on one batch
 * (section 3.1; Algorithm 1 with a single batch).  params: P elements of the
 * context dtype; v, hv: float32 [P]; tokens int32 [B, S] (ignored for QUAD_DIAG).
 * hv must not alias params or v.  Waits for the stream before returning.
 * Language-model families: FDH_ERR_NONFINITE when v holds a NaN or an
 * infinity, or when the product does (both scanned on the device, one extra
 * read of Hv); FDH_ERR_INVALID_ARG when a token lies outside [0, vocab).  On
 * either error hv is unspecified.  (QUAD_DIAG, a test operator, is not scanned.) */
fdh_status fdh_hvp(fdh_ctx* ctx, const void* params_dev, const float* v_dev, double eps,
                   const int32_t* tokens_dev, int32_t B, int32_t S, float* hv_dev);

/* Loss values L(theta + eps v), L(theta - eps v) of the most recent fdh_hvp. */
fdh_status fdh_last_losses(fdh_ctx* ctx, double* loss_plus, double* loss_minus);

/* Fix the operator used by fdh_hvp_bound / fdh_lanczos / fdh_slq_density /
 * fdh_cg_solve / fdh_block_diagonal: one batch of next-token targets (the same
 * as fdh_bind_dataset with one unlabelled batch and FDH_REDUCE_MEAN, whose
 * token scan and wait it shares).  The pointers are kept (not copied) and must
 * stay valid. */
fdh_status fdh_bind(fdh_ctx* ctx, const void* params_dev, const int32_t* tokens_dev,
                    int32_t B, int32_t S, double eps);

/* Fix a dataset operator for fdh_hvp_bound / fdh_lanczos / fdh_slq_density /
 * fdh_cg_solve / fdh_block_diagonal (Algorithm 1 with its dataloader loop,
 * section 3.1): the FD-HVP of the loss over all nbatch batches, each batch
 * weighted by its number of kept targets w_b, so that with FDH_REDUCE_MEAN
 * the result is the HVP of the token-weighted mean loss
 * sum_b w_b L_b / sum_b w_b (L_b the mean over batch b's targets), and with
 * FDH_REDUCE_SUM that of the summed loss.  Batches may differ in B and S,
 * each within the workspace plan (a plan with fused attention for S a multiple
 * of 128 takes no other lengths).  Padding is taken to sit after the real tokens (right
 * padding) with label -100: causal attention then keeps it out of every kept
 * target's context, so no attention mask is needed.  The batch array is
 * copied, the device pointers are kept (not copied) and must stay valid.
 * *n_targets (may be NULL) receives sum_b w_b.  Tokens and labels are scanned
 * on the device and the call waits for the stream; FDH_ERR_INVALID_ARG for a
 * token outside [0, vocab), a label outside [0, vocab) other than -100, or
 * when no target is left.
 * QUAD_DIAG contexts take nbatch = 0. */
fdh_status fdh_bind_dataset(fdh_ctx* ctx, const void* params_dev, const fdh_batch* batches, int32_t nbatch,
                            double eps, int32_t reduction, int64_t* n_targets);

/* fdh_bind_dataset with the rotation's positions (Llama family, head_dim <= 256).
 * positions: host array of nbatch device pointers, positions[i] int32
 * [axes, B, S] of batch i (axes = max(1, n_axes)), any int32 values, or NULL for
 * 0 .. S - 1 on every axis (text); a NULL array is fdh_bind_dataset.  The pointers
 * are kept, not copied.  The attention mask stays the causal one of the token
 * order. */
fdh_status fdh_bind_dataset_positions(fdh_ctx* ctx, const void* params_dev, const fdh_batch* batches,
                                      const int32_t* const* positions, int32_t nbatch, double eps, int32_t reduction,
                                      int64_t* n_targets);

/* The q/k front of a layer on caller-owned device memory, as the HVP runs it, for contexts of
 * the Llama family with head_dim <= 256 and n_heads <= 65536 (else FDH_ERR_UNSUPPORTED):
 * every tensor is a pair, _m the mean and _d the half difference of its values
 * at two points.  x: the q/k/v projection's output, B*S rows of
 * (n_heads + 2 n_kv_heads) head_dim elements of the context's dtype (query heads,
 * key heads, value heads), ldx elements apart; y: the same with query and key heads
 * normed (contexts with norm: gains required, otherwise NULL) and turned, value
 * heads copied.  y may be x (both pointers and the stride the same: the value heads
 * stay as they are); no other overlap.  positions_dev: int32 [axes, B, S] or NULL
 * (0 .. S - 1 in every row).  Pointers 16-byte aligned, strides in multiples of 16
 * bytes; positions and gains of any element alignment.  Any B*S from 0 (nothing is
 * done) to 2^31 - 64; needs no workspace.  Each output is rounded once from fp32
 * arithmetic with fp64 sums; a head that holds a NaN or an infinity is normed to NaN.
 * Only enqueued on the context stream (no wait, no allocation: may be captured in
 * a graph); a layer's call for one token is the call with B = S = 1. */
fdh_status fdh_qk_forward(fdh_ctx* ctx, const fdh_qk_gains* gains, const int32_t* positions_dev, int32_t B, int32_t S,
                          const void* x_m, const void* x_d, int64_t ldx, void* y_m, void* y_d, int64_t ldy);

/* Its backward: dx (context dtype, as x) from dy (float32, as y); the value heads are
 * rounded to the dtype.  With norm, x is the forward's input and dgq, dgk (float32
 * [head_dim]) receive, or with accumulate != 0 are added, the gains' entries of Hv:
 * the half difference of their gradients, summed over tokens and heads, over eps
 * (fp64 sums in a fixed order: the same bits in every call); without norm x may be
 * NULL and dgq, dgk are NULL.  scratch: device memory, 16-byte aligned, of at least
 * fdh_qk_scratch_bytes (0 without norm), in use until the call's work is done: calls
 * that may overlap on the device need scratch of their own.  No output overlaps an
 * input.  B*S = 0 sets dgq and dgk to zero (or leaves them).  Only enqueued, as
 * fdh_qk_forward. */
fdh_status fdh_qk_backward(fdh_ctx* ctx, const fdh_qk_gains* gains, const int32_t* positions_dev, int32_t B, int32_t S,
                           const void* x_m, const void* x_d, int64_t ldx, const float* dy_m, const float* dy_d,
                           int64_t lddy, void* dx_m, void* dx_d, int64_t lddx, float* dgq, float* dgk,
                           int32_t accumulate, void* scratch, size_t scratch_bytes);
fdh_status fdh_qk_scratch_bytes(const fdh_ctx* ctx, int32_t B, int32_t S, size_t* bytes);

/* Scale of the token embedding (1 after fdh_create): the model's first layer reads
 * scale * e[token] (+ p[position] for the GPT-2 family, whose positions and tied head
 * are not scaled).  Positive and finite.  Takes effect for every following call, the
 * products of a bound operator among them. */
fdh_status fdh_set_embed_scale(fdh_ctx* ctx, double scale);

/* The token embedding on caller-owned device memory, as the HVP runs it (language-model
 * families).  x: float32 pair (_m mean, _d half difference of the values at the two
 * points), B*S rows ldx elements apart, row t = scale e[token t] + p[t % S].  Tables and x
 * 16-byte aligned, ldx a multiple of 4; directions and tokens of any element alignment.
 * x overlaps neither an input nor itself.  A token outside [0, vocab) has no row: its
 * row of x is NaN.  Any B*S from 0 to 2^28; S <= max_seq for the GPT-2 family.
 * Outputs are rounded once.  Only enqueued on the context stream (no wait, no
 * allocation: may be captured in a graph); one token is the call with B = S = 1. */
fdh_status fdh_embed_forward(fdh_ctx* ctx, const fdh_embed_tables* tables, const int32_t* tokens_dev, int32_t B, int32_t S,
                             float* x_m, float* x_d, int64_t ldx);

/* Its backward: the tables' entries of Hv from dx_d, the half difference of the gradient of
 * x (float32, rows lddx apart, 16-byte aligned):
 *   hv_e[r] = scale / eps * sum of dx_d over the positions of token r   [vocab][d_model]
 *   hv_p[s] = 1 / eps * sum over the batch of dx_d at position s        [max_seq][d_model]
 * (hv_p: GPT-2 family, NULL otherwise), both whole, with zeros in the other rows, or with
 * accumulate != 0 added to what is there.  fp64 sums in an order that the tokens alone
 * set: the same bits in every call.  Positions of tokens outside [0, vocab) are left out.
 * scratch: device memory, 16-byte aligned, of at least fdh_embed_scratch_bytes, in use
 * until the call's work is done: calls that may overlap on the device need scratch of
 * their own.  No output overlaps an input.  eps positive, finite, and so 1 / eps and scale / eps.  Only
 * enqueued, as fdh_embed_forward. */
fdh_status fdh_embed_backward(fdh_ctx* ctx, const int32_t* tokens_dev, int32_t B, int32_t S, const float* dx_d, int64_t lddx,
                              double eps, float* hv_e, float* hv_p, int32_t accumulate, void* scratch, size_t scratch_bytes);
fdh_status fdh_embed_scratch_bytes(const fdh_ctx* ctx, int32_t B, int32_t S, size_t* bytes);

/* The softmax cross-entropy of x w^T against the rows' targets on caller-owned device
 * memory, a piece of the vocabulary at a time: the logits are formed piece by piece and
 * never kept (language-model families, d_model <= 2^16).
 *   loss[t] = log sum_j e^(l_tj) - l_ty as a float32 pair: _m the mean, _d the half difference of
 *   its values at the two points, not scaled; 0 for a row without a target.
 * fdh_head_grad also gives the gradients of scale * sum_t loss[t] (the loss pointers may be
 * NULL).  It forms the logits twice (once where one piece holds the vocabulary, which is chosen for
 * up to 2^26 logits, and for up to 8 rows) and rounds their gradient to the context's dtype, as the
 * HVP's products do (not for up to 8 rows; in bf16 about 2e-4 of a gradient's norm with 32000 words, which
 * float32 gradients hold too); sums and statistics are fp32 or wider, the order of the
 * additions is fixed (the same bits in every call).  Every product of the pairs is formed, x_d w_d^T in
 * the logits' mean and the logits' gradient's half difference times w_d in dx_m among them, for any T.
 * The half differences of the logits may reach 30 (bf16) or 300 (fp32) in magnitude; where a row's reach
 * so far beyond that a sum of exponentials may be cut, its loss and gradient, and dw, are NaN.
 * Rows without a target may hold anything (NaN among it): their dx is 0 and they take no
 * part in dw.  A target outside [0, vocab) other than -100, or a NaN in its row, makes the row's
 * loss and gradient, and with it dw, NaN.  Pointers 16-byte aligned (targets and losses
 * 4-byte), row strides in multiples of 16 bytes, ldx <= 2^20.  scratch: device memory, 256-byte
 * aligned, of at least fdh_head_scratch_bytes for the same T and piece, in use until the
 * call's work is done: calls that may overlap on the device need scratch of their own.  No
 * output overlaps an input, the scratch or another output.  T = 0 does nothing, but fdh_head_grad
 * sets dw to zero unless it accumulates.  Only enqueued on the context stream (no wait, no
 * allocation: may be captured in a graph); a single token is the call with T = 1. */
fdh_status fdh_head_loss(fdh_ctx* ctx, const fdh_head_inputs* in, float* loss_m, float* loss_d, void* scratch, size_t scratch_bytes);
fdh_status fdh_head_grad(fdh_ctx* ctx, const fdh_head_inputs* in, float* loss_m, float* loss_d, const fdh_head_grads* grads,
                         void* scratch, size_t scratch_bytes);
/* grads != 0: for fdh_head_grad (any dtype and eps); 0: for fdh_head_loss */
fdh_status fdh_head_scratch_bytes(const fdh_ctx* ctx, int32_t T, int32_t piece, int32_t grads, size_t* bytes);

/* hv = H v of the bound operator (fdh_bind or fdh_bind_dataset): one FD-HVP
 * per batch, accumulated into hv in batch order; fdh_last_losses then returns
 * the dataset losses at theta +- eps v.  v, hv: float32 [P] on device, not
 * aliasing each other or the parameters.  Waits for the stream and reports
 * non-finite values and bad tokens as fdh_hvp does. */
fdh_status fdh_hvp_bound(fdh_ctx* ctx, const float* v_dev, float* hv_dev);

/* Krylov-basis offload (section 7 notes that storing the whole Krylov
 * subspace bounds the scale and names offloading part of it to host memory):
 * keep at most device_rows stored Lanczos rows in the workspace and the
 * remaining ones in host_rows, caller-owned pinned host memory mapped for the
 * device (hipHostMalloc), of at least (stored rows - device_rows) * row bytes,
 * where stored rows = m (full) or min(m, window) and row bytes =
 * round_up(P, 8) * (2 for a bf16 basis, 4 for fp32).  Takes effect for the
 * following fdh_workspace_bytes / fdh_set_workspace (the workspace then holds
 * device_rows rows) and Lanczos runs; device_rows < 0 keeps every row on the
 * device (the default) and forgets host_rows.  The projection and update
 * passes read the host rows over the host link at every step, so each host
 * row adds about 2 * row bytes / link bandwidth to a step; results are the
 * same bits as with every row on the device.  FDH_ERR_INVALID_ARG when
 * host_rows is not mapped pinned memory or device_rows > 128; a Lanczos run
 * whose host part does not fit host_bytes fails with FDH_ERR_WORKSPACE. */
fdh_status fdh_set_basis_offload(fdh_ctx* ctx, int32_t device_rows, void* host_rows, size_t host_bytes);

/* m Lanczos steps (section 4) from the Rademacher probe z/sqrt(P) drawn from
 * probe_seed.  alpha_host[m], beta_host[m] receive alpha_1..alpha_s and
 * beta_2..beta_{s+1} (the last is the residual norm), s = *steps_done <= m;
 * entries past s are zero.  Returns FDH_BREAKDOWN when s < m. */
fdh_status fdh_lanczos(fdh_ctx* ctx, int32_t m, uint64_t probe_seed, const fdh_lanczos_opts* o,
                       double* alpha_host, double* beta_host, int32_t* steps_done);

/* SLQ (section 4): for probe j = 0..probes-1, Lanczos from seed + j, then the
 * eigen-decomposition of T_s: nodes_host[j*m + i] = lambda_i, weights_host[j*m+i]
 * = (U_1i)^2 (zero-padded past steps_done[j]); *trace_est = P * mean_j alpha_1. */
fdh_status fdh_slq_density(fdh_ctx* ctx, int32_t probes, int32_t m, uint64_t seed,
                           const fdh_lanczos_opts* o, double* nodes_host, double* weights_host,
                           int32_t* steps_done, double* trace_est);

/* Ritz-value diagnostics for runs that lose orthogonality (no or windowed
 * reorthogonalisation; Theorem 4.1's spurious duplicate "ghost" eigenvalues).
 * Host-only, no context.  alpha[s], beta[s] as returned by fdh_lanczos
 * (beta[s - 1] = beta_{s+1} is the residual norm), 1 <= s <= 128.  With
 * norm = max_i |theta_i| over the Ritz values theta_i of T_s (ascending):
 * nodes[i] = theta_i; weights[i] = (U_1i)^2; resid[i] = beta_{s+1} |U_si|,
 * the residual norm of the Ritz pair while the basis stays orthonormal;
 * copies[i] = size of its cluster (Ritz values chained by gaps <= tol * norm);
 * spurious[i] = 1 for a simple Ritz value that is also an eigenvalue of T_s
 * without its first row and column, within tol * norm (the test of Cullum and
 * Willoughby, 1985); *n_ghosts = sum over clusters of (size - 1).  Any output
 * pointer may be NULL.  FDH_ERR_INVALID_ARG for s outside [1, 128], a null
 * input or tol < 0. */
fdh_status fdh_ritz_diagnostics(const double* alpha, const double* beta, int32_t s, double tol, double* nodes,
                                double* weights, double* resid, int32_t* copies, int32_t* spurious,
                                int32_t* n_ghosts);

/* Per transformer layer b (section 6): out_host[3b..3b+2] = ||a_b||^2, ||b_b||^2,
 * <a_b, b_b> over the parameters of layer b; a, b float32 [P] on device. */
fdh_status fdh_block_stats(fdh_ctx* ctx, const float* a_dev, const float* b_dev, double* out_host);

/* fdh_block_stats for callers that cannot allocate device memory (code under
 * stream capture, tight serving loops, harnesses that forbid allocation): the
 * same statistics and the same kernels, with the partial sums in a fixed
 * 16 KiB device array that the library holds on every GPU it runs on until
 * the process ends, instead of the workspace.  Needs no workspace and calls
 * no device allocator.  At most 256 transformer layers (FDH_ERR_UNSUPPORTED
 * beyond, before any launch).  All calls on one GPU share that array: calls
 * that overlap on one GPU (other host threads or streams) race and must be
 * serialised by the caller.  Waits for the context stream. */
fdh_status fdh_block_stats_noalloc(fdh_ctx* ctx, const float* a_dev, const float* b_dev, double* out_host);

/* Block-diagonal hypothesis test (section 6, Exp I) on the bound operator:
 * h = H v, and for every transformer layer b, h_b = H v^(b) where v^(b) is v
 * with all entries outside layer b set to zero (not renormalised).  For each b,
 * stats_host[4b + 0] = ||h^(b) - h_b^(b)||, [4b + 1] = that over ||h^(b)||,
 * [4b + 2] = cosine of h^(b) and h_b^(b), [4b + 3] = ||h^(b)||, all restricted
 * to the parameters of layer b.  Runs L + 1 FD-HVPs; v: float32 [P] on device.
 * Needs a bound operator and a workspace planned with m >= 1 (its Lanczos vectors are
 * used as scratch).  Waits for the stream. */
fdh_status fdh_block_diagonal(fdh_ctx* ctx, const float* v_dev, double* stats_host);

/* Conjugate gradient for the damped inverse HVP on the bound operator: solves
 * (H + lambda I) x = b from x_0 = 0 (CG-based inverse-HVP solvers are the
 * second consumer the introduction and section 4 name; the method is that of
 * Hestenes and Stiefel).  b_dev, x_dev: float32 [P] on device, x overwritten,
 * not aliasing b.  Stops after max_iters steps or once ||r_k|| <= rel_tol ||b||;
 * res_host[max_iters + 1] receives ||r_0|| = ||b||, ||r_1||, ..., ||r_s||
 * (s = *steps_done, zeros after).  Returns FDH_BREAKDOWN, with x = x_s, when a
 * direction of non-positive curvature ((p, (H + lambda I) p) <= 0) stops it:
 * raise lambda.  Each step is one FD-HVP plus three vector passes; fp32
 * vectors, fp64 scalars with deterministic reductions; two scalars are read
 * back per step (the call waits for the stream).  Needs a bound operator and a
 * workspace planned with m >= 1 (its Lanczos vectors hold r, p and A p). */
fdh_status fdh_cg_solve(fdh_ctx* ctx, const float* b_dev, double lambda, int32_t max_iters, double rel_tol,
                        float* x_dev, double* res_host, int32_t* steps_done);

/* Number of transformer layers (blocks for fdh_block_stats). */
int32_t fdh_num_blocks(const fdh_ctx* ctx);

/* Message for the most recent error on this context (never NULL). */
const char* fdh_last_error(const fdh_ctx* ctx);

#ifdef __cplusplus
}
#endif
#endif /* FDHVP_H */
