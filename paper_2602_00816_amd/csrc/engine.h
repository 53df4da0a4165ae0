// Host-side engine: parameter layout, workspace plan, the lockstep HVP and the
// Lanczos / SLQ drivers.
#pragma once
#include <mutex>
#include <string>
#include <vector>

#include "../../include/fdhvp.h"
#include "kernels.h"

namespace fdh {

struct ParamRef {
  int64_t off = -1;
  int64_t rows = 0, cols = 0;
  bool valid() const { return off >= 0; }
};

struct LayerRefs {
  ParamRef n1g, n1b, wqkv, bqkv, qng, kng, wo, bo, n2g, n2b, w1, b1, w2, b2;
};

struct Entry {
  std::string name;
  int64_t off, numel, rows, cols;
  int layer, kind;
};

struct BatchRef {  // one token batch of a bound dataset (device pointers, caller-owned)
  const int32_t* tok = nullptr;
  const int32_t* lab = nullptr;  // nullptr: next-token targets
  const int32_t* pos = nullptr;  // [axes][B][S] rotation positions; nullptr: 0 .. S - 1 on every axis
  int B = 0, S = 0;
};

struct Span {  // carve of the workspace
  size_t off = 0, bytes = 0;
};

// Optional per-launch timing with HIP events on the context stream (testing
// hook used by the benchmark).  Categories: 0 GEMM, 1 Lanczos vector kernels,
// 2 fused attention (forward launch, backward launches).
struct Timing {
  static constexpr int NCAT = 4;
  static constexpr size_t POOL = 8192;
  bool on = false;
  std::vector<hipEvent_t> ev;
  size_t used = 0;
  struct Rec { int cat, e0; double flops, bytes; };
  std::vector<Rec> recs;
  double ms[NCAT] = {}, flops[NCAT] = {}, bytes[NCAT] = {};
  double count[NCAT] = {};
  hipError_t begin(hipStream_t s, int* e0);
  hipError_t end(hipStream_t s, int cat, int e0, double fl, double by);
  hipError_t harvest(hipStream_t s);
  void reset() { for (int i = 0; i < NCAT; ++i) ms[i] = flops[i] = bytes[i] = count[i] = 0.0; }
  ~Timing();
};

int ritz_diagnostics(const double* alpha, const double* beta, int s, double tol, double* nodes, double* weights,
                     double* resid, int32_t* copies, int32_t* spurious, int32_t* ghosts);

// One carve of the workspace: the span of every buffer for a plan (largest
// token batch, Lanczos steps and options) and the attention path it serves.
// Engine::plan fills a WsLayout; the engine adopts it only once a workspace
// large enough for it has been handed over, so that size queries never move
// the buffers in use.
struct WsLayout {
  struct LayerSpans {
    // (qr: the q/k/v projection before a per-head norm)
    Span x_in_m, x_in_d, a_m, a_d, qr_m, qr_d, qkv_m, qkv_d, P_m, P_d, st, o_m, o_d, xmid_m, xmid_d, b_m, b_d, u_m, u_d, z_m, z_d;
  };
  std::vector<LayerSpans> ls;
  Span xL_m, xL_d, f_m, f_d, lo, sc_m, sc_d, log_m, log_d, dlog_m, dlog_d, rowloss, losses;
  Span dx0_m, dx0_d, dx1_m, dx1_d, dxo_m, dxo_d, dz_m, dz_d, dgu_m, dgu_d, db_m, db_d, gpart, do_m, do_d, dS_m, dS_d;
  Span dqkv_m, dqkv_d, dqkvo_m, dqkvo_d, gqa_m, gqa_d, dl, da_m, da_d, emb, rope, cdf, gpartial, bpart, bout;
  Span tcount;  // two int64 counters of fdh_bind_dataset
  Span nfflag;  // non-finite flags of the input direction and the product (two int32)
  Span tgt, head_ws;   // targets and scratch of the head in pieces
  Span wsplit;  // split-K partial products of the weight-gradient GEMMs
  Span lz_w, lz_q, lz_qp, lz_basis, lz_alpha, lz_beta, lz_coef, lz_gram, lz_partial, lz_flag, lz_maxabs;
  int64_t lz_ldq = 0;   // basis row stride (elements, multiple of 8)
  int lz_dev_rows = 0;  // basis rows held in the workspace
  // attention path: fused kernels (bf16; head dim 128 and S a multiple of
  // 8, or 64 and a multiple of 128) or score/probability matrices in the workspace
  bool fused = false;
  // activation recomputation: only each layer's input pair x_in is kept; the
  // other spans of every layer alias one shared set, which the backward refills
  // by running that layer's forward again (x_in -> z) just before its backward
  bool rc = false;
  int vp = 0;   // columns of the vocabulary per piece of the head (0: whole logits)
  int planB = 0, planS = 0, planM = 0;
  fdh_lanczos_opts planO{};
  size_t total = 0;     // bytes the carve needs
};

// The loss over the vocabulary in pieces (ends.hip): the carve of its scratch, and one call.
struct HeadCarve {
  int C = 0, C1 = 0, Tp = 0;   // columns of a piece, and in the first pass; rows of the logits' gradient (multiple of 8)
  bool keep = false;           // one piece, whose logits are formed once
  bool order = false;          // rows without a target after the others
  bool thin = false;           // both gradients in one pass over w
  bool fused = true;           // logits on head_gemm.hip, else on the GEMM (fp32 models, many rows)
  size_t rows, top, z, ym, f, lm, ld, part, gm, gd, xm, xd, dm, dd, runs, split, split_bytes, total;
};
struct HeadCall {
  const void *x_m = nullptr, *x_d = nullptr;   // [T][ldx], operand type
  int64_t ldx = 0;
  const void *w_m = nullptr, *w_d = nullptr;   // [V][d], operand type
  const int32_t* tgt = nullptr;                // [T]
  int T = 0;
  HeadCarve carve;                             // head_carve of T, the piece, grads and second
  float *loss_m = nullptr, *loss_d = nullptr;  // [T] or null
  double* rowloss = nullptr;                   // scale times the losses at the two points, [2][T], or null
  double scale = 1.0;
  bool grads = false;
  double scale_w = 1.0;                        // of dw: scale / eps
  void *dx_m = nullptr, *dx_d = nullptr;       // [T][lddx]
  int64_t lddx = 0;
  void* dw = nullptr;                          // [V][d]
  bool out_f32 = true, acc = false;            // outputs fp32 (acc: added to dw), else the operand type
  bool copy_x = true;                          // rows without a target may hold anything
  // Products of two half differences in the means, x_d w_d^T of the logits' and g_d w_d of dx's: the calls on
  // caller-owned memory form them always, the HVP leaves them out (of second order in the step, as in
  // every linear layer) where a kernel without them is there.
  bool second = true;
  char* scratch = nullptr;
};
double gemm_flops(const GemmArgs& g);   // executed by a product, causal tails clipped

class Engine : public WsLayout {
 public:
  // qk: per-head norm and position axes of a Llama model (already validated)
  Engine(const fdh_model_config& cfg, const fdh_qk_config& qk, hipStream_t stream);

  // configuration
  fdh_model_config cfg;
  bool qk_norm = false;
  int n_axes = 1;
  double embed_scale = 1.0;   // of the token rows (not of learned positions)
  QkRotary rot{};   // angles of the position rotation (Llama, head_dim <= QK_MAX_DH)
  hipStream_t stream;
  bool gpt2 = false, llama = false, quad = false, bf16 = false;
  int L = 0, d = 0, Hq = 0, Hk = 0, dh = 0, F = 0, V = 0, Smax = 0, qkvd = 0;
  int64_t P = 0;
  std::vector<Entry> entries;
  std::vector<LayerRefs> layers;
  ParamRef wte, wpe, head, nfg, nfb;
  std::string err;

  // workspace
  char* ws = nullptr;
  size_t ws_bytes = 0;
  bool force_unfused = false;   // testing: plan the unfused path even where the fused one applies
  bool force_unsplit = false;   // testing: weight-gradient GEMMs over the whole token range
  bool force_unpaired = false;  // testing: no weight-gradient GEMMs paired in one launch
  bool recompute = false;       // plan (and run) with activation recomputation
  // the carve for token batches up to [B, S] and m Lanczos steps with options
  // o (o may be null when m == 0), written into *out; changes nothing else
  size_t plan(int B, int S, int m, const fdh_lanczos_opts* o, WsLayout* out) const;
  // plan, check that bytes covers it, then adopt the carve and the buffer
  int set_workspace(void* dev, size_t bytes, int B, int S, int m, const fdh_lanczos_opts* o);
  // order-sensitive digest of the adopted carve (testing)
  uint64_t layout_digest() const;

  // operator binding for Lanczos / CG / the block-diagonal test: parameters,
  // step and the batches whose token-weighted average the operator is
  std::vector<BatchRef> b_data;
  const void* b_params = nullptr;
  double b_eps = 0.0;
  double b_inv_n = 0.0;   // scale of every kept cross-entropy row (1 / targets, or 1 for a sum)
  int64_t b_targets = 0;
  bool bound = false;
  const float* quad_diag = nullptr;
  Timing timing;

  // entry points (return fdh_status)
  int hvp(const void* params, const float* v, double eps, const int32_t* tok, int B, int S, float* hv);
  int hvp_batches(const void* params, const float* v, double eps, const BatchRef* bt, int nb, double inv_n, float* hv);
  int bind_batches(const void* params, const BatchRef* bt, int nb, double eps, int reduction, int64_t* targets);
  int hvp_bound(const float* v, float* hv);        // checked: waits, reports NaN/Inf and bad tokens
  int hvp_bound_async(const float* v, float* hv);  // enqueued only (Lanczos, CG, block test)
  int last_losses(double* lp, double* lm);
  int lanczos(int m, uint64_t seed, const fdh_lanczos_opts& o, double* alpha, double* beta, int* steps);
  int slq(int probes, int m, uint64_t seed, const fdh_lanczos_opts& o, double* nodes, double* weights, int* steps,
          double* trace);
  int init_params(void* params, uint64_t seed);
  int make_tokens(int32_t* tok, int B, int S, uint64_t seed, int dist);
  int random_vector(float* out, uint64_t seed, int kind);
  int block_stats(const float* a, const float* b, double* out);
  int block_diagonal(const float* v, double* out);
  int cg_solve(const float* b, double lam, int max_iters, double rel_tol, float* x, double* res, int* steps);
  int set_basis_offload(int device_rows, void* host, size_t bytes);
  // the q/k front of a layer on caller-owned pairs (fdh_qk_forward, fdh_qk_backward)
  int qk_check(const fdh_qk_gains* g, int B, int S, QkArgs* a);
  int qk_forward(const fdh_qk_gains* g, const int32_t* pos, int B, int S, const void* x_m, const void* x_d, int64_t ldx,
                 void* y_m, void* y_d, int64_t ldy);
  int qk_backward(const fdh_qk_gains* g, const int32_t* pos, int B, int S, const void* x_m, const void* x_d, int64_t ldx,
                  const float* dy_m, const float* dy_d, int64_t lddy, void* dx_m, void* dx_d, int64_t lddx, float* dgq,
                  float* dgk, bool acc, void* scratch, size_t scratch_bytes);
  // the embedding on caller-owned memory (fdh_embed_forward, fdh_embed_backward)
  int embed_check(const int32_t* tok, int B, int S);
  int embed_forward(const fdh_embed_tables* w, const int32_t* tok, int B, int S, float* x_m, float* x_d, int64_t ldx);
  int embed_backward(const int32_t* tok, int B, int S, const float* dx_d, int64_t lddx, double eps, float* hv_e, float* hv_p,
                     bool acc, void* scratch, size_t scratch_bytes);
  // the loss over the vocabulary in pieces (fdh_head_loss, fdh_head_grad; the HVP's head with
  // vocab_piece > 0)
  int vocab_piece = 0;   // plan (and run) the head in pieces of so many columns; 0: whole logits
  HeadCarve head_carve(int T_, int piece, bool grads, bool second = true) const;
  size_t head_scratch_most(size_t tokens, int piece) const;   // of an HVP's batches of up to so many tokens
  template <typename T> int head_run(const HeadCall& c);
  int head_check(const fdh_head_inputs* in, bool grads, size_t scratch_bytes, const void* scratch, HeadCall* c);
  int head_loss(const fdh_head_inputs* in, float* loss_m, float* loss_d, void* scratch, size_t scratch_bytes);
  int head_grad(const fdh_head_inputs* in, float* loss_m, float* loss_d, const fdh_head_grads* g, void* scratch, size_t scratch_bytes);
  std::vector<int64_t> layer_ranges() const;

 private:
  size_t linear_scratch(size_t tokens) const;
  mutable std::mutex linear_mu;      // linear_scratch(linear_tokens) = linear_bytes
  mutable int linear_tokens = -1;
  mutable size_t linear_bytes = 0;
  mutable int most_tokens = -1, most_piece = 0;   // (linear_mu) head_scratch_most of these = most_bytes
  mutable size_t most_bytes = 0;
  int check_batch(const int32_t* tok, int B, int S);
  int finish_checked(const float* hv);
  template <typename T>
  int hvp_t(const T* th, const float* v, double eps, const BatchRef& bt, double inv_n, bool acc, float* hv);
  template <typename B> int lanczos_t(int m, uint64_t seed, const fdh_lanczos_opts& o, double* alpha, double* beta, int* steps);
  template <typename T> void* wsp(const Span& s) const { return (void*)(ws + s.off); }

  // basis offload: at most off_rows rows in the workspace (-1: all), the rest
  // in caller-owned pinned host memory (device-side address)
  int off_rows = -1;
  void* host_rows_dev = nullptr;
  size_t host_rows_bytes = 0;
  // set by the Lanczos normalisation when it already wrote lo = eps * v for
  // the next HVP (of this v and eps); consumed by that HVP
  const float* lo_for_v = nullptr;
  double lo_for_eps = 0.0;
};

}  // namespace fdh
