// The two ends of a model on caller-owned memory: argument checks and dispatch of
// fdh_embed_* (include/fdhvp.h).
#include <algorithm>
#include <cmath>

#include "engine.h"
#include "regions.h"

namespace fdh {

#define CK(x)                                          \
  do {                                                 \
    hipError_t e_ = (x);                               \
    if (e_ != hipSuccess) {                            \
      err = std::string(#x) + ": " + hipGetErrorString(e_); \
      return FDH_ERR_HIP;                              \
    }                                                  \
  } while (0)

// ---------------------------------------------------------------------------
// token embedding
// ---------------------------------------------------------------------------
int Engine::embed_check(const int32_t* tok, int B, int S) {
  if (quad) { err = "needs a language-model context"; return FDH_ERR_UNSUPPORTED; }
  if (B < 0 || S < 0) { err = "B and S must not be negative"; return FDH_ERR_INVALID_ARG; }
  if ((int64_t)B * S > END_MAX_TOKENS) { err = "B*S must be <= 2^31 - 64"; return FDH_ERR_UNSUPPORTED; }
  if (gpt2 && S > Smax) { err = "S must be <= max_seq"; return FDH_ERR_INVALID_ARG; }
  if ((int64_t)B * S > 0 && (!tok || (uintptr_t)tok % 4)) { err = "tokens: null or not 4-byte aligned"; return FDH_ERR_INVALID_ARG; }
  return FDH_OK;
}

int Engine::embed_forward(const fdh_embed_tables* w, const int32_t* tok, int B, int S, float* x_m, float* x_d, int64_t ldx) {
  const int rc = embed_check(tok, B, S);
  if (rc != FDH_OK) return rc;
  if (!w || !w->e) { err = "null table"; return FDH_ERR_INVALID_ARG; }
  if (gpt2 ? !w->p : (w->p || w->v_p)) {
    err = "the GPT-2 family has learned positions and the Llama family none: p (and v_p) must be given or null";
    return FDH_ERR_INVALID_ARG;
  }
  if (!(w->eps > 0.0) || !std::isfinite(w->eps)) { err = "eps must be positive and finite"; return FDH_ERR_INVALID_ARG; }
  const int64_t T_ = (int64_t)B * S;
  if (T_ == 0) return FDH_OK;
  if ((uintptr_t)w->e % 16 || (uintptr_t)w->p % 16 || (uintptr_t)w->v_e % 4 || (uintptr_t)w->v_p % 4) {
    err = "tables must be 16-byte aligned, directions 4-byte aligned";
    return FDH_ERR_INVALID_ARG;
  }
  if (bad_rows(x_m, ldx, d, 4) || bad_rows(x_d, ldx, d, 4)) {
    err = "x: 16-byte aligned rows, at least d_model elements apart";
    return FDH_ERR_INVALID_ARG;
  }
  const int64_t ob = bf16 ? 2 : 4, te = (int64_t)V * d, tp = (int64_t)S * d;
  const Region o[2] = {{(const char*)x_m, T_, ldx * 4, (int64_t)d * 4}, {(const char*)x_d, T_, ldx * 4, (int64_t)d * 4}};
  const Region r[5] = {flat(w->e, te * ob), flat(w->v_e, te * 4), flat(w->p, tp * ob), flat(w->v_p, tp * 4), flat(tok, 4 * T_)};
  if (any_overlap(o, 2, r, 5)) { err = "x overlaps an input or itself"; return FDH_ERR_INVALID_ARG; }
  const EmbedTables t{w->e, w->v_e, w->p, w->v_p, w->eps, embed_scale};
  const PairF x{x_m, x_d};
  if (bf16) CK(launch_embed_fwd<bf16_t>(x, ldx, tok, T_, S, d, V, t, nullptr, stream));
  else CK(launch_embed_fwd<float>(x, ldx, tok, T_, S, d, V, t, nullptr, stream));
  return FDH_OK;
}

int Engine::embed_backward(const int32_t* tok, int B, int S, const float* dx_d, int64_t lddx, double eps, float* hv_e, float* hv_p,
                           bool acc, void* scratch, size_t scratch_bytes) {
  const int rc = embed_check(tok, B, S);
  if (rc != FDH_OK) return rc;
  if (!(eps > 0.0) || !std::isfinite(eps)) { err = "eps must be positive and finite"; return FDH_ERR_INVALID_ARG; }
  if (!hv_e || (uintptr_t)hv_e % 4) { err = "hv_e: null or not 4-byte aligned"; return FDH_ERR_INVALID_ARG; }
  if (gpt2 ? (!hv_p || (uintptr_t)hv_p % 4) : hv_p != nullptr) {
    err = "the GPT-2 family has learned positions and the Llama family none: hv_p must be given or null";
    return FDH_ERR_INVALID_ARG;
  }
  const int64_t T_ = (int64_t)B * S;
  const size_t need = embed_scratch_bytes(T_, d);
  if (need && (!scratch || scratch_bytes < need)) { err = "scratch smaller than fdh_embed_scratch_bytes"; return FDH_ERR_WORKSPACE; }
  if (need && (uintptr_t)scratch % 16) { err = "scratch must be 16-byte aligned"; return FDH_ERR_WORKSPACE; }
  if (T_ > 0 && bad_rows(dx_d, lddx, d, 4)) {
    err = "dx_d: 16-byte aligned rows, at least d_model elements apart";
    return FDH_ERR_INVALID_ARG;
  }
  const Region none = flat(nullptr, 0);
  const Region o[3] = {flat(hv_e, (int64_t)V * d * 4), flat(hv_p, (int64_t)Smax * d * 4), need ? flat(scratch, (int64_t)need) : none};
  const Region r[2] = {T_ > 0 ? Region{(const char*)dx_d, T_, lddx * 4, (int64_t)d * 4} : none, flat(tok, 4 * T_)};
  if (any_overlap(o, 3, r, 2)) { err = "an output or the scratch overlaps an input or another output"; return FDH_ERR_INVALID_ARG; }
  CK(launch_embed_bwd(hv_e, tok, dx_d, lddx, T_, d, V, embed_scale / eps, acc, scratch, stream));
  if (gpt2) CK(launch_pos_bwd(hv_p, dx_d, lddx, B, S, d, 1.0 / eps, Smax, acc, stream));
  return FDH_OK;
}

}  // namespace fdh
