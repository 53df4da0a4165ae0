// The two ends of a model on caller-owned memory: argument checks and dispatch of
// fdh_embed_* and fdh_head_* (include/fdhvp.h), and the loop over the vocabulary's pieces.
#include <algorithm>
#include <cmath>
#include <type_traits>

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
  if ((int64_t)B * S > END_MAX_TOKENS) { err = "B*S must be <= 2^28"; return FDH_ERR_UNSUPPORTED; }
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
  if (!(eps > 0.0) || !std::isfinite(eps) || !std::isfinite(1.0 / eps) || !std::isfinite(embed_scale / eps)) {
    err = "eps must be positive and finite, and so 1 / eps and the embedding's scale / eps";
    return FDH_ERR_INVALID_ARG;
  }
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
  CK(launch_embed_bwd(EmbedGrad{hv_e, hv_p, embed_scale / eps, 1.0 / eps, Smax, acc, acc}, tok, dx_d, lddx, B, S, d, V, scratch, stream));
  return FDH_OK;
}

// ---------------------------------------------------------------------------
// loss over the vocabulary in pieces
// ---------------------------------------------------------------------------
namespace {

// elements of one channel of a piece's logits that are aimed at
constexpr int64_t HEAD_PIECE_ELEMS = (int64_t)64 << 20;
// bytes of statistics of column groups that are aimed at where no gradient takes more
constexpr size_t HEAD_PART = (size_t)64 << 20;
constexpr int HEAD_PIECE_ROUND = 256, HEAD_PIECE_MIN = 1024;
// most elements of a launch's logits (2^20 of the largest tiles, 2^29 threads)
constexpr int64_t HEAD_LAUNCH_ELEMS = (int64_t)1 << 35;
// Operations of the logits from which on the rows without a target are put behind the others (a launch
// of 5 us, of some 150 here), so that only the others are multiplied: 2500 x 32000 x 1024, of which 30%
// have none: 520 -> 385 us, with none 517 -> 523; gradients of 8192 x 32000 x 2048 with half of them
// 10.85 -> 7.97 ms, with none 11.37 -> 11.38.
constexpr double HEAD_ORDER_OPS = 1.5e11;
// rows up to which the target's logits are formed in fp64
constexpr int HEAD_FINE_ROWS = 32;
// scratch that the plan of a split contraction may take
constexpr size_t HEAD_SPLIT = (size_t)512 << 20;

GemmOperand kmaj(const void* p, int64_t ld) {
  GemmOperand o;
  o.ptr = p;
  o.s_row = ld;
  o.s_k = 1;
  return o;
}
GemmOperand mnmaj(const void* p, int64_t ld) {
  GemmOperand o;
  o.ptr = p;
  o.s_row = 1;
  o.s_k = ld;
  return o;
}

// products of the mean's logits on the GEMM (few rows: x_d w_d in the HVP too, as the tiles of 32 rows have it)
int logit_pairs(int T_, bool second) { return second || T_ <= HEAD_FINE_ROWS ? 2 : 1; }

// scratch of the products of a piece of C columns: those that its gradient goes to and, unless fused, its logits'
template <typename T>
size_t piece_split(int T_, int Tp, int C, int d, bool grads, bool fused, bool second) {
  GemmArgs g[2];
  auto need = [&](int M, int N, int K, int n, int mean_pairs) {
    for (int p = 0; p < 2; ++p) {
      g[p].M = M;
      g[p].N = N;
      g[p].K = K;
      g[p].ldc = N;
      g[p].npairs = p ? mean_pairs : 2;
    }
    return gemm_scratch<T>(g, n, HEAD_SPLIT);
  };
  size_t mx = fused ? 0 : need(T_, C, d, 2, logit_pairs(T_, second));
  if (grads) mx = std::max(mx, std::max(need(T_, d, C, 2, second ? 2 : 1), need(C, d, Tp, 1, 1)));
  return mx;
}

}  // namespace

HeadCarve Engine::head_carve(int T_, int piece, bool grads, bool second) const {
  HeadCarve c;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  };
  const size_t ob = bf16 ? 2 : 4, t = (size_t)T_;
  c.Tp = (int)((t + 7) / 8 * 8);
  if (piece > 0) piece = (int)std::min<int64_t>(piece, HEAD_LAUNCH_ELEMS / std::max(1, T_));
  c.thin = grads && T_ <= HEAD_THIN;   // (no more logits than w has rows 8 wide)
  const bool whole = c.thin || (piece > 0 ? piece >= V : (int64_t)T_ * V <= HEAD_PIECE_ELEMS);
  int64_t C = piece > 0 ? piece : std::max<int64_t>(HEAD_PIECE_MIN, HEAD_PIECE_ELEMS / std::max(1, T_) / HEAD_PIECE_ROUND * HEAD_PIECE_ROUND);
  C = (C + HEAD_PIECE_ROUND - 1) / HEAD_PIECE_ROUND * HEAD_PIECE_ROUND;
  c.C = (int)(whole ? V : std::min<int64_t>(C, V));
  c.keep = grads && c.C == V;   // the logits of the one piece are formed once
  const size_t tp = (size_t)c.Tp, pc = tp * c.C, td = tp * d;
  c.fused = bf16 || head_f32_fused(T_, c.C, d, second);
  c.order = c.fused && 6.0 * (double)T_ * V * d >= HEAD_ORDER_OPS;
  c.rows = take(c.order ? (t + 1) * 4 : 0);
  c.top = take(t * 4);
  c.z = take(4 * t * 8);
  c.ym = take(2 * t * 4);
  c.f = take(4 * t * 8);
  // The gradient of a piece and, where they are formed in memory, its logits (whose place the gradient
  // takes in fp32 models).
  // The first pass has the statistics of column groups in the gradient's place, of as many columns as
  // fit there, alone of up to HEAD_PART bytes.
  const bool whole_logits = c.keep || !c.fused, inplace = whole_logits && !bf16;
  c.lm = take(whole_logits ? pc * 4 : 0);
  c.ld = take(whole_logits ? pc * 4 : 0);
  const size_t gb = grads && !c.thin && !inplace ? pc * ob : 0, pb = bf16 ? 20 : 40;
  const HeadTile tile = head_tile(T_, c.C);
  c.C1 = c.C;
  size_t part = (size_t)ceil_div(c.C, HEAD_CHUNK) * pb * t;
  if (c.fused) {
    const size_t col = std::max<size_t>(1, t * pb / tile.group), room = std::max<size_t>(2 * gb, piece > 0 ? 0 : HEAD_PART);
    const size_t fit = std::min<size_t>(room / col, HEAD_LAUNCH_ELEMS / std::max<size_t>(1, t));
    c.C1 = (int)std::min<size_t>(V, std::max<size_t>(c.C, fit / HEAD_PIECE_ROUND * HEAD_PIECE_ROUND));
    part = (size_t)ceil_div(c.C1, tile.group) * pb * t;
  }
  c.gm = take(gb);
  c.gd = take(gb);
  c.part = c.gm;
  if (part > at - c.gm) take(part - (at - c.gm));
  if (inplace) {
    c.gm = c.lm;
    c.gd = c.ld;
  }
  const bool products = grads && !c.thin;
  c.xm = take(products ? td * ob : 0);
  c.xd = take(products ? td * ob : 0);
  c.dm = take(products && bf16 ? t * d * 4 : 0);
  c.dd = take(products && bf16 ? t * d * 4 : 0);
  c.runs = take(c.thin ? head_thin_part(T_, V, d) : 0);
  auto split = [&](int cols) {
    return bf16 ? piece_split<bf16_t>(T_, c.Tp, cols, d, products, c.fused, second) : piece_split<float>(T_, c.Tp, cols, d, products, c.fused, second);
  };
  size_t sp = split(c.C);
  if (V % c.C) sp = std::max(sp, split(V % c.C));
  c.split_bytes = sp;
  c.split = take(sp);
  c.total = T_ > 0 ? at : 0;
  return c;
}

// Smaller batches may take more: contractions that are cut, other ways of the logits, a few rows.
// (A batch has a multiple of 8 tokens.)
size_t Engine::head_scratch_most(size_t tokens, int piece) const {
  const int T_ = (int)std::min<size_t>(tokens, 16384);   // of one batch
  std::lock_guard<std::mutex> lk(linear_mu);
  if (T_ == most_tokens && piece == most_piece) return most_bytes;
  most_tokens = T_;
  most_piece = piece;
  most_bytes = head_carve(T_, piece, true, false).total;
  for (int t = 8; t < T_; t += 8) most_bytes = std::max(most_bytes, head_carve(t, piece, true, false).total);
  return most_bytes;
}

template <typename T>
int Engine::head_run(const HeadCall& c) {
  const HeadCarve& k = c.carve;
  hipStream_t st = stream;
  char* ws = c.scratch;
  const int T_ = c.T;
  const int64_t t = T_;
  HeadRows r;
  r.top = (float*)(ws + k.top);
  r.ym = (float*)(ws + k.ym);
  r.yd = r.ym + t;
  for (int q = 0; q < 4; ++q) {
    r.z[q] = (double*)(ws + k.z) + q * t;
    r.f[q] = (double*)(ws + k.f) + q * t;
  }
  float *lm = (float*)(ws + k.lm), *ld = (float*)(ws + k.ld);
  const HeadTile tile = head_tile(T_, k.C);
  const PairT<T> g{(T*)(ws + k.gm), (T*)(ws + k.gd)};
  const T *wm = (const T*)c.w_m, *wd = (const T*)c.w_d;
  const T *xm = (const T*)c.x_m, *xd = (const T*)c.x_d;
  int64_t ldx = c.ldx;
  // (the statistics and the gradient read x where the caller has it or its copy: both within 31 bits)
  const bool near = ((t - 1) * std::max<int64_t>(ldx, d) + d) * (int64_t)sizeof(T) < ((int64_t)1 << 31);
  int32_t* rows = k.order && near ? (int32_t*)(ws + k.rows) : nullptr;
  auto product = [&](GemmArgs* a, int n) -> int {
    for (int p = 0; p < n; ++p)
      if (const char* msg = gemm_check<T>(a[p])) { err = msg; return FDH_ERR_UNSUPPORTED; }
    const GemmScratch sc{(float*)(ws + k.split), HEAD_SPLIT, k.split_bytes};
    int e0 = 0;
    if (timing.on) CK(timing.begin(st, &e0));
    CK(gemm<T>(a, n, sc, st));
    if (timing.on) CK(timing.end(st, 0, e0, gemm_flops(a[0]) + (n > 1 ? gemm_flops(a[1]) : 0.0), 0.0));
    return FDH_OK;
  };
  const bool copy = c.grads && !k.thin && (c.copy_x || T_ != k.Tp);
  HeadCopy cp{};
  if (copy) cp = HeadCopy{ws + k.xm, ws + k.xd, xm, xd, ldx, T_, k.Tp, d, c.tgt};
  int formed = T_;   // rows of the tiles that are formed (for the timing alone)
  // the product that forms columns n0 .. n0 + C - 1 of the logits, for their statistics (keeping them, if
  // they are kept) or for their gradient
  auto logits = [&](int n0, int C, bool grad) -> int {
    if (!k.fused) {
      GemmArgs a[2];
      for (GemmArgs& x : a) {
        x.M = T_; x.N = C; x.K = d;
        x.ldc = C;
      }
      a[0].npairs = 2;
      a[0].A[0] = kmaj(xd, ldx); a[0].B[0] = kmaj(wm + (int64_t)n0 * d, d);
      a[0].A[1] = kmaj(xm, ldx); a[0].B[1] = kmaj(wd + (int64_t)n0 * d, d);
      a[0].C = ld;
      a[1].npairs = logit_pairs(T_, c.second);
      a[1].A[0] = kmaj(xm, ldx); a[1].B[0] = kmaj(wm + (int64_t)n0 * d, d);
      a[1].A[1] = kmaj(xd, ldx); a[1].B[1] = kmaj(wd + (int64_t)n0 * d, d);
      a[1].C = lm;
      return product(a, 2);
    }
    HeadLogits h{};
    h.xm = xm; h.xd = xd; h.ldx = ldx;
    h.wm = wm + (int64_t)n0 * d; h.wd = wd + (int64_t)n0 * d;
    h.T = T_; h.Tp = k.Tp; h.C = C; h.d = d; h.n0 = n0;
    h.tgt = c.tgt;
    h.part = ws + k.part;
    h.gm = g.m; h.gd = g.d;
    if (k.keep) {
      h.lm = lm; h.ld = ld;
    }
    h.tile = tile;
    h.second = c.second;
    h.rows = rows;
    if (n0 == 0 && !grad) h.copy = cp;
    int e0 = 0;
    if (timing.on) CK(timing.begin(st, &e0));
    CK(launch_head_logits<T>(h, r, grad, st));
    if (timing.on) CK(timing.end(st, 0, e0, 2.0 * head_products<T>(tile, c.second) * formed * C * d, 0.0));
    return FDH_OK;
  };
  if (rows) {
    CK(launch_head_rows(rows, c.tgt, T_, st));
    if (timing.on) {
      int32_t live = 0;
      CK(hipMemcpyAsync(&live, rows + T_, sizeof live, hipMemcpyDeviceToHost, st));
      CK(hipStreamSynchronize(st));
      formed = std::min(T_, (int)ceil_div(live, tile.BM) * tile.BM);
    }
  }
  if (copy && !k.fused) CK(launch_head_copy(cp, st));
  HeadOut out{V, c.scale, c.loss_m, c.loss_d, c.rowloss, nullptr, nullptr, ldx, wm, wd, d};
  if (T_ <= HEAD_FINE_ROWS) {
    out.xm = xm;
    out.xd = xd;
  }
  for (int n0 = 0; n0 < V; n0 += k.C1) {
    const int C = std::min(k.C1, V - n0);
    const int rc = logits(n0, C, false);
    if (rc != FDH_OK) return rc;
    const bool last = n0 + C == V;
    typedef std::conditional_t<sizeof(T) == 4, double, float> P;
    if (!k.fused) CK(launch_head_stats(r, (double*)(ws + k.part), lm, ld, T_, C, n0, c.tgt, st));
    CK(launch_head_join(r, (const P*)(ws + k.part), (int)ceil_div(C, k.fused ? tile.group : HEAD_CHUNK), T_, c.tgt, n0 == 0, last, out, st));
  }
  if (copy) {   // (for the products: the statistics read x where it is)
    xm = (const T*)cp.om;
    xd = (const T*)cp.od;
    ldx = d;
  }
  if (!c.grads) return FDH_OK;
  if (k.thin) {
    HeadThin h{};
    h.xm = xm; h.xd = xd; h.ldx = ldx;
    h.wm = wm; h.wd = wd;
    h.lm = lm; h.ld = ld;
    h.tgt = c.tgt;
    h.T = T_; h.V = V; h.d = d;
    h.scale = (float)c.scale;
    h.alpha_w = (float)c.scale_w;
    h.dxm = c.dx_m; h.dxd = c.dx_d; h.lddx = c.lddx;
    h.dw = c.dw;
    h.acc = c.acc;
    h.part = (float*)(ws + k.runs);
    CK(launch_head_thin<T>(h, r, c.out_f32, st));
    return FDH_OK;
  }
  // the gradient of x is added up over the pieces in fp32
  const bool round = !c.out_f32 && k.C < V;
  const bool op_out = !c.out_f32 && !round;
  void* dxm = round ? (void*)(ws + k.dm) : c.dx_m;
  void* dxd = round ? (void*)(ws + k.dd) : c.dx_d;
  const int64_t lddx = round ? d : c.lddx;
  const size_t ob = c.out_f32 ? 4 : sizeof(T);
  for (int n0 = 0; n0 < V; n0 += k.C) {
    const int C = std::min(k.C, V - n0);
    int rc = k.keep ? FDH_OK : logits(n0, C, true);
    if (rc != FDH_OK) return rc;
    if (k.keep || !k.fused) CK(launch_head_dlogits<T>(g, r, lm, ld, T_, k.Tp, C, n0, c.tgt, st));
    GemmArgs a[2];
    for (GemmArgs& x : a) {
      x.M = T_; x.N = d; x.K = C;
      x.ldc = lddx;
      x.out_type = op_out ? OUT_OP : OUT_F32;
      x.alpha = (float)c.scale;
      x.beta = n0 > 0 ? 1.f : 0.f;
    }
    a[0].npairs = 2;
    a[0].A[0] = kmaj(g.d, C); a[0].B[0] = mnmaj(wm + (int64_t)n0 * d, d);
    a[0].A[1] = kmaj(g.m, C); a[0].B[1] = mnmaj(wd + (int64_t)n0 * d, d);
    a[0].C = dxd;
    a[1].npairs = c.second ? 2 : 1;
    a[1].A[0] = kmaj(g.m, C); a[1].B[0] = mnmaj(wm + (int64_t)n0 * d, d);
    a[1].A[1] = kmaj(g.d, C); a[1].B[1] = mnmaj(wd + (int64_t)n0 * d, d);
    a[1].C = dxm;
    rc = product(a, 2);
    if (rc != FDH_OK) return rc;
    GemmArgs w;
    w.M = C; w.N = d; w.K = k.Tp; w.npairs = 2;
    w.A[0] = mnmaj(g.m, C); w.B[0] = mnmaj(xd, ldx);
    w.A[1] = mnmaj(g.d, C); w.B[1] = mnmaj(xm, ldx);
    w.C = (char*)c.dw + (size_t)n0 * d * ob;
    w.ldc = d;
    w.out_type = c.out_f32 ? OUT_F32 : OUT_OP;
    w.alpha = (float)c.scale_w;
    w.beta = c.acc ? 1.f : 0.f;
    rc = product(&w, 1);
    if (rc != FDH_OK) return rc;
  }
  if (round) {
    const PairT<bf16_t> o{(bf16_t*)c.dx_m, (bf16_t*)c.dx_d};
    CK(launch_head_round(o, c.lddx, (const float*)dxm, (const float*)dxd, T_, d, st));
  }
  return FDH_OK;
}
template int Engine::head_run<float>(const HeadCall&);
template int Engine::head_run<bf16_t>(const HeadCall&);

int Engine::head_check(const fdh_head_inputs* in, bool grads, size_t scratch_bytes, const void* scratch, HeadCall* c) {
  if (quad) { err = "needs a language-model context"; return FDH_ERR_UNSUPPORTED; }
  if (!in) { err = "null inputs"; return FDH_ERR_INVALID_ARG; }
  if (in->T < 0 || in->piece < 0 || in->reserved != 0) { err = "T and piece must not be negative, reserved 0"; return FDH_ERR_INVALID_ARG; }
  if (in->T > HEAD_MAX_ROWS || d > HEAD_MAX_WIDTH) { err = "T must be <= 2^20 and d_model <= 2^16"; return FDH_ERR_UNSUPPORTED; }
  const int ob = bf16 ? 2 : 4;
  if (in->T > 0) {
    if (bad_rows(in->x_m, in->ldx, d, ob) || bad_rows(in->x_d, in->ldx, d, ob) || in->ldx > HEAD_MAX_LD) {
      err = "x: 16-byte aligned rows, d_model to 2^20 elements apart";
      return FDH_ERR_INVALID_ARG;
    }
    if (bad_rows(in->w_m, d, d, ob) || bad_rows(in->w_d, d, d, ob)) { err = "w: null or not 16-byte aligned"; return FDH_ERR_INVALID_ARG; }
    if (!in->targets || (uintptr_t)in->targets % 4) { err = "targets: null or not 4-byte aligned"; return FDH_ERR_INVALID_ARG; }
    c->carve = head_carve(in->T, in->piece, grads);
    if (!scratch || scratch_bytes < c->carve.total) { err = "scratch smaller than fdh_head_scratch_bytes"; return FDH_ERR_WORKSPACE; }
    if ((uintptr_t)scratch % 256) { err = "scratch must be 256-byte aligned"; return FDH_ERR_WORKSPACE; }
  }
  c->x_m = in->x_m; c->x_d = in->x_d; c->ldx = in->ldx;
  c->w_m = in->w_m; c->w_d = in->w_d;
  c->tgt = in->targets;
  c->T = in->T;
  c->scratch = (char*)scratch;
  return FDH_OK;
}

int Engine::head_loss(const fdh_head_inputs* in, float* loss_m, float* loss_d, void* scratch, size_t scratch_bytes) {
  HeadCall c;
  const int rc = head_check(in, false, scratch_bytes, scratch, &c);
  if (rc != FDH_OK) return rc;
  if (c.T == 0) return FDH_OK;
  if (!loss_m || !loss_d || (uintptr_t)loss_m % 4 || (uintptr_t)loss_d % 4) { err = "loss: null or not 4-byte aligned"; return FDH_ERR_INVALID_ARG; }
  const int64_t ob = bf16 ? 2 : 4, T_ = c.T, wd = (int64_t)d * ob;
  const Region o[3] = {flat(loss_m, 4 * T_), flat(loss_d, 4 * T_), flat(scratch, (int64_t)c.carve.total)};
  const Region r[5] = {{(const char*)c.x_m, T_, c.ldx * ob, wd}, {(const char*)c.x_d, T_, c.ldx * ob, wd}, flat(c.w_m, V * wd),
                       flat(c.w_d, V * wd), flat(c.tgt, 4 * T_)};
  if (any_overlap(o, 3, r, 5)) { err = "an output or the scratch overlaps an input or another output"; return FDH_ERR_INVALID_ARG; }
  c.loss_m = loss_m; c.loss_d = loss_d;
  return bf16 ? head_run<bf16_t>(c) : head_run<float>(c);
}

int Engine::head_grad(const fdh_head_inputs* in, float* loss_m, float* loss_d, const fdh_head_grads* g, void* scratch,
                      size_t scratch_bytes) {
  HeadCall c;
  const int rc = head_check(in, true, scratch_bytes, scratch, &c);
  if (rc != FDH_OK) return rc;
  if (!g) { err = "null gradients"; return FDH_ERR_INVALID_ARG; }
  if ((loss_m == nullptr) != (loss_d == nullptr) || (uintptr_t)loss_m % 4 || (uintptr_t)loss_d % 4) {
    err = "loss: both or neither, 4-byte aligned";
    return FDH_ERR_INVALID_ARG;
  }
  if (!(g->eps > 0.0) || !std::isfinite(g->eps) || !std::isfinite((float)g->scale) || !std::isfinite((float)(g->scale / g->eps))) {
    err = "eps must be positive and finite, scale and scale / eps finite in float32";
    return FDH_ERR_INVALID_ARG;
  }
  if (g->dtype != FDH_F32 && g->dtype != cfg.dtype) { err = "gradients are float32 or of the context's dtype"; return FDH_ERR_INVALID_ARG; }
  if (g->accumulate && g->dtype != FDH_F32) { err = "accumulate needs float32 gradients"; return FDH_ERR_INVALID_ARG; }
  const int64_t ob = bf16 ? 2 : 4, T_ = c.T, wd = (int64_t)d * ob, gb = g->dtype == FDH_F32 ? 4 : 2, gw = (int64_t)d * gb;
  if (!g->dw || (uintptr_t)g->dw % 16) { err = "dw: null or not 16-byte aligned"; return FDH_ERR_INVALID_ARG; }
  if (T_ > 0 && (bad_rows(g->dx_m, g->lddx, d, (int)gb) || bad_rows(g->dx_d, g->lddx, d, (int)gb))) {
    err = "dx: 16-byte aligned rows, at least d_model elements apart";
    return FDH_ERR_INVALID_ARG;
  }
  if (T_ == 0) {
    if (!g->accumulate) CK(launch_fill_f32((float*)g->dw, V * gw / 4, 0.f, stream));
    return FDH_OK;
  }
  const Region o[6] = {flat(loss_m, 4 * T_), flat(loss_d, 4 * T_), {(const char*)g->dx_m, T_, g->lddx * gb, gw},
                       {(const char*)g->dx_d, T_, g->lddx * gb, gw}, flat(g->dw, V * gw),
                       flat(scratch, (int64_t)c.carve.total)};
  const Region r[5] = {{(const char*)c.x_m, T_, c.ldx * ob, wd}, {(const char*)c.x_d, T_, c.ldx * ob, wd}, flat(c.w_m, V * wd),
                       flat(c.w_d, V * wd), flat(c.tgt, 4 * T_)};
  if (any_overlap(o, 6, r, 5)) { err = "an output or the scratch overlaps an input or another output"; return FDH_ERR_INVALID_ARG; }
  c.loss_m = loss_m; c.loss_d = loss_d;
  c.grads = true;
  c.scale = g->scale;
  c.scale_w = g->scale / g->eps;
  c.dx_m = g->dx_m; c.dx_d = g->dx_d; c.lddx = g->lddx;
  c.dw = g->dw;
  c.out_f32 = g->dtype == FDH_F32;
  c.acc = g->accumulate != 0;
  return bf16 ? head_run<bf16_t>(c) : head_run<float>(c);
}

}  // namespace fdh
