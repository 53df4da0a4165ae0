// The loss over the vocabulary at both points, a piece of the vocabulary at a time.
//
// For the logits' pair (lm, ld) of a row and its reference c = max_j (lm_j + |ld_j|) let
//   a_j = e^(lm_j - c) cosh ld_j,  s_j = e^(lm_j - c) sinh ld_j,  so that  e^(l_j+- - c) = a_j +- s_j,
// each with full relative precision however small ld is, and Zm = sum a, Zd = sum s.  Then
//   loss.m = c + log(Z+ Z-) / 2 - lm_y,          loss.d = log(Z+ / Z-) / 2 - ld_y   (Z+- = Zm +- Zd),
//   P.m = (a Zm - s Zd) / (Z+ Z-),               P.d = (s Zm - a Zd) / (Z+ Z-)
// and the logits' gradient is w (P.m - [j = y]) and w P.d with the rows' weight w.  Where the two
// points are far apart (|ld| >= 1/2) a - s would lose bits: there p = a + s and q = a - s are formed
// instead, their sums kept apart (Z+ = Sa + Ss + Sp, Z- = Sa - Ss + Sq) and P+- = p / Z+, q / Z-.
// A first pass over the pieces leaves c, the four sums and the target's logits of every row, a
// second one forms the logits again and gives their gradient to the products: nothing of the
// size of the logits stays.
#include "head_dev.h"
#include "kernels.h"

namespace fdh {

namespace {

constexpr int NT = 256;

// targets of a [B, S] batch, aligned with the rows that predict them (the next token or its
// label; none for the last position); out of range: clamped, the batch's check reports it
__global__ void head_targets_kernel(int32_t* tgt, const int32_t* tok, const int32_t* lab, int T_, int S, int V) {
  const int t = blockIdx.x * NT + threadIdx.x;
  if (t >= T_) return;
  const int y = t % S == S - 1 ? IGNORE_LABEL : (lab ? lab[t + 1] : tok[t + 1]);
  tgt[t] = y == IGNORE_LABEL ? y : min(max(y, 0), V - 1);
}

// Statistics of one piece of the logits, columns n0 .. n0 + C - 1 of the vocabulary, joined to
// those of the pieces before (fp32 models).  One workgroup per row; every thread keeps its sums
// relative to its own maximum.
__global__ __launch_bounds__(NT) void head_stats_kernel(HeadRows r, const float* lm, const float* ld, int C, int n0,
                                                        const int32_t* tgt, bool first) {
  __shared__ double sh[NT / 64];
  const int64_t t = blockIdx.x;
  const int y = tgt[t];
  if (y == IGNORE_LABEL) return;
  const float* m = lm + t * C;
  const float* d = ld + t * C;
  float mt = -INFINITY;
  double z[4] = {0.0, 0.0, 0.0, 0.0};   // Sa, Ss, Sp, Sq
  for (int j = 4 * threadIdx.x; j < C; j += 4 * NT) {
    const float4 a = *reinterpret_cast<const float4*>(m + j), b = *reinterpret_cast<const float4*>(d + j);
    const float top = fmaxf(fmaxf(head_ref(a.x, b.x), head_ref(a.y, b.y)), fmaxf(head_ref(a.z, b.z), head_ref(a.w, b.w)));
    if (top > mt) {
      const double f = mt > -INFINITY ? exp((double)mt - (double)top) : 0.0;
#pragma unroll
      for (int k = 0; k < 4; ++k) z[k] *= f;
      mt = top;
    }
    auto add = [&](float x, float y) {
      double p, s;
      pair_exp(x, y, mt, p, s);
      const int k = far_apart(y) ? 2 : 0;
      z[0] += k ? 0.0 : p;
      z[1] += k ? 0.0 : s;
      z[2] += k ? p : 0.0;
      z[3] += k ? s : 0.0;
    };
    add(a.x, b.x);
    add(a.y, b.y);
    add(a.z, b.z);
    add(a.w, b.w);
  }
  const float old = first ? -INFINITY : r.top[t];
  const float mx = (float)block_max<NT>(fmax((double)mt, (double)old), sh);
  // (a thread that saw NaN alone has no maximum: its sums are NaN at any factor but none)
  const double f = mt > -INFINITY ? exp((double)mt - (double)mx) : 1.0;
#pragma unroll
  for (int k = 0; k < 4; ++k) z[k] = block_sum<NT>(z[k] * f, sh);
  if (threadIdx.x != 0) return;
  if (!first) {
    const double g = old > -INFINITY ? exp((double)old - (double)mx) : 1.0;
#pragma unroll
    for (int k = 0; k < 4; ++k) z[k] += r.z[k][t] * g;
  }
  r.top[t] = mx;
#pragma unroll
  for (int k = 0; k < 4; ++k) r.z[k][t] = z[k];
  if (y >= n0 && y < n0 + C) {
    r.ym[t] = m[y - n0];
    r.yd[t] = d[y - n0];
  }
}

// Losses of the rows and the factors of their gradients.  A target outside the vocabulary makes
// its row NaN; rows without a target have no loss and no gradient.
__global__ void head_rows_kernel(HeadRows r, const int32_t* tgt, int T_, int V, double scale, float* loss_m, float* loss_d,
                                 double* rowloss) {
  const int t = blockIdx.x * NT + threadIdx.x;
  if (t >= T_) return;
  const int y = tgt[t];
  double m = 0.0, d = 0.0, f[4] = {0.0, 0.0, 0.0, 0.0};
  if (y != IGNORE_LABEL) {
    if (y < 0 || y >= V) {
      m = d = f[0] = f[1] = f[2] = f[3] = __builtin_nan("");
    } else {
      const double sa = r.z[0][t], ss = r.z[1][t], sp = r.z[2][t], sq = r.z[3][t];
      const double zp = sa + ss + sp, zn = sa - ss + sq, zm = sa + 0.5 * (sp + sq), zd = ss + 0.5 * (sp - sq);
      const double lp = log(zp), ln = log(zn);
      m = (double)r.top[t] - (double)r.ym[t] + 0.5 * (lp + ln);
      d = (fabs(zd) < 0.5 * zm ? atanh(zd / zm) : 0.5 * (lp - ln)) - (double)r.yd[t];
      f[0] = scale * (zm / (zp * zn));
      f[1] = scale * (zd / (zp * zn));
      f[2] = 0.5 * scale / zp;
      f[3] = 0.5 * scale / zn;
    }
  }
  if (loss_m) {
    loss_m[t] = (float)m;
    loss_d[t] = (float)d;
  }
  if (rowloss) {
    rowloss[t] = (m + d) * scale;
    rowloss[T_ + t] = (m - d) * scale;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) r.f[k][t] = f[k];
}

// Gradient of one piece of the logits in their place, [Tp][C] (fp32 models); rows without a target
// and rows behind the last are zeros.
__global__ __launch_bounds__(NT) void head_dlogits_kernel(HeadRows r, float* lm, float* ld, int T_, int C, int n0,
                                                          const int32_t* tgt, double scale) {
  const int64_t t = blockIdx.x;
  const int y = t < T_ ? tgt[t] : IGNORE_LABEL;
  const int64_t base = t * C;
  if (y == IGNORE_LABEL) {
    for (int j = threadIdx.x; j < C; j += NT) {
      lm[base + j] = 0.f;
      ld[base + j] = 0.f;
    }
    return;
  }
  const float c = r.top[t];
  const double f0 = r.f[0][t], f1 = r.f[1][t], f2 = r.f[2][t], f3 = r.f[3][t];
  for (int j = threadIdx.x; j < C; j += NT) {
    double p, s;
    const float b = ld[base + j];
    pair_exp(lm[base + j], b, c, p, s);
    const bool far = far_apart(b);
    const double m = far ? p * f2 + s * f3 : p * f0 - s * f1;
    lm[base + j] = (float)(m - (n0 + j == y ? scale : 0.0));
    ld[base + j] = (float)(far ? p * f2 - s * f3 : s * f0 - p * f1);
  }
}

// x as the gradients' products read it: contiguous, with zeros in the rows that have no target
// (whatever stands there) and in those behind the last
template <typename T>
__global__ __launch_bounds__(NT) void head_copy_kernel(PairT<T> o, const T* xm, const T* xd, int64_t ldx, int T_, int dm,
                                                       const int32_t* tgt) {
  constexpr int VEC = 16 / sizeof(T);
  const int64_t t = blockIdx.x;
  const bool live = t < T_ && tgt[t] != IGNORE_LABEL;
  for (int c = VEC * threadIdx.x; c < dm; c += VEC * NT) {
    const uint4 none = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(o.m + t * dm + c) = live ? *reinterpret_cast<const uint4*>(xm + t * ldx + c) : none;
    *reinterpret_cast<uint4*>(o.d + t * dm + c) = live ? *reinterpret_cast<const uint4*>(xd + t * ldx + c) : none;
  }
}

// bf16 copy of the fp32 pair [T][dm]
__global__ __launch_bounds__(NT) void head_round_kernel(PairT<bf16_t> o, int64_t ldo, const float* m, const float* d, int dm) {
  const int64_t t = blockIdx.x;
  for (int c = 4 * threadIdx.x; c < dm; c += 4 * NT) {
    const float4 a = *reinterpret_cast<const float4*>(m + t * dm + c), b = *reinterpret_cast<const float4*>(d + t * dm + c);
    auto two = [](float x, float y) { return (uint32_t)f32_to_bf16(x) | ((uint32_t)f32_to_bf16(y) << 16); };
    *reinterpret_cast<uint2*>(o.m + t * ldo + c) = make_uint2(two(a.x, a.y), two(a.z, a.w));
    *reinterpret_cast<uint2*>(o.d + t * ldo + c) = make_uint2(two(b.x, b.y), two(b.z, b.w));
  }
}

}  // namespace

hipError_t launch_head_targets(int32_t* tgt, const int32_t* tok, const int32_t* lab, int T_, int S, int V, hipStream_t s) {
  hipLaunchKernelGGL(head_targets_kernel, dim3(ceil_div(T_, NT)), dim3(NT), 0, s, tgt, tok, lab, T_, S, V);
  return hipGetLastError();
}
hipError_t launch_head_stats(const HeadRows& r, const float* lm, const float* ld, int T_, int C, int n0, const int32_t* tgt, bool first,
                             hipStream_t s) {
  hipLaunchKernelGGL(head_stats_kernel, dim3(T_), dim3(NT), 0, s, r, lm, ld, C, n0, tgt, first);
  return hipGetLastError();
}
hipError_t launch_head_rows(const HeadRows& r, const int32_t* tgt, int T_, int V, double scale, float* loss_m, float* loss_d,
                            double* rowloss, hipStream_t s) {
  hipLaunchKernelGGL(head_rows_kernel, dim3(ceil_div(T_, NT)), dim3(NT), 0, s, r, tgt, T_, V, scale, loss_m, loss_d, rowloss);
  return hipGetLastError();
}
hipError_t launch_head_dlogits(const HeadRows& r, float* lm, float* ld, int T_, int Tp, int C, int n0, const int32_t* tgt,
                               double scale, hipStream_t s) {
  hipLaunchKernelGGL(head_dlogits_kernel, dim3(Tp), dim3(NT), 0, s, r, lm, ld, T_, C, n0, tgt, scale);
  return hipGetLastError();
}
template <typename T>
hipError_t launch_head_copy(PairT<T> o, const T* xm, const T* xd, int64_t ldx, int T_, int Tp, int dm, const int32_t* tgt, hipStream_t s) {
  hipLaunchKernelGGL(head_copy_kernel<T>, dim3(Tp), dim3(NT), 0, s, o, xm, xd, ldx, T_, dm, tgt);
  return hipGetLastError();
}
hipError_t launch_head_round(PairT<bf16_t> o, int64_t ldo, const float* m, const float* d, int T_, int dm, hipStream_t s) {
  hipLaunchKernelGGL(head_round_kernel, dim3(T_), dim3(NT), 0, s, o, ldo, m, d, dm);
  return hipGetLastError();
}

template hipError_t launch_head_copy<float>(PairT<float>, const float*, const float*, int64_t, int, int, int, const int32_t*, hipStream_t);
template hipError_t launch_head_copy<bf16_t>(PairT<bf16_t>, const bf16_t*, const bf16_t*, int64_t, int, int, int, const int32_t*,
                                             hipStream_t);

}  // namespace fdh
