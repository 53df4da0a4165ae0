// The loss over the vocabulary at both points, a piece of the vocabulary at a time.
//
// For the logits' pair (lm, ld) of a row and its reference c, from max_j (lm_j + |ld_j|) to max lm + max |ld|, let
//   a_j = e^(lm_j - c) cosh ld_j,  s_j = e^(lm_j - c) sinh ld_j,  so that  e^(l_j+- - c) = a_j +- s_j,
// each with full relative precision however small ld is, and Zm = sum a, Zd = sum s.  Then
//   loss.m = c + log(Z+ Z-) / 2 - lm_y,          loss.d = log(Z+ / Z-) / 2 - ld_y   (Z+- = Zm +- Zd),
//   P.m = (a Zm - s Zd) / (Z+ Z-),               P.d = (s Zm - a Zd) / (Z+ Z-)
// and the logits' gradient is P.m - [j = y] and P.d (the rows' weight is the products' factor: in the
// rounded gradient it would put one and the same error into every row).  Where the two
// points are far apart (|ld| >= 1/2) a - s would lose bits: there p = a + s and q = a - s are formed
// instead, their sums kept apart (Z+ = Sa + Ss + Sp, Z- = Sa - Ss + Sq) and P+- = p / Z+, q / Z-.
// Which of the two a logit takes may differ between the passes: only the sums' totals are used.
// A first pass over the pieces leaves c, the four sums and the target's logits of every row, a
// second one forms the logits again and gives their gradient to the products: nothing of the
// size of the logits stays.  Where one piece holds the vocabulary its logits are formed once.
#include <algorithm>
#include <type_traits>

#include "head_dev.h"

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

// One workgroup: a wavefront counts a run of rows, the runs' counts are added up over the wavefronts.
constexpr int RT = 1024;
__global__ __launch_bounds__(RT) void head_rows_kernel(int32_t* rows, const int32_t* tgt, int T_) {
  __shared__ int sh[RT / 64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int per = (T_ + RT - 1) / RT * 64, from = min(w * per, T_), end = min(from + per, T_);
  auto live = [&](int t) { return t + lane < end && tgt[min(t + lane, T_ - 1)] != IGNORE_LABEL; };
  int n = 0;
#pragma unroll 8
  for (int t = from; t < end; t += 64) n += __popcll(__ballot(live(t)));
  if (lane == 0) sh[w] = n;
  __syncthreads();
  int at = 0, all = 0;
  for (int q = 0; q < RT / 64; ++q) {
    if (q < w) at += sh[q];
    all += sh[q];
  }
  int none = all + from - at;   // (of the rows before, from - at have no target)
#pragma unroll 8
  for (int t = from; t < end; t += 64) {
    const bool y = live(t);
    const uint64_t m = __ballot(y);
    const int ahead = __popcll(m & (((uint64_t)1 << lane) - 1)), count = __popcll(m);
    if (t + lane < end) rows[y ? at + ahead : none + lane - ahead] = t + lane;
    at += count;
    none += min(64, end - t) - count;
  }
  if (threadIdx.x == 0) rows[T_] = all;
}

// Statistics of one piece of the logits (fp32 models, many rows), part [chunks][5][T]: the maximum and the four
// sums of a row's CHUNK columns, one workgroup each; every thread keeps its sums relative to its own
// maximum.
constexpr int CHUNK = HEAD_CHUNK;
__global__ __launch_bounds__(NT) void head_stats_kernel(HeadRows r, double* part, const float* lm, const float* ld, int T_, int C, int n0,
                                                        const int32_t* tgt) {
  __shared__ double sh[NT / 64];
  const int64_t t = blockIdx.x;
  const int y = tgt[t];
  if (y == IGNORE_LABEL) return;
  const float* m = lm + t * C;
  const float* d = ld + t * C;
  const int from = blockIdx.y * CHUNK, end = min(from + CHUNK, C);
  float mt = -INFINITY;
  double z[4] = {0.0, 0.0, 0.0, 0.0};   // Sa, Ss, Sp, Sq
  for (int j = from + 4 * threadIdx.x; j < end; j += 4 * NT) {
    const float4 a = *reinterpret_cast<const float4*>(m + j), b = *reinterpret_cast<const float4*>(d + j);
    const float top = fmaxf(fmaxf(head_ref(a.x, b.x), head_ref(a.y, b.y)), fmaxf(head_ref(a.z, b.z), head_ref(a.w, b.w)));
    if (top > mt) {
      const double f = mt > -INFINITY ? exp((double)mt - (double)top) : 0.0;
#pragma unroll
      for (int k = 0; k < 4; ++k) z[k] *= f;
      mt = top;
    }
    const float x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
    float sa = 0.f, ss = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (far_apart_fine(x[e], y[e], mt)) {
        double p, q;
        pair_exp_far(x[e], y[e], mt, p, q);
        z[2] += p;
        z[3] += q;
      } else {
        float p, s;
        pair_exp<true>(x[e], y[e], mt, p, s);
        sa += p;
        ss += s;
      }
    }
    z[0] += sa;
    z[1] += ss;
  }
  const float mx = (float)block_max<NT>((double)mt, sh);
  // (a thread that saw NaN alone has no maximum: its sums are NaN at any factor but none)
  const double f = mt > -INFINITY ? exp((double)mt - (double)mx) : 1.0;
#pragma unroll
  for (int k = 0; k < 4; ++k) z[k] = block_sum<NT>(z[k] * f, sh);
  if (threadIdx.x != 0) return;
  double* o = part + (int64_t)blockIdx.y * 5 * T_ + t;
  o[0] = mx;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[(int64_t)(k + 1) * T_] = z[k];
  if (y >= n0 + from && y < n0 + end) {
    r.ym[t] = m[y - n0];
    r.yd[t] = d[y - n0];
  }
}

__device__ inline void wide(const float* p, double (&v)[4]) {
  const float4 u = *reinterpret_cast<const float4*>(p);
  v[0] = u.x; v[1] = u.y; v[2] = u.z; v[3] = u.w;
}
__device__ inline void wide(const bf16_t* p, double (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t x[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = __uint_as_float(x[k] << 16);
    v[2 * k + 1] = __uint_as_float(x[k] & 0xffff0000u);
  }
}

// Joins the groups' statistics of the rows to those of the pieces before: 256 / R threads per row
// take every 256 / R-th group, each relative to its own maximum; then the row's maximum, and the sums
// relative to it, across the wavefronts' lanes and the wavefronts (a fixed order).  After the last
// piece the rows' losses and the factors of their gradients: a target outside the vocabulary makes
// its row NaN, rows without a target have no loss and no gradient.  loss.d is the difference of a mean
// over the vocabulary, whose errors average out, and the target's ld_y, whose error stands alone:
// of a few rows it may be all that they hold, so there the target's logits are formed in fp64 (1 row of
// 32000 x 2048 bf16 whose loss.d is a fifth of ld's spread: 2e-6 of it off before).
template <int R, typename P>
__global__ __launch_bounds__(NT) void head_join_kernel(HeadRows r, const P* part, int groups, int T_, const int32_t* tgt, bool first,
                                                       bool last, HeadOut out) {
  constexpr int L = NT / R, W = NT / 64;
  typedef std::conditional_t<sizeof(P) == 8, float, bf16_t> T;
  __shared__ double sh[W][R][7];
  const int lr = threadIdx.x % R, l = threadIdx.x / R, w = threadIdx.x >> 6;
  const int64_t t = (int64_t)blockIdx.x * R + lr;
  const int y = t < T_ ? tgt[t] : IGNORE_LABEL;
  const bool on = y != IGNORE_LABEL;
  double top = -INFINITY, z[4] = {0.0, 0.0, 0.0, 0.0};
  // sums at no maximum are NaN or nothing: their factor is 1
  auto factor = [](double from, double to) { return from == to || from == -INFINITY ? 1.0 : exp(from - to); };
  auto join = [&](double m, double x0, double x1, double x2, double x3) {
    const double mx = fmax(top, m);
    const double f = factor(top, mx), g = factor(m, mx);
    z[0] = z[0] * f + x0 * g;
    z[1] = z[1] * f + x1 * g;
    z[2] = z[2] * f + x2 * g;
    z[3] = z[3] * f + x3 * g;
    top = mx;
  };
  if (on) {
    constexpr int U = 4;
    for (int g0 = l; g0 < groups; g0 += U * L) {
      P v[U][5];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < 5; ++k) v[u][k] = part[((int64_t)min(g0 + u * L, groups - 1) * 5 + k) * T_ + t];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (g0 + u * L < groups) join(v[u][0], v[u][1], v[u][2], v[u][3], v[u][4]);
    }
    if (!first && l == 0) join(r.top[t], r.z[0][t], r.z[1][t], r.z[2][t], r.z[3][t]);
  }
  double ym = 0.0, yd = 0.0;
  const bool fine = R == 1 && last && out.xm;
  if (fine && on && y >= 0 && y < out.V) {
    constexpr int VEC = 16 / sizeof(T);
    const T *xm = (const T*)out.xm + t * out.ldx, *xd = (const T*)out.xd + t * out.ldx;
    const T *wm = (const T*)out.wm + (int64_t)y * out.d, *wd = (const T*)out.wd + (int64_t)y * out.d;
    for (int j = VEC * l; j < out.d; j += VEC * NT) {
      double a[VEC], b[VEC], p[VEC], q[VEC];
      wide(xm + j, a);
      wide(xd + j, b);
      wide(wm + j, p);
      wide(wd + j, q);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        ym += a[e] * p[e] + b[e] * q[e];
        yd += b[e] * p[e] + a[e] * q[e];
      }
    }
  }
  double mx = top;
#pragma unroll
  for (int o = R; o < 64; o <<= 1) mx = fmax(mx, __shfl_xor(mx, o, 64));
  if (l % (64 / R) == 0) sh[w][lr][0] = mx;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < W; ++q) mx = fmax(mx, sh[q][lr][0]);
  const double f0 = factor(top, mx);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    z[k] *= f0;
#pragma unroll
    for (int o = R; o < 64; o <<= 1) z[k] += __shfl_xor(z[k], o, 64);
    if (l % (64 / R) == 0) sh[w][lr][k + 1] = z[k];
  }
  if (fine) {
#pragma unroll
    for (int o = R; o < 64; o <<= 1) {
      ym += __shfl_xor(ym, o, 64);
      yd += __shfl_xor(yd, o, 64);
    }
    if (l % (64 / R) == 0) {
      sh[w][lr][5] = ym;
      sh[w][lr][6] = yd;
    }
  }
  __syncthreads();
  if (l != 0 || t >= T_) return;
  top = mx;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    z[k] = sh[0][lr][k + 1];
#pragma unroll
    for (int q = 1; q < W; ++q) z[k] += sh[q][lr][k + 1];
  }
  if (on) r.top[t] = (float)top;   // (a maximum of floats)
  if (!last) {
    if (on)
#pragma unroll
      for (int k = 0; k < 4; ++k) r.z[k][t] = z[k];
    return;
  }
  double m = 0.0, d = 0.0, f[4] = {0.0, 0.0, 0.0, 0.0};
  if (on && (y < 0 || y >= out.V)) {
    m = d = f[0] = f[1] = f[2] = f[3] = __builtin_nan("");
  } else if (on) {
    const double sa = z[0], ss = z[1], sp = z[2], sq = z[3];
    double zp = sa + ss + sp, zn = sa - ss + sq;
    const double zm = sa + 0.5 * (sp + sq), zd = ss + 0.5 * (sp - sq);
    // Half differences to H leave both sums at e^(-2 H) or more.  Below LEAST, which 30 (bf16) and 300 (fp32) do
    // not reach, the range of the exponentials may have cut terms (2^-126 in fp32: of 2^18 words 2^-18 of a
    // sum of 2^-90 at the most; 2^-1022 in fp64), so the row is NaN.
    constexpr double LEAST = sizeof(P) == 8 ? 0x1p-900 : 0x1p-90;
    if (!(zp >= LEAST && zn >= LEAST)) zp = zn = __builtin_nan("");
    const double lp = log(zp), ln = log(zn);
    if (fine) {
      ym = yd = 0.0;
#pragma unroll
      for (int q = 0; q < W; ++q) {
        ym += sh[q][lr][5];
        yd += sh[q][lr][6];
      }
    } else {
      ym = r.ym[t];
      yd = r.yd[t];
    }
    m = top - ym + 0.5 * (lp + ln);
    d = (fabs(zd) < 0.5 * zm ? atanh(zd / zm) : 0.5 * (lp - ln)) - yd;
    f[0] = zm / (zp * zn);
    f[1] = zd / (zp * zn);
    f[2] = 0.5 / zp;
    f[3] = 0.5 / zn;
  }
  if (out.loss_m) {
    out.loss_m[t] = (float)m;
    out.loss_d[t] = (float)d;
  }
  if (out.rowloss) {
    out.rowloss[t] = (m + d) * out.scale;
    out.rowloss[T_ + t] = (m - d) * out.scale;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) r.f[k][t] = f[k];
}

// Gradient of logits that are in memory (one piece holds the vocabulary, or an fp32 model's many rows)
// in the operand type (what its rounding costs stands at head_gemm.hip's), [Tp][C]; rows without a target
// and rows behind the last are zeros.  o may be the logits (fp32 models).
__device__ inline void store4(float* p, float a, float b, float c, float d) { *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d); }
__device__ inline void store4(bf16_t* p, float a, float b, float c, float d) {
  auto two = [](float x, float y) { return (uint32_t)f32_to_bf16(x) | ((uint32_t)f32_to_bf16(y) << 16); };
  *reinterpret_cast<uint2*>(p) = make_uint2(two(a, b), two(c, d));
}
template <typename T>
__global__ __launch_bounds__(NT) void head_dlogits_kernel(PairT<T> o, HeadRows r, const float* lm, const float* ld, int T_, int C, int n0,
                                                          const int32_t* tgt) {
  const int64_t t = blockIdx.x;
  const int y = t < T_ ? tgt[t] : IGNORE_LABEL;
  const int64_t base = t * C;
  const int from = blockIdx.y * CHUNK, end = min(from + CHUNK, C);
  if (y == IGNORE_LABEL) {
    for (int j = from + 4 * threadIdx.x; j < end; j += 4 * NT) {
      store4(o.m + base + j, 0.f, 0.f, 0.f, 0.f);
      store4(o.d + base + j, 0.f, 0.f, 0.f, 0.f);
    }
    return;
  }
  const float c = r.top[t];
  const double f0 = r.f[0][t], f1 = r.f[1][t], f2 = r.f[2][t], f3 = r.f[3][t];
  for (int j = from + 4 * threadIdx.x; j < end; j += 4 * NT) {
    const float4 a4 = *reinterpret_cast<const float4*>(lm + base + j), b4 = *reinterpret_cast<const float4*>(ld + base + j);
    const float a[4] = {a4.x, a4.y, a4.z, a4.w}, b[4] = {b4.x, b4.y, b4.z, b4.w};
    float gm[4], gd[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      logit_grad<sizeof(T) == 4>(a[e], b[e], c, f0, f1, f2, f3, gm[e], gd[e]);
      if (n0 + j + e == y) gm[e] -= 1.f;
    }
    store4(o.m + base + j, gm[0], gm[1], gm[2], gm[3]);
    store4(o.d + base + j, gd[0], gd[1], gd[2], gd[3]);
  }
}

__global__ __launch_bounds__(NT) void head_copy_kernel(HeadCopy c) {
  copy_rows<float>(c, blockIdx.x, gridDim.x);
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
hipError_t launch_head_rows(int32_t* rows, const int32_t* tgt, int T_, hipStream_t s) {
  hipLaunchKernelGGL(head_rows_kernel, dim3(1), dim3(RT), 0, s, rows, tgt, T_);
  return hipGetLastError();
}
hipError_t launch_head_stats(const HeadRows& r, double* part, const float* lm, const float* ld, int T_, int C, int n0, const int32_t* tgt,
                             hipStream_t s) {
  hipLaunchKernelGGL(head_stats_kernel, dim3(T_, ceil_div(C, CHUNK)), dim3(NT), 0, s, r, part, lm, ld, T_, C, n0, tgt);
  return hipGetLastError();
}
// (16 rows per workgroup read 64 or 128 bytes at a time; where they would leave most of the chip idle
// a workgroup takes one)
template <typename P>
hipError_t launch_head_join(const HeadRows& r, const P* part, int groups, int T_, const int32_t* tgt, bool first, bool last,
                            const HeadOut& out, hipStream_t s) {
  if (T_ >= 1024) hipLaunchKernelGGL((head_join_kernel<16, P>), dim3(ceil_div(T_, 16)), dim3(NT), 0, s, r, part, groups, T_, tgt, first, last, out);
  else hipLaunchKernelGGL((head_join_kernel<1, P>), dim3(T_), dim3(NT), 0, s, r, part, groups, T_, tgt, first, last, out);
  return hipGetLastError();
}
template hipError_t launch_head_join<float>(const HeadRows&, const float*, int, int, const int32_t*, bool, bool, const HeadOut&, hipStream_t);
template hipError_t launch_head_join<double>(const HeadRows&, const double*, int, int, const int32_t*, bool, bool, const HeadOut&, hipStream_t);
template <typename T>
hipError_t launch_head_dlogits(PairT<T> o, const HeadRows& r, const float* lm, const float* ld, int T_, int Tp, int C, int n0,
                               const int32_t* tgt, hipStream_t s) {
  hipLaunchKernelGGL(head_dlogits_kernel<T>, dim3(Tp, ceil_div(C, CHUNK)), dim3(NT), 0, s, o, r, lm, ld, T_, C, n0, tgt);
  return hipGetLastError();
}
template hipError_t launch_head_dlogits<float>(PairT<float>, const HeadRows&, const float*, const float*, int, int, int, int,
                                               const int32_t*, hipStream_t);
template hipError_t launch_head_dlogits<bf16_t>(PairT<bf16_t>, const HeadRows&, const float*, const float*, int, int, int, int,
                                                const int32_t*, hipStream_t);
hipError_t launch_head_copy(const HeadCopy& c, hipStream_t s) {
  hipLaunchKernelGGL(head_copy_kernel, dim3(std::min(c.Tp, 2048)), dim3(NT), 0, s, c);
  return hipGetLastError();
}
hipError_t launch_head_round(PairT<bf16_t> o, int64_t ldo, const float* m, const float* d, int T_, int dm, hipStream_t s) {
  hipLaunchKernelGGL(head_round_kernel, dim3(T_), dim3(NT), 0, s, o, ldo, m, d, dm);
  return hipGetLastError();
}

}  // namespace fdh
