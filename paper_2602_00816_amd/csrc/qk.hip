// Queries and keys between the projection and attention: per-head RMSNorm and
// the position rotation in one pass, forward and backward, in the pair form
// (mean m and half difference d of the two points theta +- eps v).
//
// With the pair product (a o b).m = a.m b.m + a.d b.d, (a o b).d = a.m b.d + a.d b.m
// (exact, and free of differences of nearly equal values), per token and head
// of n elements, e the norm's epsilon:
//   forward   S+- = mean((x.m +- x.d)^2) + e,  b = 2 mean(x.m x.d) = (S+ - S-) / 2,
//             r+- = S+-^(-1/2),  r.m = (r+ + r-) / 2,
//             rho = r.d / r.m = (r+ - r-) / (r+ + r-) = -2 b (r+ r-)^2 / (r+ + r-)^2,
//             u = x o r = (x o (1, rho)) r.m,  z = u o g  (g = (theta_g, eps v_g)),  y = R z;
//   backward  dz = R^T dy,  dg = sum over tokens and heads of dz o u,  du = dz o g,
//             c = mean(u o du) = r o mean(x o du),  dx = r o (du - u o c).
// R turns pair i (elements i and i + n/2) by base^(-2i/n) times the token's
// position along the axis of pair i; without a norm y = R x and dx = R^T dy.
//
// The sums over a head and all that is formed from them once per head are fp64
// (no overflow or underflow; rho in place of r.d keeps the elements' arithmetic in
// the normal range, too, up to |x| of 1e37), the elements fp32, each output rounded
// once to its type.  A head that holds a NaN or an infinity gives NaN in
// all its elements, other heads are not touched by it.
//
// Memory-bound: 8 bytes per bf16 element forward, 16 backward, against some 25 and 50
// vector instructions.
#include "kernels.h"

#include <algorithm>

namespace fdh {

namespace {

constexpr int NT = 256, NWAVE = NT / 64;

// ---- vectors of V elements ------------------------------------------------------
template <typename T, int V>
__device__ inline void load(float (&x)[V], const T* p) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p + e);
      x[e] = v.x; x[e + 1] = v.y; x[e + 2] = v.z; x[e + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; e += 4) {
      const uint2 v = *reinterpret_cast<const uint2*>(p + e);
      x[e] = bf16_to_f32((bf16_t)(v.x & 0xFFFF));
      x[e + 1] = bf16_to_f32((bf16_t)(v.x >> 16));
      x[e + 2] = bf16_to_f32((bf16_t)(v.y & 0xFFFF));
      x[e + 3] = bf16_to_f32((bf16_t)(v.y >> 16));
    }
  }
}
template <typename T, int V>
__device__ inline void store(T* p, const float (&x)[V]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < V; e += 4) *reinterpret_cast<float4*>(p + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
  } else {
#pragma unroll
    for (int e = 0; e < V; e += 4)
      *reinterpret_cast<uint2*>(p + e) = make_uint2((uint32_t)f32_to_bf16(x[e]) | ((uint32_t)f32_to_bf16(x[e + 1]) << 16),
                                                    (uint32_t)f32_to_bf16(x[e + 2]) | ((uint32_t)f32_to_bf16(x[e + 3]) << 16));
  }
}

// ---- sums over aligned groups of G lanes ------------------------------------------
// each step adds the partner group's sum: lane xor 1 and xor 2 by quad
// permutations, then the mirrored half row (8 lanes) and row (16 lanes), whose
// lanes all hold the same sum by then, then lane xor 16 through LDS hardware
template <int CTRL>
__device__ inline double dpp(double x) {
  const long long b = __builtin_bit_cast(long long, x);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xF, 0xF, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xF, 0xF, false);
  return __builtin_bit_cast(double, ((long long)hi << 32) | (unsigned)lo);
}
template <int G>
__device__ inline double group_sum(double x) {
  if constexpr (G >= 2) x += dpp<0xB1>(x);    // quad_perm [1,0,3,2]
  if constexpr (G >= 4) x += dpp<0x4E>(x);    // quad_perm [2,3,0,1]
  if constexpr (G >= 8) x += dpp<0x141>(x);   // row_half_mirror
  if constexpr (G >= 16) x += dpp<0x140>(x);  // row_mirror
  if constexpr (G >= 32) x += __shfl_xor(x, 16, 64);
  return x;
}

// ---- per-head statistics ------------------------------------------------------------
// 1 / sqrt(x) and 1 / x: the hardware's approximation and one Newton step (relative error below 2^-44)
__device__ inline double rsqrt_nr(double x) {
  const double y = __builtin_amdgcn_rsq(x);
  return fma(0.5 * fma(-x * y, y, 1.0), y, y);
}
__device__ inline double rcp_nr(double x) {
  const double y = __builtin_amdgcn_rcp(x);
  return fma(fma(-x, y, 1.0), y, y);
}
// r.m and rho = r.d / r.m of the head from sum (m + d)^2, sum (m - d)^2, sum m d
struct Rms { double m, rho; };
__device__ inline Rms rms_pair(double sp, double sm, double md, double inv_n, double neps) {
  const double rp = rsqrt_nr(fma(sp, inv_n, neps)), rm = rsqrt_nr(fma(sm, inv_n, neps));
  const double s = rp + rm, p = rp * rm * rcp_nr(s);
  return {0.5 * s, -4.0 * md * inv_n * p * p};
}

// ---- angles --------------------------------------------------------------------
// cos and sin of 2 pi f pos in fp64, rounded once.  The product is taken to
// the nearest quarter turn with its rounding error kept (fma), so the angle is
// good to 2^-53 relative in f alone, for every int32 position; the rest,
// |theta| <= pi / 4, goes through the Taylor series up to theta^12 (remainders
// below 1e-11).
__device__ inline void cos_sin(int pos, double f, float& c, float& s) {
  const double p = (double)pos, t = p * f, err = fma(p, f, -t);
  const double q = rint(4.0 * t);
  const double r = (4.0 * t - q) + 4.0 * err;
  const double th = r * 1.5707963267948966192, w = th * th;
  double sn = -1.0 / 39916800.0, cn = 1.0 / 479001600.0;
  sn = fma(sn, w, 1.0 / 362880.0);
  cn = fma(cn, w, -1.0 / 3628800.0);
  sn = fma(sn, w, -1.0 / 5040.0);
  cn = fma(cn, w, 1.0 / 40320.0);
  sn = fma(sn, w, 1.0 / 120.0);
  cn = fma(cn, w, -1.0 / 720.0);
  sn = fma(sn, w, -1.0 / 6.0);
  cn = fma(cn, w, 1.0 / 24.0);
  sn = fma(sn * w, th, th);
  cn = fma(cn, w, -0.5);
  cn = fma(cn, w, 1.0);
  const int k = (int)q & 3;   // |4 t| < 2^31: f <= 1 / (2 pi)
  const float fs = (float)sn, fc = (float)cn;
  const float a = k & 1 ? fs : fc, b = k & 1 ? fc : fs;
  c = (k == 1 || k == 2) ? -a : a;
  s = k >= 2 ? -b : b;
}

template <int V>
__device__ inline void token_angles(const QkArgs& a, int t, int i0, bool on, float (&c)[V], float (&s)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    c[e] = 1.f;
    s[e] = 0.f;
  }
  if (!on) return;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    const int pos = a.pos ? a.pos[(int64_t)a.rot.axis[i0 + e] * a.T + t] : t % a.S;
    cos_sin(pos, a.rot.freq[i0 + e], c[e], s[e]);
  }
}

// gains of the lane's elements (first and second half of the head)
template <typename T, int V>
__device__ inline void load_gains(const T* g, const float* v, double eps, int i0, int half, bool on, float (&gm)[2 * V],
                                  float (&gd)[2 * V]) {
#pragma unroll
  for (int e = 0; e < 2 * V; ++e) {
    const int j = i0 + (e < V ? e : half + e - V);
    gm[e] = on ? ldf(g, j) : 0.f;
    gd[e] = on && v ? (float)(eps * (double)v[j]) : 0.f;
  }
}

// Work split: a wavefront takes 64 / G heads of one token at a time (a unit), G
// lanes per head, lane g of a head its pairs g V .. g V + V - 1, so that a lane
// turns pairs it holds itself.  G is the power of two from half / V up; lanes past
// the head hold zeros.  The units of the query heads, then those of the key heads
// are dealt to wavefronts in runs of `per` (cosines and gains are kept along a
// run); the last workgroups move the value columns.
struct Unit {
  int seg, t, c, left;
};
template <int G>
__device__ inline bool first_unit(const QkArgs& a, const QkSplit& w, Unit& u) {
  u.seg = (int)blockIdx.x >= w.blocks[0] ? 1 : 0;
  const int b = blockIdx.x - (u.seg ? w.blocks[0] : 0);
  const int64_t first = ((int64_t)b * NWAVE + (threadIdx.x >> 6)) * w.per[u.seg];
  const int64_t units = (int64_t)a.T * w.chunks[u.seg];
  u.left = (int)max((int64_t)0, min((int64_t)w.per[u.seg], units - first));
  u.t = u.left ? (int)(first / w.chunks[u.seg]) : 0;
  u.c = u.left ? (int)(first % w.chunks[u.seg]) : 0;
  return u.left > 0;
}

// value columns: V = 8 elements per step
template <typename T, typename TI>
__device__ inline void move_values(const QkArgs& a, const TI* im, const TI* id, int64_t ldi, T* om, T* od, int64_t ldo,
                                   int block, int nblocks) {
  const int c0 = (a.Hq + a.Hk) * a.dh, n8 = a.Hk * a.dh / 8;
  const int64_t n = (int64_t)a.T * n8;
  for (int64_t i = (int64_t)block * NT + threadIdx.x; i < n; i += (int64_t)nblocks * NT) {
    const int64_t t = i / n8;
    const int c = c0 + 8 * (int)(i % n8);
    float x[8], y[8];
    load<TI, 8>(x, im + t * ldi + c);
    load<TI, 8>(y, id + t * ldi + c);
    store<T, 8>(om + t * ldo + c, x);
    store<T, 8>(od + t * ldo + c, y);
  }
}

template <typename T, int V, int G, bool NORM>
__global__ __launch_bounds__(NT) void qk_fwd_kernel(QkArgs a, QkSplit w) {
  const T *xm = (const T*)a.x_m, *xd = (const T*)a.x_d;
  T *ym = (T*)a.y_m, *yd = (T*)a.y_d;
  const int nqk = w.blocks[0] + w.blocks[1];
  if ((int)blockIdx.x >= nqk) {
    move_values<T, T>(a, xm, xd, a.ldx, ym, yd, a.ldy, blockIdx.x - nqk, w.vblocks);
    return;
  }
  Unit u;
  if (!first_unit<G>(a, w, u)) return;
  const int lane = threadIdx.x & 63, half = a.dh / 2;
  const int i0 = (lane & (G - 1)) * V;
  const bool on = i0 < half;
  const int H = u.seg ? a.Hk : a.Hq, col0 = u.seg ? a.Hq * a.dh : 0;
  float gm[2 * V], gd[2 * V], c[V], s[V];
  if constexpr (NORM) load_gains<T, V>((const T*)(u.seg ? a.gk : a.gq), u.seg ? a.vk : a.vq, a.eps, i0, half, on, gm, gd);
  token_angles<V>(a, u.t, i0, on, c, s);
  while (true) {
    const int head = u.c * (64 / G) + lane / G;
    const bool ok = on && head < H;
    float m[2 * V], d[2 * V];
    {
      float l[V], h[V];
      const int64_t o = (int64_t)u.t * a.ldx + col0 + head * a.dh + i0;
#pragma unroll
      for (int e = 0; e < V; ++e) l[e] = h[e] = 0.f;
      if (ok) {
        load<T, V>(l, xm + o);
        load<T, V>(h, xm + o + half);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        m[e] = l[e];
        m[V + e] = h[e];
        l[e] = h[e] = 0.f;
      }
      if (ok) {
        load<T, V>(l, xd + o);
        load<T, V>(h, xd + o + half);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        d[e] = l[e];
        d[V + e] = h[e];
      }
    }
    if constexpr (NORM) {
      double sp = 0.0, sm = 0.0, md = 0.0;
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) {
        const double p = (double)m[e] + (double)d[e], q = (double)m[e] - (double)d[e];
        sp = fma(p, p, sp);
        sm = fma(q, q, sm);
        md = fma((double)m[e], (double)d[e], md);
      }
      const Rms r = rms_pair(group_sum<G>(sp), group_sum<G>(sm), group_sum<G>(md), a.inv_n, a.neps);
      const float rm = (float)r.m, rho = (float)r.rho;
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) {
        const float um = (m[e] + d[e] * rho) * rm, ud = (m[e] * rho + d[e]) * rm;
        m[e] = um * gm[e] + ud * gd[e];
        d[e] = um * gd[e] + ud * gm[e];
      }
    }
    if (ok) {
      const int64_t o = (int64_t)u.t * a.ldy + col0 + head * a.dh + i0;
      float l[V], h[V];
#pragma unroll
      for (int e = 0; e < V; ++e) {
        l[e] = m[e] * c[e] - m[V + e] * s[e];
        h[e] = m[V + e] * c[e] + m[e] * s[e];
      }
      store<T, V>(ym + o, l);
      store<T, V>(ym + o + half, h);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        l[e] = d[e] * c[e] - d[V + e] * s[e];
        h[e] = d[V + e] * c[e] + d[e] * s[e];
      }
      store<T, V>(yd + o, l);
      store<T, V>(yd + o + half, h);
    }
    if (--u.left == 0) break;
    if (++u.c == w.chunks[u.seg]) {
      u.c = 0;
      ++u.t;
      token_angles<V>(a, u.t, i0, on, c, s);
    }
  }
}

// Backward.  Every workgroup leaves its sum of the gain gradient's half
// difference (fp64, fixed order) as row blockIdx.x of part.
template <typename T, int V, int G, bool NORM>
__global__ __launch_bounds__(NT) void qk_bwd_kernel(QkArgs a, QkSplit w) {
  const T *xm = (const T*)a.x_m, *xd = (const T*)a.x_d;
  T *ym = (T*)a.y_m, *yd = (T*)a.y_d;
  const int nqk = w.blocks[0] + w.blocks[1];
  if ((int)blockIdx.x >= nqk) {
    move_values<T, float>(a, a.dy_m, a.dy_d, a.lddy, ym, yd, a.ldy, blockIdx.x - nqk, w.vblocks);
    return;
  }
  __shared__ double sh[NORM ? NWAVE * 2 * V * G : 1];
  Unit u;
  const bool any = first_unit<G>(a, w, u);
  if (!NORM && !any) return;
  const int lane = threadIdx.x & 63, half = a.dh / 2;
  const int i0 = (lane & (G - 1)) * V;
  const bool on = i0 < half;
  const int H = u.seg ? a.Hk : a.Hq, col0 = u.seg ? a.Hq * a.dh : 0;
  float gm[2 * V], gd[2 * V], c[V], s[V];
  double acc[2 * V];
  if constexpr (NORM) {
    load_gains<T, V>((const T*)(u.seg ? a.gk : a.gq), u.seg ? a.vk : a.vq, a.eps, i0, half, on, gm, gd);
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) acc[e] = 0.0;
  }
  if (any) token_angles<V>(a, u.t, i0, on, c, s);
  while (u.left > 0) {
    const int head = u.c * (64 / G) + lane / G;
    const bool ok = on && head < H;
    float zm[2 * V], zd[2 * V], m[2 * V], d[2 * V];
    {
      const int64_t o = (int64_t)u.t * a.lddy + col0 + head * a.dh + i0;
      float l[V], h[V];
#pragma unroll
      for (int ch = 0; ch < 2; ++ch) {
        const float* g = ch ? a.dy_d : a.dy_m;
        float* z = ch ? zd : zm;
#pragma unroll
        for (int e = 0; e < V; ++e) l[e] = h[e] = 0.f;
        if (ok) {
          load<float, V>(l, g + o);
          load<float, V>(h, g + o + half);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
          z[e] = l[e] * c[e] + h[e] * s[e];
          z[V + e] = h[e] * c[e] - l[e] * s[e];
        }
      }
    }
    if constexpr (NORM) {
      const int64_t o = (int64_t)u.t * a.ldx + col0 + head * a.dh + i0;
      float l[V], h[V];
#pragma unroll
      for (int ch = 0; ch < 2; ++ch) {
        const T* x = ch ? xd : xm;
        float* q = ch ? d : m;
#pragma unroll
        for (int e = 0; e < V; ++e) l[e] = h[e] = 0.f;
        if (ok) {
          load<T, V>(l, x + o);
          load<T, V>(h, x + o + half);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) {
          q[e] = l[e];
          q[V + e] = h[e];
        }
      }
      double sp = 0.0, sm = 0.0, md = 0.0;
      double xum = 0.0, xud = 0.0;   // of x o du
      float dum[2 * V], dud[2 * V];
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) {
        dum[e] = zm[e] * gm[e] + zd[e] * gd[e];
        dud[e] = zm[e] * gd[e] + zd[e] * gm[e];
        const double x = m[e], y = d[e], p = x + y, q = x - y;
        sp = fma(p, p, sp);
        sm = fma(q, q, sm);
        md = fma(x, y, md);
        xum = fma(x, (double)dum[e], fma(y, (double)dud[e], xum));
        xud = fma(x, (double)dud[e], fma(y, (double)dum[e], xud));
      }
      const Rms r = rms_pair(group_sum<G>(sp), group_sum<G>(sm), group_sum<G>(md), a.inv_n, a.neps);
      const double rn = r.m * a.inv_n, wm = group_sum<G>(xum) * rn, wd = group_sum<G>(xud) * rn;
      const float rm = (float)r.m, rho = (float)r.rho;
      const float cm = (float)fma(wd, r.rho, wm), cd = (float)fma(wm, r.rho, wd);
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) {
        const float um = (m[e] + d[e] * rho) * rm, ud = (m[e] * rho + d[e]) * rm;
        acc[e] += (double)(zm[e] * ud + zd[e] * um);
        const float tm = dum[e] - (um * cm + ud * cd), td = dud[e] - (um * cd + ud * cm);
        zm[e] = (tm + td * rho) * rm;
        zd[e] = (tm * rho + td) * rm;
      }
    }
    if (ok) {
      const int64_t o = (int64_t)u.t * a.ldy + col0 + head * a.dh + i0;
      float l[V], h[V];
#pragma unroll
      for (int ch = 0; ch < 2; ++ch) {
        const float* z = ch ? zd : zm;
        T* y = ch ? yd : ym;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          l[e] = z[e];
          h[e] = z[V + e];
        }
        store<T, V>(y + o, l);
        store<T, V>(y + o + half, h);
      }
    }
    if (--u.left == 0) break;
    if (++u.c == w.chunks[u.seg]) {
      u.c = 0;
      ++u.t;
      token_angles<V>(a, u.t, i0, on, c, s);
    }
  }
  if constexpr (NORM) {
    // over the wavefront's head groups, then over the wavefronts
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) {
#pragma unroll
      for (int o = G; o < 64; o <<= 1) acc[e] += __shfl_xor(acc[e], o, 64);
      if (lane < G) sh[((threadIdx.x >> 6) * 2 * V + e) * G + lane] = acc[e];
    }
    __syncthreads();
    for (int j = threadIdx.x; j < 2 * V * G; j += NT) {
      double t = 0.0;
#pragma unroll
      for (int v = 0; v < NWAVE; ++v) t += sh[v * 2 * V * G + j];
      // entry j: element e = j / G of lane j % G
      const int e = j / G, i = (j % G) * V;
      if (i < half) a.part[(int64_t)blockIdx.x * a.dh + i + (e < V ? e : half + e - V)] = t;
    }
  }
}

// out[seg][j] (+)= scale * sum of the segment's rows of part: 16 columns and 64
// row groups per workgroup, added in a fixed order
__global__ __launch_bounds__(1024) void qk_gain_kernel(const double* part, QkSplit w, int dh, double scale, float* dgq,
                                                       float* dgk, bool acc) {
  __shared__ double sh[16][16];
  const int seg = blockIdx.y, cl = threadIdx.x & 15, j = blockIdx.x * 16 + cl;
  const int r0 = seg ? w.blocks[0] : 0, r1 = r0 + w.blocks[seg];
  double t = 0.0;
  if (j < dh)
    for (int r = r0 + (threadIdx.x >> 4); r < r1; r += 64) t += part[(int64_t)r * dh + j];
  t += __shfl_xor(t, 16, 64);
  t += __shfl_xor(t, 32, 64);
  if ((threadIdx.x & 63) < 16) sh[threadIdx.x >> 6][cl] = t;
  __syncthreads();
  if (threadIdx.x >= 16 || j >= dh) return;
  t = 0.0;
#pragma unroll
  for (int v = 0; v < 16; ++v) t += sh[v][cl];
  t *= scale;
  float* out = (seg ? dgk : dgq) + j;
  *out = acc ? (float)((double)*out + t) : (float)t;
}

// lanes per head
int group_lanes(int dh) {
  int g = 1;
  while (4 * g < dh / 2) g *= 2;
  return g;
}

QkSplit split(const QkArgs& a, bool bwd, bool values) {
  QkSplit w{};
  const int hpw = 64 / group_lanes(a.dh);
  for (int k = 0; k < 2; ++k) {
    w.chunks[k] = (int)ceil_div(k ? a.Hk : a.Hq, hpw);
    const int64_t units = (int64_t)a.T * w.chunks[k];
    const int64_t waves = (int64_t)NWAVE * (bwd ? QK_BWD_BLOCKS : 4096);
    w.per[k] = (int)std::max<int64_t>(1, (units + waves - 1) / waves);
    w.blocks[k] = (int)((units + (int64_t)NWAVE * w.per[k] - 1) / ((int64_t)NWAVE * w.per[k]));
  }
  if (values) w.vblocks = (int)std::min<int64_t>(1024, ((int64_t)a.T * (a.Hk * a.dh / 8) + NT - 1) / NT);
  return w;
}

template <typename T, bool BWD, bool NORM>
hipError_t dispatch(const QkArgs& a, const QkSplit& w, hipStream_t s) {
  const dim3 g(w.blocks[0] + w.blocks[1] + w.vblocks);
  if (g.x == 0) return hipSuccess;
#define QK(G)                                                                                      \
  case G:                                                                                          \
    if constexpr (BWD) hipLaunchKernelGGL((qk_bwd_kernel<T, 4, G, NORM>), g, dim3(NT), 0, s, a, w); \
    else hipLaunchKernelGGL((qk_fwd_kernel<T, 4, G, NORM>), g, dim3(NT), 0, s, a, w);               \
    break
  switch (group_lanes(a.dh)) {
    QK(1);
    QK(2);
    QK(4);
    QK(8);
    QK(16);
    QK(32);
    default: return hipErrorInvalidValue;
  }
#undef QK
  return hipGetLastError();
}

}  // namespace

size_t qk_scratch_bytes(int64_t T_, int Hq, int Hk, int dh) {
  // (the workgroups of split(), which takes as many as this or fewer)
  const int hpw = 64 / group_lanes(dh);
  int64_t rows = 0;
  for (int H : {Hq, Hk}) rows += std::min<int64_t>(QK_BWD_BLOCKS, (T_ * ceil_div(H, hpw) + NWAVE - 1) / NWAVE);
  return (size_t)rows * dh * sizeof(double);
}

template <typename T>
hipError_t launch_qk_fwd(QkArgs a, hipStream_t s) {
  if (a.dh % 8 || a.dh > QK_MAX_DH || a.T < 0) return hipErrorInvalidValue;
  a.inv_n = 1.0 / a.dh;
  const QkSplit w = split(a, false, a.x_m != a.y_m);
  return a.gq ? dispatch<T, false, true>(a, w, s) : dispatch<T, false, false>(a, w, s);
}

template <typename T>
hipError_t launch_qk_bwd(QkArgs a, float* dgq, float* dgk, bool acc, hipStream_t s) {
  if (a.dh % 8 || a.dh > QK_MAX_DH || a.T < 0) return hipErrorInvalidValue;
  a.inv_n = 1.0 / a.dh;
  const QkSplit w = split(a, true, true);
  if (!a.gq) return dispatch<T, true, false>(a, w, s);
  const hipError_t r = dispatch<T, true, true>(a, w, s);
  if (r != hipSuccess) return r;
  hipLaunchKernelGGL(qk_gain_kernel, dim3(ceil_div(a.dh, 16), 2), dim3(1024), 0, s, a.part, w, a.dh, 1.0 / a.eps, dgq, dgk, acc);
  return hipGetLastError();
}

template hipError_t launch_qk_fwd<float>(QkArgs, hipStream_t);
template hipError_t launch_qk_fwd<bf16_t>(QkArgs, hipStream_t);
template hipError_t launch_qk_bwd<float>(QkArgs, float*, float*, bool, hipStream_t);
template hipError_t launch_qk_bwd<bf16_t>(QkArgs, float*, float*, bool, hipStream_t);

}  // namespace fdh
