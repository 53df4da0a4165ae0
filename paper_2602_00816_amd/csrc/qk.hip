// Queries and keys between the projection and attention: per-head RMSNorm and
// the position rotation in one pass, forward and backward, in the pair form
// (mean m and half difference d of the two points theta +- eps v).
//
// With the pair product (a o b).m = a.m b.m + a.d b.d, (a o b).d = a.m b.d + a.d b.m
// (exact, and free of differences of nearly equal values where the two points are of like
// size), per token and head of n elements, e the norm's epsilon:
//   forward   S+- = mean((x.m +- x.d)^2) + e,  b = 2 mean(x.m x.d) = (S+ - S-) / 2,
//             r+- = S+-^(-1/2),  r.m = (r+ + r-) / 2,
//             rho = r.d / r.m = (r+ - r-) / (r+ + r-) = -2 b (r+ r-)^2 / (r+ + r-)^2,
//             u = x o r = (x o (1, rho)) r.m,  z = u o g  (g = (theta_g, eps v_g)),  y = R z;
//   backward  dz = R^T dy,  dg = sum over tokens and heads of dz o u,  du = dz o g,
//             c = mean(u o du) = r o mean(x o du),  dx = r o (du - u o c).
// R turns pair i (elements i and i + n/2) by base^(-2i/n) times the token's
// position along the axis of pair i; without a norm y = R x and dx = R^T dy.
//
// Heads with a small point, that is x.d close to x.m (sigma = 1, S- small) or to -x.m
// (sigma = -1, S+ small): there the smaller S is itself a difference, and u's terms are larger
// than u+- by up to half the ratio of the r's.  From a ratio of 8 on (up to it, 4.5 times) the
// smaller S is the mean of (x.m - sigma x.d)^2, and forward
//   u = (x.m - sigma x.d + kappa x.d, x.d - sigma x.m + kappa x.m) r.m,
//   kappa = sigma + rho = 2 sigma r / (r+ + r-),  r the smaller of the two,
// whose terms are no larger than u+- (other heads: sigma = 0).  Backward all of it is done at the
// two points, whose gradients may differ as much: u+- = (x.m +- x.d) r+-, du+- = dz+- g+-,
// dx+- = r+- (du+- - u+- mean(u+- du+-)), then the mean and half difference of the two.
// (Elsewhere the points would lose a half difference that is small.)
//
// The sums behind r and all that is formed from them once per head are fp64, with
// S+- = mean(x.m^2 + x.d^2) +- 2 mean(x.m x.d) + e (no overflow or underflow; rho in
// place of r.d keeps the elements' arithmetic in the normal range, too, up to |x| of
// 1e37, kappa up to 1e35 for e = 1e-5); the elements, and c, whose terms are bounded by du, are fp32; the gains' sums
// are fp64; each output is rounded once to its type.  A head that holds a NaN or an
// infinity gives NaN in all its elements, other heads are not touched by it.
//
// Memory-bound: 8 bytes per bf16 element forward and 16 backward against some 35 and 45
// vector instructions.  One layer of 16 + 16 + 16 heads of 128 at 8192 tokens, bf16:
// forward 76 us (403 MB, 5.3 TB/s), backward 140 us with the gains' sums (738 MB, 5.3 TB/s);
// rotation alone of 32 + 8 + 8 heads at 16384 tokens 144 us (805 MB, 5.6 TB/s).  A plain
// copy of as many bytes runs at 6.0 TB/s; the vector units are busy for less than half the time.
#include "kernels.h"

#include <algorithm>

namespace fdh {

namespace {

// Threads per workgroup.  Forward: 256, but 128 where the bf16 norm's registers and angles
// leave fewer wavefronts ready (2^26 elements in 4 + 1 + 1 heads of 128: 117 us against 127, 14 + 2 + 2 of
// 64: 111 against 115, 32 + 8 + 8 of 128: 97 against 98; rotation alone, of 64: 110 against 93).
constexpr int fwd_threads(bool bf16, bool norm) { return bf16 && norm ? 128 : 256; }
// Most wavefronts of a backward with gains, as each workgroup leaves a row of gain sums: as many as are
// resident at once, four per SIMD, in kernels of up to 128 registers (the layer above: 140 us
// with 4096, 143 with 8192, 152 with 32768).  Those are all but the fp32 ones of 2 to 16 lanes per head where tokens share a
// wavefront: at 129 registers and 512 threads two per SIMD are resident, and the grid takes two rounds.
constexpr int BWD_WAVES = 4096;
// 32 lanes per head (wider than 128): a workgroup of 1024 threads holds the kernel to 128 registers and so
// four wavefronts per SIMD.  fp32 spills 24 bytes per lane for it (36 where tokens share a wavefront):
// 16 + 8 + 8 heads of 144, 164 us against 220 with 512 threads, of 192, 149 against 178; bf16 spills
// nothing: of 144, 255 against 273, of 192 and 256 within 2%.  With 16 lanes the two are within 2%.
constexpr int bwd_threads(int g) { return g == 32 ? 1024 : 512; }

// ---- vectors of V elements ------------------------------------------------------
// as they lie in memory (4 V or 2 V bytes), so that loads can be held in flight
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x3 __attribute__((ext_vector_type(3), aligned(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <typename T, int V>
struct Raw {
  static constexpr int N = V * sizeof(T) / 4;
  uint32_t w[N];
};
// STREAM: nontemporal accesses, in the backward, which reads dy and x for the last time: the
// layer above takes 140 us with them, 154 with the loads alone; 32 + 8 + 8 heads of 128 in fp32,
// 5456 tokens, 143 and 155.  In the forward the loads gain nothing (77 us against 76).  (A store whose vector is
// filled element by element, or through a dependent type, loses the hint in hipcc.)
__device__ inline u32x2 words(const uint32_t* w, u32x2) { return {w[0], w[1]}; }
__device__ inline u32x3 words(const uint32_t* w, u32x3) { return {w[0], w[1], w[2]}; }
__device__ inline u32x4 words(const uint32_t* w, u32x4) { return {w[0], w[1], w[2], w[3]}; }
template <typename W, int K, int N, bool STREAM>
__device__ inline void load_words(uint32_t (&w)[N], const void* p) {
#pragma unroll
  for (int i = 0; i < N; i += K) {
    const W* q = reinterpret_cast<const W*>((const uint32_t*)p + i);
    const W v = STREAM ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
    for (int k = 0; k < K; ++k) w[i + k] = v[k];
  }
}
template <typename W, int K, int N, bool STREAM>
__device__ inline void store_words(const uint32_t (&w)[N], void* p) {
#pragma unroll
  for (int i = 0; i < N; i += K) {
    W* q = reinterpret_cast<W*>((uint32_t*)p + i);
    const W v = words(w + i, W{});
    if constexpr (STREAM) __builtin_nontemporal_store(v, q);
    else *q = v;
  }
}
template <typename T, int V, bool STREAM = false>
__device__ inline void load(Raw<T, V>& r, const T* p) {
  constexpr int N = Raw<T, V>::N;
  if constexpr (N % 4 == 0) load_words<u32x4, 4, N, STREAM>(r.w, p);
  else if constexpr (N % 2 == 0) load_words<u32x2, 2, N, STREAM>(r.w, p);
  else load_words<u32x3, 3, N, STREAM>(r.w, p);
}
template <typename T, int V>
__device__ inline float get(const Raw<T, V>& r, int e) {
  if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, r.w[e]);
  else return __builtin_bit_cast(float, e & 1 ? r.w[e / 2] & 0xFFFF0000u : r.w[e / 2] << 16);
}
template <typename T, int V, bool STREAM = false>
__device__ inline void store(T* p, const float* x) {
  Raw<T, V> r;
  constexpr int N = Raw<T, V>::N;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (sizeof(T) == 4) r.w[i] = __builtin_bit_cast(uint32_t, x[i]);
    else r.w[i] = (uint32_t)f32_to_bf16(x[2 * i]) | ((uint32_t)f32_to_bf16(x[2 * i + 1]) << 16);
  }
  if constexpr (N % 4 == 0) store_words<u32x4, 4, N, STREAM>(r.w, p);
  else if constexpr (N % 2 == 0) store_words<u32x2, 2, N, STREAM>(r.w, p);
  else store_words<u32x3, 3, N, STREAM>(r.w, p);
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

template <int CTRL>
__device__ inline float dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xF, 0xF, false));
}
template <int G>
__device__ inline float group_sum(float x) {
  if constexpr (G >= 2) x += dpp<0xB1>(x);
  if constexpr (G >= 4) x += dpp<0x4E>(x);
  if constexpr (G >= 8) x += dpp<0x141>(x);
  if constexpr (G >= 16) x += dpp<0x140>(x);
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
// r.m and rho = r.d / r.m of the head from sum (m^2 + d^2) and sum m d, the smaller r, and whether the
// other one, of a small point, is more than 8 times that: |rho| = |r+ - r-| / (r+ + r-) > 7/9.
// (A NaN is no small point.)
struct Rms {
  double m, rho, large;   // (large: the larger point's, the smaller r)
  bool small;
};
__device__ inline Rms rms_pair(double sq, double md, double inv_n, double neps) {
  const double b = 2.0 * md, p = sq + b, q = sq - b;   // sums of (m + d)^2, (m - d)^2
  const double rp = rsqrt_nr(fma(p < 0.0 ? 0.0 : p, inv_n, neps)), rn = rsqrt_nr(fma(q < 0.0 ? 0.0 : q, inv_n, neps));
  const double s = rp + rn, x = rp * rn * rcp_nr(s), rho = -2.0 * b * inv_n * x * x;
  return {0.5 * s, rho, rho < 0.0 ? rp : rn, fabs(rho) > 7.0 / 9.0};
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

// Angles of the tokens t0 .. t0 + ntok - 1 that a wavefront's heads belong to, formed
// by the lanes in turn, to LDS (cs: the wavefront's own part, whose accesses keep
// their order); every lane then takes those of its token (tok after t0) and its own
// V pairs.  The heads of a token share the 45 or so fp64 operations of an angle; formed
// by every lane for its own pairs, they took a third of the forward's time.
template <int V, bool GROUP>
__device__ inline void token_angles(const QkArgs& a, const QkSplit& w, int t0, int ntok, int tok, int i0, float2* cs,
                                    float (&c)[V], float (&s)[V]) {
  const int half = a.dh / 2, s0 = a.pos ? 0 : t0 % a.S;
  // (what the lanes read of the last token's angles stays before this)
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int i = threadIdx.x & 63; i < (GROUP ? ntok * half : half); i += 64) {
    const int k = GROUP ? i * w.rhalf >> 16 : 0, j = i - k * half;   // i / half, i % half
    int pos;
    if (a.pos) {
      pos = a.pos[(int64_t)a.rot.axis[j] * a.T + (GROUP ? min(t0 + k, a.T - 1) : t0)];
    } else {
      pos = s0 + k;
      if (GROUP && pos >= a.S) pos %= a.S;
    }
    float x, y;
    cos_sin(pos, a.rot.freq[j], x, y);
    cs[i] = make_float2(x, y);
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const float2* q = cs + (GROUP ? tok * half : 0) + i0;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    c[e] = q[e].x;
    s[e] = q[e].y;
  }
}

// offset of row t (both below 2^32)
__device__ inline int64_t row(int t, int64_t ld) { return (int64_t)((uint64_t)(uint32_t)t * (uint32_t)ld); }

// gains of the lane's elements (first and second half of the head), as a pair
template <typename T, int V>
__device__ inline void lane_gains(const QkArgs& a, int seg, int i0, float (&gm)[2 * V], float (&gd)[2 * V]) {
  const T* g = (const T*)(seg ? a.gk : a.gq);
  const float* v = seg ? a.vk : a.vq;
  const int half = a.dh / 2;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = i0 + (h ? half : 0);
    if (a.gvec) {
      Raw<T, V> r;
      load<T, V>(r, g + j);
#pragma unroll
      for (int e = 0; e < V; ++e) gm[h * V + e] = get<T, V>(r, e);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) gm[h * V + e] = ldf(g, j + e);
    }
    if (!v) {
#pragma unroll
      for (int e = 0; e < V; ++e) gd[h * V + e] = 0.f;
    } else if (a.gvec) {
      Raw<float, V> r;
      load<float, V>(r, v + j);
#pragma unroll
      for (int e = 0; e < V; ++e) gd[h * V + e] = (float)(a.eps * (double)get<float, V>(r, e));
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) gd[h * V + e] = (float)(a.eps * (double)v[j + e]);
    }
  }
}

// Work split: a wavefront takes 64 / G heads at a time, G lanes per head, lane g of a
// head its pairs g V .. g V + V - 1, so that a lane turns pairs that it holds itself.
// G is the power of two from half / V up; lanes past the head and past the last head work
// on elements of another lane, outside the sums, and store nothing.  The query heads of
// `group` tokens one after the other, their key heads and their value heads are cut into
// `chunks` pieces of 64 / G heads (group > 1 where a token's heads would not fill
// them).  A wavefront keeps one piece, its gains and its gain sums, and goes from
// group to group in steps of `step`, so that the wavefronts of the grid read and write
// memory in its order.
struct Piece {
  int seg;            // 0 queries, 1 keys, 2 values
  int t0, ntok, tok;  // first token in the group, tokens, the lane's one after t0
  int i0, col;        // the lane's first pair in its head, its first column
  bool on, ok;        // a lane of the head; of a head that the piece has
};
template <int V, int G, bool GROUP>
__device__ inline Piece piece(const QkArgs& a, const QkSplit& w, int c, int lane) {
  constexpr int HPW = 64 / G;
  const int i0 = (lane & (G - 1)) * V;
  Piece p;
  p.seg = c < w.chunks[0] ? 0 : c < w.chunks[0] + w.chunks[1] ? 1 : 2;
  const int r0 = HPW * (c - (p.seg == 0 ? 0 : p.seg == 1 ? w.chunks[0] : w.chunks[0] + w.chunks[1]));
  const int h0 = p.seg == 0 ? 0 : p.seg == 1 ? a.Hq : a.Hq + a.Hk;
  const int H = p.seg ? a.Hk : a.Hq, rows = GROUP ? w.group * H : H;   // heads of the segment in the group
  const int r = min(r0 + lane / G, rows - 1);
  p.on = i0 < a.dh / 2;
  p.ok = p.on && r0 + lane / G < rows;
  p.i0 = p.on ? i0 : 0;
  p.t0 = GROUP ? r0 / H : 0;
  p.ntok = GROUP ? (min(r0 + HPW, rows) - 1) / H - p.t0 + 1 : 1;
  p.tok = GROUP ? r / H - p.t0 : 0;
  p.col = (h0 + (GROUP ? r % H : r)) * a.dh + p.i0;
  return p;
}

template <typename T, int V, int G, bool NORM, bool GROUP>
__global__ __launch_bounds__(fwd_threads(sizeof(T) == 2, NORM)) void qk_fwd_kernel(QkArgs a, QkSplit w) {
  constexpr int FWD_NT = fwd_threads(sizeof(T) == 2, NORM);
  __shared__ float2 cs[FWD_NT / 64][64 * V];   // 64 / G tokens of half <= G V pairs
  const T *xm = (const T*)a.x_m, *xd = (const T*)a.x_d;
  T *ym = (T*)a.y_m, *yd = (T*)a.y_d;
  const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (FWD_NT / 64) + (threadIdx.x >> 6)));
  const int C = w.chunks[0] + w.chunks[1] + w.chunks[2];
  if (wave / C >= w.step) return;
  const Piece p = piece<V, G, GROUP>(a, w, wave % C, threadIdx.x & 63);
  const int half = a.dh / 2;
  float gm[2 * V], gd[2 * V];
  if constexpr (NORM)
    if (p.seg < 2) lane_gains<T, V>(a, p.seg, p.i0, gm, gd);
  for (int64_t g = wave / C; g < w.groups; g += w.step) {
    // (a wavefront of heads of one token knows its token as a scalar)
    const int t0 = GROUP ? (int)g * w.group + p.t0 : (int)g, t = GROUP ? min(t0 + p.tok, a.T - 1) : t0;
    const bool ok = GROUP ? p.ok && t0 + p.tok < a.T : p.ok;
    Raw<T, V> in[4];   // mean and half difference, first and second half of the head
    const int64_t o = row(t, a.ldx) + p.col;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      load<T, V>(in[k], (k & 2 ? xd : xm) + o + (k & 1 ? half : 0));
    }
    float m[2 * V], d[2 * V], c[V], s[V];
    if (p.seg < 2) token_angles<V, GROUP>(a, w, t0, p.ntok, p.tok, p.i0, cs[threadIdx.x >> 6], c, s);
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) {
      m[e] = get<T, V>(in[e / V], e % V);
      d[e] = get<T, V>(in[2 + e / V], e % V);
    }
    if (p.seg < 2) {
      if constexpr (NORM) {
        double sq = 0.0, md = 0.0;
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
          const double x = m[e], y = d[e];
          sq = fma(x, x, fma(y, y, sq));
          md = fma(x, y, md);
        }
        const Rms r = rms_pair(group_sum<G>(p.on ? sq : 0.0), group_sum<G>(p.on ? md : 0.0), a.inv_n, a.neps);
        float rm = (float)r.m, kappa = (float)r.rho, sigma = 0.f;
        if (r.small) {   // (all lanes of a head alike)
          sigma = r.rho < 0.0 ? 1.f : -1.f;
          double q = 0.0;
#pragma unroll
          for (int e = 0; e < 2 * V; ++e) {
            const double x = fmaf(-sigma, d[e], m[e]);
            q = fma(x, x, q);
          }
          const double rs = rsqrt_nr(fma(group_sum<G>(p.on ? q : 0.0), a.inv_n, a.neps)), t = r.large + rs;
          rm = (float)(0.5 * t);
          kappa = sigma * (float)(2.0 * r.large * rcp_nr(t));
        }
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
          const float um = fmaf(d[e], kappa, fmaf(-sigma, d[e], m[e])) * rm;
          const float ud = fmaf(m[e], kappa, fmaf(-sigma, m[e], d[e])) * rm;
          m[e] = um * gm[e] + ud * gd[e];
          d[e] = um * gd[e] + ud * gm[e];
        }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float ml = m[e], mh = m[V + e], dl = d[e], dh = d[V + e];
        m[e] = ml * c[e] - mh * s[e];
        m[V + e] = mh * c[e] + ml * s[e];
        d[e] = dl * c[e] - dh * s[e];
        d[V + e] = dh * c[e] + dl * s[e];
      }
    }
    if (ok) {
      const int64_t q = row(t, a.ldy) + p.col;
      store<T, V>(ym + q, m);
      store<T, V>(ym + q + half, m + V);
      store<T, V>(yd + q, d);
      store<T, V>(yd + q + half, d + V);
    }
  }
}

// ---- backward of heads with a small point ---------------------------------------------
// Rare, so it comes after the loop over the wavefront's groups, from memory to memory, an element
// after the other: inside the loop it took the kernel from 126 registers to 138 or more, three
// wavefronts per SIMD instead of four (4 + 1 + 1 heads of 128: 306 us against 220).
// One head of a layer in a thousand: 152 us where there are none 141, all of them: 523.
struct Points { float p, n; };
template <typename T>
__device__ inline Points points(const T* m, const T* d, int64_t i) {
  const float x = ldf(m, i), y = ldf(d, i);
  return {x + y, x - y};
}
template <typename T>
__device__ inline Points gain_points(const QkArgs& a, int seg, int j) {
  const float* v = seg ? a.vk : a.vq;
  const float g = ldf((const T*)(seg ? a.gk : a.gq), j), w = v ? (float)(a.eps * (double)v[j]) : 0.f;
  return {g + w, g - w};
}
// The heads of token t that the wavefront's lanes hold, by the whole wavefront; cs: the angles of the
// lane's pairs.  The gain's terms are added over the wavefront's heads to sums[e G + lane].
template <typename T, int V, int G>
__device__ inline void bwd_points(const QkArgs& a, const Piece& p, int t, bool ok, const float2* cs, double* sums) {
  const int half = a.dh / 2, lane = threadIdx.x & 63;
  const T *xm = (const T*)a.x_m, *xd = (const T*)a.x_d;
  const int64_t o = row(t, a.ldx) + p.col, og = row(t, a.lddy) + p.col, oy = row(t, a.ldy) + p.col;
  double sq = 0.0, md = 0.0, sp = 0.0, sn = 0.0;
#pragma unroll 1
  for (int e = 0; e < 2 * V; ++e) {
    const int64_t i = o + (e < V ? e : half + e - V);
    const double x = ldf(xm, i), y = ldf(xd, i);
    sq = fma(x, x, fma(y, y, sq));   // as the loop over the groups adds them: the same heads are small
    md = fma(x, y, md);
    sp = fma(x + y, x + y, sp);
    sn = fma(x - y, x - y, sn);
  }
  const bool take = rms_pair(group_sum<G>(p.on ? sq : 0.0), group_sum<G>(p.on ? md : 0.0), a.inv_n, a.neps).small && ok;
  if (!__ballot(take)) return;
  const Points r = {(float)rsqrt_nr(fma(group_sum<G>(p.on ? sp : 0.0), a.inv_n, a.neps)),
                    (float)rsqrt_nr(fma(group_sum<G>(p.on ? sn : 0.0), a.inv_n, a.neps))};
  Points c = {0.f, 0.f};
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
    for (int e = 0; e < V; ++e) {
      const float co = cs[e].x, si = cs[e].y;
      const Points lo = points(a.dy_m, a.dy_d, og + e), hi = points(a.dy_m, a.dy_d, og + e + half);
      const Points z[2] = {{lo.p * co + hi.p * si, lo.n * co + hi.n * si}, {hi.p * co - lo.p * si, hi.n * co - lo.n * si}};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int j = e + h * half;
        const Points x = points(xm, xd, o + j), g = gain_points<T>(a, p.seg, p.i0 + j);
        const Points u = {x.p * r.p, x.n * r.n}, du = {z[h].p * g.p, z[h].n * g.n};
        if (pass == 0) {
          c.p += u.p * du.p;
          c.n += u.n * du.n;
          double w = take ? 0.5 * (double)(z[h].p * u.p - z[h].n * u.n) : 0.0;
#pragma unroll
          for (int k = G; k < 64; k <<= 1) w += __shfl_xor(w, k, 64);
          if (lane < G) sums[(h * V + e) * G + lane] += w;
        } else if (take) {
          const Points dx = {(du.p - u.p * c.p) * r.p, (du.n - u.n * c.n) * r.n};
          stf((T*)a.y_m, oy + j, 0.5f * (dx.p + dx.n));
          stf((T*)a.y_d, oy + j, 0.5f * (dx.p - dx.n));
        }
      }
    }
    if (pass == 0) {
      c.p = group_sum<G>(p.on ? c.p : 0.f) * (float)a.inv_n;
      c.n = group_sum<G>(p.on ? c.n : 0.f) * (float)a.inv_n;
    }
  }
}

// Backward.  Every workgroup leaves its sums of the gain gradients' half differences
// (fp64, fixed order) as rows 2 blockIdx.x (queries) and 2 blockIdx.x + 1 (keys) of part.
template <typename T, int V, int G, bool NORM, bool GROUP>
__global__ __launch_bounds__(bwd_threads(G)) void qk_bwd_kernel(QkArgs a, QkSplit w) {
  constexpr int BWD_NT = bwd_threads(G), NW = BWD_NT / 64;
  __shared__ float2 cs[NW][64 * V];   // 64 / G tokens of half <= G V pairs
  __shared__ double sh[NORM ? NW : 1][NORM ? 2 * V * G : 1];
  const T *xm = (const T*)a.x_m, *xd = (const T*)a.x_d;
  T *ym = (T*)a.y_m, *yd = (T*)a.y_d;
  const int wv = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * NW + wv)), id = wave;
  const int C = w.chunks[0] + w.chunks[1] + w.chunks[2];
  const int groups = wave / C < w.step ? w.groups : 0;   // (the last workgroup may hold wavefronts without work)
  const Piece p = piece<V, G, GROUP>(a, w, wave % C, lane);
  const int half = a.dh / 2;
  float gm[2 * V], gd[2 * V];
  double acc[2 * V];
  uint64_t small = 0;   // steps (modulo 64) with a head that has a small point
  int step = 0;
  if constexpr (NORM) {
    if (p.seg < 2) lane_gains<T, V>(a, p.seg, p.i0, gm, gd);
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) acc[e] = 0.0;
  }
  for (int64_t g = wave / C; g < groups; g += w.step) {
    const int t0 = GROUP ? (int)g * w.group + p.t0 : (int)g, t = GROUP ? min(t0 + p.tok, a.T - 1) : t0;
    const bool ok = GROUP ? p.ok && t0 + p.tok < a.T : p.ok;
    const int64_t og = row(t, a.lddy) + p.col, ox = row(t, a.ldx) + p.col;
    Raw<float, V> dy[4];
    Raw<T, V> in[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = k & 1 ? half : 0;
      load<float, V, true>(dy[k], (k & 2 ? a.dy_d : a.dy_m) + og + j);
      if constexpr (NORM)
        if (p.seg < 2) load<T, V, true>(in[k], (k & 2 ? xd : xm) + ox + j);
    }
    float zm[2 * V], zd[2 * V];
    bool leave = false;
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) {
      zm[e] = get<float, V>(dy[e / V], e % V);
      zd[e] = get<float, V>(dy[2 + e / V], e % V);
    }
    if constexpr (NORM && GROUP)
      if (!ok)   // a token past the last: nothing for the gains' sums
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) zm[e] = zd[e] = 0.f;
    if (p.seg < 2) {
      float c[V], s[V];
      token_angles<V, GROUP>(a, w, t0, p.ntok, p.tok, p.i0, cs[wv], c, s);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float ml = zm[e], mh = zm[V + e], dl = zd[e], dh = zd[V + e];
        zm[e] = ml * c[e] + mh * s[e];
        zm[V + e] = mh * c[e] - ml * s[e];
        zd[e] = dl * c[e] + dh * s[e];
        zd[V + e] = dh * c[e] - dl * s[e];
      }
      if constexpr (NORM) {
        float m[2 * V], d[2 * V];
        double sq = 0.0, md = 0.0;
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
          m[e] = get<T, V>(in[e / V], e % V);
          d[e] = get<T, V>(in[2 + e / V], e % V);
          const double x = m[e], y = d[e];
          sq = fma(x, x, fma(y, y, sq));
          md = fma(x, y, md);
        }
        const Rms r = rms_pair(group_sum<G>(p.on ? sq : 0.0), group_sum<G>(p.on ? md : 0.0), a.inv_n, a.neps);
        leave = r.small;
        if (__ballot(leave)) small |= 1ull << (step & 63);
        const float rm = leave ? 0.f : (float)r.m, rho = (float)r.rho;   // (u = 0: nothing to the gains' sums here)
        float cm = 0.f, cd = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
          const float um = (m[e] + d[e] * rho) * rm, ud = (m[e] * rho + d[e]) * rm;
          m[e] = um;
          d[e] = ud;
          acc[e] += (double)(zm[e] * ud + zd[e] * um);
          const float dum = zm[e] * gm[e] + zd[e] * gd[e], dud = zm[e] * gd[e] + zd[e] * gm[e];
          zm[e] = dum;
          zd[e] = dud;
          cm += um * dum + ud * dud;
          cd += um * dud + ud * dum;
        }
        cm = group_sum<G>(p.on ? cm : 0.f) * (float)a.inv_n;
        cd = group_sum<G>(p.on ? cd : 0.f) * (float)a.inv_n;
#pragma unroll
        for (int e = 0; e < 2 * V; ++e) {
          const float tm = zm[e] - (m[e] * cm + d[e] * cd), td = zd[e] - (m[e] * cd + d[e] * cm);
          zm[e] = (tm + td * rho) * rm;
          zd[e] = (tm * rho + td) * rm;
        }
      }
    }
    if (ok && !leave) {
      const int64_t q = row(t, a.ldy) + p.col;
      store<T, V, true>(ym + q, zm);
      store<T, V, true>(ym + q + half, zm + V);
      store<T, V, true>(yd + q, zd);
      store<T, V, true>(yd + q + half, zd + V);
    }
    ++step;
  }
  if constexpr (NORM) {
    // Thread, wavefront and arguments once more, as values of their own: what follows uses them, and
    // kept through the loop above they cost it registers (138 of them in fp32 where tokens share a
    // wavefront, 129 so).
    struct Kernarg { QkArgs a; QkSplit w; };   // as the kernel's arguments lie
    auto again = (const __attribute__((address_space(4))) Kernarg*)__builtin_amdgcn_kernarg_segment_ptr();
    int tid = threadIdx.x, wave = id;
    asm volatile("" : "+v"(tid), "+s"(wave), "+s"(again));
    const QkArgs& a = *(const QkArgs*)&again->a;
    const QkSplit& w = *(const QkSplit*)&again->w;
    const int C = w.chunks[0] + w.chunks[1] + w.chunks[2], half = a.dh / 2, lane = tid & 63, wv = wave % NW;
    // over the wavefront's heads, then over the wavefronts of each segment
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) {
      if (!p.ok) acc[e] = 0.0;
#pragma unroll
      for (int o = G; o < 64; o <<= 1) acc[e] += __shfl_xor(acc[e], o, 64);
      if (lane < G) sh[wv][e * G + lane] = acc[e];
    }
    if (small) {
      const Piece p = piece<V, G, GROUP>(a, w, wave % C, lane);
      int step = 0;
      for (int64_t g = wave / C; g < w.groups; g += w.step, ++step) {
        if (!(small >> (step & 63) & 1)) continue;
        const int t0 = GROUP ? (int)g * w.group + p.t0 : (int)g, t = GROUP ? min(t0 + p.tok, a.T - 1) : t0;
        float c[V], s[V];
        token_angles<V, GROUP>(a, w, t0, p.ntok, p.tok, p.i0, cs[wv], c, s);
        bwd_points<T, V, G>(a, p, t, GROUP ? p.ok && t0 + p.tok < a.T : p.ok, cs[wv] + (GROUP ? p.tok * half : 0) + p.i0, sh[wv]);
      }
    }
    __syncthreads();
    for (int k = tid; k < 2 * 2 * V * G; k += BWD_NT) {
      const int seg = k / (2 * V * G), j = k % (2 * V * G);
      double x = 0.0;
#pragma unroll
      for (int v = 0; v < NW; ++v) {
        const int c = (int)((blockIdx.x * NW + v) % C);
        const int sv = c < w.chunks[0] ? 0 : c < w.chunks[0] + w.chunks[1] ? 1 : 2;
        if (sv == seg) x += sh[v][j];
      }
      // entry j: element e = j / G of lane j % G
      const int e = j / G, i = (j % G) * V;
      if (i < half) a.part[(int64_t)(2 * blockIdx.x + seg) * a.dh + i + (e < V ? e : half + e - V)] = x;
    }
  }
}

// out[seg][j] (+)= scale * sum over the workgroups' rows of the segment: 16 columns
// and 64 row groups per workgroup, added in a fixed order.  GU rows in flight per
// thread: with one after the other a backward of 512 rows takes 1.5 us more or longer; 8 or 4
// columns per workgroup take as long.
__global__ __launch_bounds__(1024) void qk_gain_kernel(const double* part, int rows, int dh, double scale, float* dgq,
                                                       float* dgk, bool acc) {
  constexpr int GU = 8;
  __shared__ double sh[16][16];
  const int seg = blockIdx.y, cl = threadIdx.x & 15, j = blockIdx.x * 16 + cl;
  double t = 0.0;
  if (j < dh)
    for (int r = threadIdx.x >> 4; r < rows; r += 64 * GU) {
      double v[GU];
#pragma unroll
      for (int u = 0; u < GU; ++u) v[u] = r + 64 * u < rows ? part[(int64_t)(2 * (r + 64 * u) + seg) * dh + j] : 0.0;
#pragma unroll
      for (int u = 0; u < GU; ++u) t += v[u];
    }
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
int group_lanes(int dh, int v) {
  int g = 1;
  while (v * g < dh / 2) g *= 2;
  return g;
}
// Pairs per lane: 4; in the bf16 forward 8 or 6 where a head divides into them (accesses of
// 16 or 12 bytes), the number that leaves the fewest lanes idle, the larger of two alike.  The layer
// above: 76 us with 8, 77 with 4; 16 + 4 + 4 heads of 256, 105 against 132; with the norm, 72-wide
// heads take 114 us with 6 and 150 with 4, 144-wide ones 132 with 6 and 142 with 8, 96-wide ones
// 110 with 6 and 111 with 8.  In fp32 6 is slower (96-wide 104 us, 98 with 4), and so is more than 4 in
// the backward: 8 leaves two wavefronts per SIMD (204 registers) and takes the layer above 7% longer.
template <typename T, bool BWD>
int lane_pairs(int dh) {
  int v = 4;
  if (!BWD && sizeof(T) == 2)
    for (int c = 6; c <= 8; c += 2)
      if (dh / 2 % c == 0 && c * group_lanes(dh, c) <= v * group_lanes(dh, v)) v = c;
  return v;
}
int pieces(int64_t heads, int dh, int v) { return (int)ceil_div(heads, 64 / group_lanes(dh, v)); }

QkSplit split(const QkArgs& a, int v, bool bf16, bool bwd, bool values) {
  QkSplit w{};
  // The group that gives the fewest pieces in all, the smallest such, if it saves enough: one
  // token per piece is a kernel of its own, which knows the token as a scalar and shares no
  // piece's angles with lanes of other tokens.  A fifth in the bf16 norm forward, whose arithmetic
  // weighs most (28 + 4 + 4 heads of 128, a quarter saved: 107 us, 108 without), a third in other
  // bf16 kernels (the same heads turned alone, forward: 101, 94 without; 5 + 5 + 5 of 40, three
  // eighths saved, 130 and 151, backward 192 and 189), two fifths in fp32 (8 + 1 + 1 of 128, three
  // eighths saved, norm backward: 170 and 142).  Forward and backward share a threshold; at half
  // saved in fp32 (4 + 1 + 1 of 128) the norm's forward gains by it, 101 and 116, and its
  // backward loses, 169 and 141.
  const int worth = !bf16 ? 60 : !bwd && a.gq ? 80 : 66;
  int64_t C = 0, units = 0, most = 0;
  for (int g = 1; g <= 64 && g <= std::max(1, a.T); g *= 2) {
    const int64_t c = pieces((int64_t)g * a.Hq, a.dh, v) + (values ? 2 : 1) * (int64_t)pieces((int64_t)g * a.Hk, a.dh, v);
    const int64_t n = (a.T + g - 1) / g;
    if (g > 1 && n * c >= most) continue;
    most = g == 1 ? n * c * worth / 100 : n * c;
    units = n * c;
    C = c;
    w.group = g;
    w.groups = (int)n;
  }
  w.chunks[0] = pieces((int64_t)w.group * a.Hq, a.dh, v);
  w.chunks[1] = pieces((int64_t)w.group * a.Hk, a.dh, v);
  w.chunks[2] = values ? w.chunks[1] : 0;
  const int nw = (bwd ? bwd_threads(group_lanes(a.dh, v)) : fwd_threads(bf16, a.gq)) / 64;
  // Groups per wavefront.  Backward with the norm: as few as a resident grid leaves.  Elsewhere
  // short runs: many wavefronts, which the scheduler interleaves and which walk through memory
  // closer to its order (the layer above forward 76 us, 86 with the 8 of a resident grid;
  // rotation alone, backward: 98 against 108).  The norm pays for its gains with two tokens per
  // wavefront in bf16 (65536 tokens: 562 us, 563 with one, 610 with four; fp32, 16384: 95 with
  // one, 100 with two), and with twice as many where a quarter or more of the lanes are idle
  // (80-wide bf16 heads: 118 us with four, 125 with two; 96-wide fp32 ones 100 with two, 97 with one,
  // 103 with four), four times in heads wider than 128 (136-wide in fp32: 121 us with four, 131 with
  // two).
  // Up to SHORT units the chip is not full: one.
  constexpr int64_t SHORT = 16384, MOST = (int64_t)1 << 25;   // (a launch has fewer than 2^32 threads)
  int64_t step;
  if (bwd && a.gq) {
    // full steps of the resident grid and a rest (dealt evenly, 2048 tokens took seven steps of 293 where
    // six of 341 and one of 2 do: 44.0 us against 42.3; the layer above 142.3 against 139.6)
    step = std::max<int64_t>(1, BWD_WAVES / C);
  } else {
    const int lanes = group_lanes(a.dh, v);
    const bool idle = 2 * a.dh <= 3 * lanes * v;
    const int64_t run = !a.gq || units <= SHORT ? 1 : (bf16 ? 2 : 1) * (!idle ? 1 : a.dh > 128 ? 4 : 2);
    step = std::min((w.groups + run - 1) / run, std::max<int64_t>(1, MOST / C));
  }
  w.step = (int)std::min<int64_t>(w.groups, step);
  w.blocks = (int)((w.step * C + nw - 1) / nw);
  w.rhalf = (65536 + a.dh / 2 - 1) / (a.dh / 2);   // i * rhalf >> 16 = i / half for i < 512
  return w;
}

// what the workgroups of a backward with gains write of part
size_t part_bytes(const QkArgs& a, const QkSplit& w) { return (size_t)w.blocks * 2 * a.dh * sizeof(double); }

template <typename T, bool BWD, bool NORM, int V, int G>
void launch(const QkArgs& a, const QkSplit& w, hipStream_t s) {
  if constexpr (BWD) {
    if (w.group == 1) hipLaunchKernelGGL((qk_bwd_kernel<T, V, G, NORM, false>), dim3(w.blocks), dim3(bwd_threads(G)), 0, s, a, w);
    else hipLaunchKernelGGL((qk_bwd_kernel<T, V, G, NORM, true>), dim3(w.blocks), dim3(bwd_threads(G)), 0, s, a, w);
  } else {
    constexpr int NT = fwd_threads(sizeof(T) == 2, NORM);
    if (w.group == 1) hipLaunchKernelGGL((qk_fwd_kernel<T, V, G, NORM, false>), dim3(w.blocks), dim3(NT), 0, s, a, w);
    else hipLaunchKernelGGL((qk_fwd_kernel<T, V, G, NORM, true>), dim3(w.blocks), dim3(NT), 0, s, a, w);
  }
}
template <typename T, bool BWD, bool NORM, int V>
hipError_t dispatch_v(const QkArgs& a, const QkSplit& w, hipStream_t s) {
  if (w.blocks == 0) return hipSuccess;
  // (widths that reach no other count: the bf16 forward takes 4 pairs per lane at 8, 40, 56 and
  // other odd multiples of 8 alone, and 6 at 24, 48, 72, 96, 144, 168 and 192)
  constexpr bool ALL = BWD || sizeof(T) == 4;
  switch (group_lanes(a.dh, V)) {
    case 1:
      if constexpr (V != 6) launch<T, BWD, NORM, V, 1>(a, w, s);
      break;
    case 2:
      if constexpr (ALL || V != 4) launch<T, BWD, NORM, V, 2>(a, w, s);
      break;
    case 4:
      if constexpr (ALL || V != 4) launch<T, BWD, NORM, V, 4>(a, w, s);
      break;
    case 8: launch<T, BWD, NORM, V, 8>(a, w, s); break;
    case 16: launch<T, BWD, NORM, V, 16>(a, w, s); break;
    default:   // 32, heads wider than 128
      if constexpr (V == 4) launch<T, BWD, NORM, V, 32>(a, w, s);
  }
  return hipGetLastError();
}
template <typename T, bool BWD, bool NORM>
hipError_t dispatch(const QkArgs& a, bool values, QkSplit* out, hipStream_t s) {
  const int v = lane_pairs<T, BWD>(a.dh);
  const QkSplit w = split(a, v, sizeof(T) == 2, BWD, values);
  if (BWD && NORM && part_bytes(a, w) > a.part_bytes) return hipErrorInvalidValue;
  if (out) *out = w;
  if constexpr (!BWD && sizeof(T) == 2) {
    if (v == 8) return dispatch_v<T, BWD, NORM, 8>(a, w, s);
    if (v == 6) return dispatch_v<T, BWD, NORM, 6>(a, w, s);
  }
  return dispatch_v<T, BWD, NORM, 4>(a, w, s);
}

}  // namespace

size_t qk_scratch_bytes(int64_t T_, int Hq, int Hk, int dh) {
  // split(): no more wavefronts than pieces without groups, nor than the larger of
  // BWD_WAVES and the pieces of one group
  const int64_t c1 = pieces(Hq, dh, 4) + 2 * (int64_t)pieces(Hk, dh, 4);
  const int64_t c64 = pieces((int64_t)64 * Hq, dh, 4) + 2 * (int64_t)pieces((int64_t)64 * Hk, dh, 4);
  const int64_t waves = std::min<int64_t>(T_ * c1, std::max<int64_t>(BWD_WAVES, c64));
  const int nw = bwd_threads(group_lanes(dh, 4)) / 64;
  return (size_t)((waves + nw - 1) / nw) * 2 * dh * sizeof(double);
}

QkPlan qk_plan(const QkArgs& a, bool bf16, bool bwd, bool values) {
  QkPlan p;
  p.pairs = bf16 ? (bwd ? lane_pairs<bf16_t, true>(a.dh) : lane_pairs<bf16_t, false>(a.dh)) : lane_pairs<float, false>(a.dh);
  p.lanes = group_lanes(a.dh, p.pairs);
  p.threads = bwd ? bwd_threads(p.lanes) : fwd_threads(bf16, a.gq);
  p.split = split(a, p.pairs, bf16, bwd, values);
  p.part_bytes = bwd && a.gq ? part_bytes(a, p.split) : 0;
  return p;
}

template <typename T>
hipError_t launch_qk_fwd(QkArgs a, hipStream_t s) {
  if (a.dh % 8 || a.dh > QK_MAX_DH || a.T < 0) return hipErrorInvalidValue;
  a.inv_n = 1.0 / a.dh;
  a.gvec = (((uintptr_t)a.gq | (uintptr_t)a.gk | (uintptr_t)a.vq | (uintptr_t)a.vk) & 15) == 0;
  const bool values = a.x_m != a.y_m;
  return a.gq ? dispatch<T, false, true>(a, values, nullptr, s) : dispatch<T, false, false>(a, values, nullptr, s);
}

template <typename T>
hipError_t launch_qk_bwd(QkArgs a, float* dgq, float* dgk, bool acc, hipStream_t s) {
  if (a.dh % 8 || a.dh > QK_MAX_DH || a.T < 0) return hipErrorInvalidValue;
  a.inv_n = 1.0 / a.dh;
  a.gvec = (((uintptr_t)a.gq | (uintptr_t)a.gk | (uintptr_t)a.vq | (uintptr_t)a.vk) & 15) == 0;
  QkSplit w;
  if (!a.gq) return dispatch<T, true, false>(a, true, &w, s);
  const hipError_t r = dispatch<T, true, true>(a, true, &w, s);
  if (r != hipSuccess) return r;
  hipLaunchKernelGGL(qk_gain_kernel, dim3(ceil_div(a.dh, 16), 2), dim3(1024), 0, s, a.part, w.blocks, a.dh, 1.0 / a.eps, dgq, dgk, acc);
  return hipGetLastError();
}

template hipError_t launch_qk_fwd<float>(QkArgs, hipStream_t);
template hipError_t launch_qk_fwd<bf16_t>(QkArgs, hipStream_t);
template hipError_t launch_qk_bwd<float>(QkArgs, float*, float*, bool, hipStream_t);
template hipError_t launch_qk_bwd<bf16_t>(QkArgs, float*, float*, bool, hipStream_t);

}  // namespace fdh
