// The logits' pair without logits in memory: the product of a tile of rows and a tile of the
// vocabulary, both channels at once, whose epilogue leaves either the rows' statistics over the
// tile's columns or the logits' gradient in the operand type.
//
// lm = xm wm^T + xd wd^T and ld = xd wm^T + xm wd^T share their operands: a K slice of the four
// tiles (x and w, mean and half difference) feeds four matrix operations per output block (three in the
// HVP, which leaves xd wd^T out), fewer bytes per operation than a 256 x 256 tile of one product takes.  Slices of 64 bytes a row
// (32 k in bf16, 16 in fp32) come by direct loads to LDS into a ring of three stages, two slices
// ahead; a wavefront keeps two fragment sets (half slices) and reads one while the matrix operations
// run on the other.  A stage is free as soon as every wavefront has the second half of its slice in
// registers, which the wait before the slice's one barrier makes sure of.
#include "gemm_dev.h"
#include "head_dev.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace fdh {

namespace {

constexpr uint32_t OOB = 0x80000000u;   // byte offset at which the buffer resources end
constexpr int ROW = 64;                 // bytes of a row's slice

// byte offset of 16-byte chunk c of a row of a tile: 16 lanes that read 16 consecutive rows hit 64 banks
__device__ inline int tile_at(int row, int c) { return row * ROW + ((c ^ ((row >> 2) & 3)) << 4); }

// A fragment holds a lane's 16 bytes of a row: chunk 2 half + (lane >> 5).  fp32: the four operations
// that a pair of fragments feeds take one element each, k and k + 4 in the two halves of the wavefront.
template <typename T> struct Frag;
template <> struct Frag<bf16_t> {
  typedef bf16x8_t type;
  static constexpr int OPS = 1;
  static __device__ inline f32x16_t mma(const type& w, const type& x, int, const f32x16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, x, c, 0, 0, 0);
  }
};
template <> struct Frag<float> {
  typedef float type __attribute__((ext_vector_type(4)));
  static constexpr int OPS = 4;
  static __device__ inline f32x16_t mma(const type& w, const type& x, int e, const f32x16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(w[e], x[e], c, 0, 0, 0);
  }
};
template <typename T>
__device__ inline typename Frag<T>::type fragment(const char* t, int r0, int half, int lane) {
  return *reinterpret_cast<const typename Frag<T>::type*>(t + tile_at(r0 + (lane & 31), 2 * half + (lane >> 5)));
}

// ALL: with xd wd^T
template <typename T, int BM, int BN, int WM, int WN, bool GRAD, bool ALL>
__global__ __launch_bounds__(64 * WM * WN) void head_logits_kernel(HeadLogits a, HeadRows r) {
  constexpr int NW = WM * WN, WTM = BM / WM, WTN = BN / WN, IM = WTM / 32, JN = WTN / 32;
  typedef typename Frag<T>::type F;
  typedef std::conditional_t<sizeof(T) == 4, double, float> P;   // of the statistics and of points far apart
  constexpr int KT = ROW / sizeof(T), CE = 16 / sizeof(T);   // k per slice and per 16 bytes
  constexpr int STAGE = 2 * (BM + BN) * ROW;         // bytes: xm, xd, wm, wd
  constexpr int NU = 2 * (BM + BN) / 16 / NW;        // 1 KB loads per wavefront and slice
  constexpr int NF = 2 * (IM + JN);                  // fragments of a half slice
  // fp32 models and few rows (the operands' bytes bound the tile): exponentials to the last bits.  What
  // __expf rounds is 1e-6 of a gradient or of a loss's half difference: more than fp32 products lose, and in
  // bf16 seen where that half difference is small by chance and no other rows stand beside it.
  constexpr bool FINE = BM == 32 || sizeof(T) == 4;
  constexpr int NM = (ALL ? 4 : 3) * IM * JN * Frag<T>::OPS;       // matrix operations of a half slice
  static_assert(2 * (BM + BN) / 16 % NW == 0 && BM % 16 == 0 && BN % 16 == 0, "whole loads per wavefront");
  __shared__ __attribute__((aligned(1024))) char st0[STAGE];
  __shared__ __attribute__((aligned(1024))) char st1[STAGE];
  __shared__ __attribute__((aligned(1024))) char st2[STAGE];

  const int gx = (a.C + BN - 1) / BN, tiles = gx * ((a.T + BM - 1) / BM);
  if ((int)blockIdx.x >= tiles) return copy_rows<T>(a.copy, blockIdx.x - tiles, gridDim.x - tiles);
  // rows without a target come last, and tiles that hold no other are not formed
  const int live_rows = a.rows ? a.rows[a.T] : a.T, gy = (live_rows + BM - 1) / BM;
  const int32_t* rows = live_rows < a.T ? a.rows : nullptr;
  auto at = [&](int row) { return rows && row < a.T ? rows[row] : row; };
  if ((int)blockIdx.x >= gx * gy) {
    if constexpr (GRAD) {
      const int q = blockIdx.x - gx * gy, c = q % gx * BN, n = min(BN, a.C - c) / CE, end = min((gy + q / gx + 1) * BM, a.Tp);
      for (int row = (gy + q / gx) * BM + (int)threadIdx.x / (BN / CE); row < end; row += 64 * NW / (BN / CE)) {
        const int i = threadIdx.x % (BN / CE);
        if (i >= n) continue;
        const int64_t o = (int64_t)at(row) * a.C + c + CE * i;
        *reinterpret_cast<uint4*>((T*)a.gm + o) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>((T*)a.gd + o) = make_uint4(0, 0, 0, 0);
      }
    }
    return;
  }
  const int lin = xcd_order(blockIdx.x, gx * gy);
  // tiles run down 4 tile rows before the next column (an XCD's tiles share 4 row and 8 column blocks)
  constexpr int GM = 4;
  const int gsize = GM * gx, first_m = lin / gsize * GM, gm_rows = min(gy - first_m, GM);
  const int tm = first_m + lin % gsize % gm_rows, tn = lin % gsize / gm_rows;
  const int m0 = tm * BM, n0 = tn * BN;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int total = (a.d + KT - 1) / KT;

  // load q of a slice: 16 rows of one of the four tiles.  Rows past the end read the last one
  // (their outputs are not used), lanes past the contraction's end nothing (zeros).
  const int ck = (lane & 3) ^ ((lane >> 4) & 3);   // (row >> 2 is lane >> 4 modulo 4)
  const T* base[NU];
  uint32_t vo[NU];
#pragma clang loop unroll(full)
  for (int u = 0; u < NU; ++u) {
    const int q = wave + u * NW;
    const bool isx = q < 2 * BM / 16;
    const int qx = isx ? q : q - 2 * BM / 16;
    const int per = isx ? BM / 16 : BN / 16;
    const bool half = qx >= per;
    const int row = (half ? qx - per : qx) * 16 + (lane >> 2);
    const int64_t ld = isx ? a.ldx : a.d;
    const int first = isx ? m0 : n0, end = isx ? a.T : a.C;
    const T* p = (const T*)(isx ? (half ? a.xd : a.xm) : (half ? a.wd : a.wm));
    const bool moved = isx && rows;   // (all of x within 31 bits)
    const int src = min(first + row, end - 1);
    base[u] = moved ? p : p + first * ld;
    vo[u] = (uint32_t)sizeof(T) * (uint32_t)((moved ? at(src) : src - first) * ld + CE * ck);
  }
  auto stage = [&](auto s) -> char* {
    constexpr int S = decltype(s)::value % 3;
    if constexpr (S == 0) return st0;
    else if constexpr (S == 1) return st1;
    else return st2;
  };
  // load u of slice t (past the last: the last again, into a stage that nobody reads)
  auto dma = [&](char* st, int t, int u) {
    const int k0 = min(t, total - 1) * KT;
    const uint64_t b = (uint64_t)(uintptr_t)(base[u] + k0);
    const i32x4_t rs{(int)(uint32_t)b, (int)((b >> 32) & 0xffffu), (int)OOB, 0x00020000};
    const uint32_t off = CE * ck < a.d - k0 ? vo[u] : OOB;
    const uint32_t ldsaddr = (uint32_t)(uintptr_t)(lds_void_t*)st + (uint32_t)((wave + u * NW) * 1024);
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %1, %2, 0 offen lds"
        :
        : "s"(ldsaddr), "v"(off), "s"(rs)
        : "memory", "m0");
  };

  f32x16_t cm[IM][JN], cd[IM][JN];
#pragma clang loop unroll(full)
  for (int i = 0; i < IM; ++i)
#pragma clang loop unroll(full)
    for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
      for (int e = 0; e < 16; ++e) cm[i][j][e] = cd[i][j][e] = 0.f;

  // fragments 0 .. IM - 1: xm, then JN of wm, IM of xd, JN of wd (the order in which they are used)
  F f0[NF], f1[NF];
  auto rd = [&](F& f, const char* st, int x, int half) {
    if (x < IM) f = fragment<T>(st, wm * WTM + x * 32, half, lane);
    else if (x < IM + JN) f = fragment<T>(st + 2 * BM * ROW, wn * WTN + (x - IM) * 32, half, lane);
    else if (x < 2 * IM + JN) f = fragment<T>(st + BM * ROW, wm * WTM + (x - IM - JN) * 32, half, lane);
    else f = fragment<T>(st + (2 * BM + BN) * ROW, wn * WTN + (x - 2 * IM - JN) * 32, half, lane);
  };
  auto mma = [&](const F (&f)[NF], int e) {
    constexpr int NB = IM * JN;
    const int kind = e / (NB * Frag<T>::OPS), k = e / NB % Frag<T>::OPS, i = e % NB / JN, j = e % JN;
    const F *xm = f, *wmf = f + IM, *xd = f + IM + JN, *wdf = f + 2 * IM + JN;
    if (kind == 0) cm[i][j] = Frag<T>::mma(wmf[j], xm[i], k, cm[i][j]);
    else if (kind == 1) cd[i][j] = Frag<T>::mma(wmf[j], xd[i], k, cd[i][j]);
    else if (kind == 2) cd[i][j] = Frag<T>::mma(wdf[j], xm[i], k, cd[i][j]);
    else cm[i][j] = Frag<T>::mma(wdf[j], xd[i], k, cm[i][j]);
  };
  auto step = [&](auto s, int t) {
    constexpr int S = decltype(s)::value;
    char* cur = stage(s);
    const char* nxt = stage(std::integral_constant<int, S + 1>{});
#pragma clang loop unroll(full)
    for (int x = 0; x < NF; ++x) {
      rd(f1[x], cur, x, 1);
#pragma clang loop unroll(full)
      for (int e = x * NM / NF; e < (x + 1) * NM / NF; ++e) mma(f0, e);
      __builtin_amdgcn_sched_barrier(0);
    }
    // own loads of slice t + 1 are there (slice t + 2's may be on their way) and own reads of slice
    // t are done: after the barrier everyone's are, and stage S is free
    __builtin_amdgcn_s_waitcnt((NU & 15) | ((NU >> 4) << 14) | (7 << 4) | (0 << 8));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
#pragma clang loop unroll(full)
    for (int x = 0; x < NF; ++x) {
      if (x < NU) dma(cur, t + 3, x);
      if (x == NF - 1) {
#pragma clang loop unroll(full)
        for (int u = NF; u < NU; ++u) dma(cur, t + 3, u);
      }
      rd(f0[x], nxt, x, 0);
#pragma clang loop unroll(full)
      for (int e = x * NM / NF; e < (x + 1) * NM / NF; ++e) mma(f1, e);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  // slices 0, 1 and 2; the first is waited for
#pragma clang loop unroll(full)
  for (int u = 0; u < NU; ++u) dma(st0, 0, u);
#pragma clang loop unroll(full)
  for (int u = 0; u < NU; ++u) dma(st1, 1, u);
#pragma clang loop unroll(full)
  for (int u = 0; u < NU; ++u) dma(st2, 2, u);
  wait_vm<2 * NU>();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
#pragma clang loop unroll(full)
  for (int x = 0; x < NF; ++x) rd(f0[x], st0, x, 0);
  for (int t = 0; t < total; t += 3) {
    step(std::integral_constant<int, 0>{}, t);
    if (t + 1 < total) step(std::integral_constant<int, 1>{}, t + 1);
    if (t + 2 < total) step(std::integral_constant<int, 2>{}, t + 2);
  }
  wait_vm<0>();   // no load may land in LDS from here on

  // A block holds its part of the logits' transpose: lane l has row l & 31 and, for g = 0 .. 3, the
  // columns 8 g + 4 (l >> 5) + 0 .. 3.  Lanes l and l + 32 share a row.
  const int h = lane >> 5;
  const int c0 = n0 + wn * WTN, live = a.C - c0;   // the wavefront's first column and how many there are
  if constexpr (!GRAD) {
    if (live <= 0) return;
    if (live < WTN) {
#pragma clang loop unroll(full)
      for (int i = 0; i < IM; ++i)
#pragma clang loop unroll(full)
        for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
          for (int e = 0; e < 16; ++e)
            if (j * 32 + 8 * (e / 4) + 4 * h + e % 4 >= live) {
              cm[i][j][e] = -INFINITY;
              cd[i][j][e] = 0.f;
            }
    }
#pragma clang loop unroll(full)
    for (int i = 0; i < IM; ++i) {
      const int place = m0 + wm * WTM + i * 32 + (lane & 31), row = at(place);
      float mx = -INFINITY, far = 0.f;
#pragma clang loop unroll(full)
      for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
        for (int e = 0; e < 16; ++e) {
          mx = fmaxf(mx, cm[i][j][e]);
          far = fmaxf(far, fabsf(cd[i][j][e]));
        }
      mx += far;   // (any reference that no logit of the row exceeds will do)
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      float za = 0.f, zs = 0.f;
      P zp = 0, zq = 0;
      if (!__any(!(far < HEAD_NEAR))) {   // (NaN: a half difference that is NaN makes the sums NaN either way)
#pragma clang loop unroll(full)
        for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
          for (int e = 0; e < 16; ++e) {
            float p, s;
            pair_exp_near<FINE>(cm[i][j][e], cd[i][j][e], mx, p, s);
            za += p;
            zs += s;
          }
      } else {
#pragma clang loop unroll(full)
        for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
          for (int e = 0; e < 16; ++e) {
            const float m = cm[i][j][e], d = cd[i][j][e];
            if (sizeof(T) == 4 ? far_apart_fine(m, d, mx) : far_apart(d)) {
              P p, q;
              pair_exp_far(m, d, mx, p, q);
              zp += p;
              zq += q;
            } else {
              float p, s;
              pair_exp<FINE>(m, d, mx, p, s);
              za += p;
              zs += s;
            }
          }
      }
      P z[4] = {za, zs, zp, zq};
#pragma clang loop unroll(full)
      for (int k = 0; k < 4; ++k) z[k] += __shfl_xor(z[k], 32, 64);
      if (place >= a.T) continue;
      if (a.lm) {   // (one piece: kept for its gradient)
        const int64_t o = (int64_t)row * a.C + c0 + 4 * h;
#pragma clang loop unroll(full)
        for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
          for (int g = 0; g < 4; ++g)
            if (j * 32 + 8 * g < live) {   // (C is a multiple of 8)
              *reinterpret_cast<float4*>(a.lm + o + j * 32 + 8 * g) =
                  make_float4(cm[i][j][4 * g], cm[i][j][4 * g + 1], cm[i][j][4 * g + 2], cm[i][j][4 * g + 3]);
              *reinterpret_cast<float4*>(a.ld + o + j * 32 + 8 * g) =
                  make_float4(cd[i][j][4 * g], cd[i][j][4 * g + 1], cd[i][j][4 * g + 2], cd[i][j][4 * g + 3]);
            }
      }
      if (h == 0) {
        P* o = (P*)a.part + (int64_t)(c0 / WTN) * 5 * a.T + row;
        o[0] = mx;
#pragma clang loop unroll(full)
        for (int k = 0; k < 4; ++k) o[(int64_t)(k + 1) * a.T] = z[k];
      }
      const int y = a.tgt[row] - a.n0 - c0;   // (a row without a target has a negative one)
      if (y >= 0 && y < min(live, WTN) && ((y >> 2) & 1) == h) {
        float ym = 0.f, yd = 0.f;
#pragma clang loop unroll(full)
        for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
          for (int e = 0; e < 16; ++e)
            if (j * 32 + 8 * (e / 4) + 4 * h + e % 4 == y) {
              ym = cm[i][j][e];
              yd = cd[i][j][e];
            }
        r.ym[row] = ym;
        r.yd[row] = yd;
      }
    }
  } else {
    // The gradient is held in the operand type, which its products read: bf16's half step, 2^-9 to 2^-8 of an
    // element, is independent from one to the next and leaves 1.0e-4 of dx.m and 2.1e-4 of dx.d and dw
    // (1024 x 32000 x 2048, float32 outputs; rounded to bf16 they are off by 1.7e-3).  Two bf16 parts
    // would double the products.
    // bf16: through LDS, so that a store covers 8 rows of 64 columns (JN = 2) or 16 of 32; a wavefront's
    // own area, 32 rows of WTN columns for each channel in turn
    constexpr int LD = WTN + 4;      // elements: 8-byte rows, lanes of 32 rows on distinct banks
    static_assert(sizeof(T) == 4 || NW * 32 * LD * 2 <= STAGE, "staging areas exceed a stage");
    __syncthreads();                 // every wavefront is done with the ring
    bf16_t* stg = reinterpret_cast<bf16_t*>(st0) + wave * 32 * LD;
    constexpr int LPR = WTN / 8, RPS = 64 / LPR;   // lanes per row of a store, rows per store
#pragma clang loop unroll(full)
    for (int i = 0; i < IM; ++i) {
      const int rb = m0 + wm * WTM + i * 32;
      const int row = at(rb + (lane & 31));
      const int t = min(row, a.T - 1);
      const int y = row < a.T ? a.tgt[t] : IGNORE_LABEL;
      const bool none = y == IGNORE_LABEL;
      const float top = r.top[t];
      const double e0 = r.f[0][t], e1 = r.f[1][t], e2 = r.f[2][t], e3 = r.f[3][t];
      const float w0 = (float)e0, w1 = (float)e1;
      const int yc = y - a.n0 - c0;
      float far = 0.f, low = 0.f;
#pragma clang loop unroll(full)
      for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
        for (int e = 0; e < 16; ++e) {
          far = fmaxf(far, fabsf(cd[i][j][e]));
          if constexpr (sizeof(T) == 4) low = fminf(low, cm[i][j][e] - top);
        }
      if (!__any(!(far < HEAD_NEAR) || low < -60.f)) {
#pragma clang loop unroll(full)
        for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
          for (int e = 0; e < 16; ++e) {
            float p, s;
            pair_exp_near<FINE>(cm[i][j][e], cd[i][j][e], top, p, s);
            cm[i][j][e] = p * w0 - s * w1;
            cd[i][j][e] = s * w0 - p * w1;
          }
      } else {
#pragma clang loop unroll(full)
        for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
          for (int e = 0; e < 16; ++e) {
            float gm, gd;
            logit_grad<sizeof(T) == 4>(cm[i][j][e], cd[i][j][e], top, e0, e1, e2, e3, gm, gd);
            cm[i][j][e] = gm;
            cd[i][j][e] = gd;
          }
      }
      if (yc >= 0 && yc < WTN) {
#pragma clang loop unroll(full)
        for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
          for (int e = 0; e < 16; ++e)
            if (j * 32 + 8 * (e / 4) + 4 * h + e % 4 == yc) cm[i][j][e] -= 1.f;
      }
      if constexpr (sizeof(T) == 4) {
        if (row >= a.Tp) continue;
        const int64_t o = (int64_t)row * a.C + c0 + 4 * h;
#pragma clang loop unroll(full)
        for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
          for (int g = 0; g < 4; ++g)
            if (j * 32 + 8 * g < live) {   // (C is a multiple of 8)
              auto four = [&](const f32x16_t& v) {
                return none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]);
              };
              *reinterpret_cast<float4*>((float*)a.gm + o + j * 32 + 8 * g) = four(cm[i][j]);
              *reinterpret_cast<float4*>((float*)a.gd + o + j * 32 + 8 * g) = four(cd[i][j]);
            }
        continue;
      }
#pragma clang loop unroll(full)
      for (int ch = 0; ch < 2; ++ch) {
#pragma clang loop unroll(full)
        for (int j = 0; j < JN; ++j)
#pragma clang loop unroll(full)
          for (int g = 0; g < 4; ++g) {
            const f32x16_t& v = ch ? cd[i][j] : cm[i][j];
            auto two = [&](int e) {
              return (uint32_t)f32_to_bf16(none ? 0.f : v[e]) | ((uint32_t)f32_to_bf16(none ? 0.f : v[e + 1]) << 16);
            };
            *reinterpret_cast<uint2*>(stg + (lane & 31) * LD + j * 32 + 8 * g + 4 * h) = make_uint2(two(4 * g), two(4 * g + 2));
          }
        wave_lds_order();
        bf16_t* o = (bf16_t*)(ch ? a.gd : a.gm);
#pragma clang loop unroll(full)
        for (int k = 0; k < 32 / RPS; ++k) {
          const int lr = k * RPS + lane / LPR, lc = 8 * (lane % LPR);
          const uint2* p = reinterpret_cast<const uint2*>(stg + lr * LD + lc);
          const uint2 u = p[0], v = p[1];
          const int to = __shfl(row, lr, 64);
          if (rb + lr < a.Tp && lc < live)   // (C is a multiple of 8)
            *reinterpret_cast<uint4*>(o + (int64_t)to * a.C + c0 + lc) = make_uint4(u.x, u.y, v.x, v.y);
        }
        wave_lds_order();   // the next writes come after these reads
      }
    }
  }
}

template <typename T, int BM, int BN, int WM, int WN>
void launch_tile(const HeadLogits& a, const HeadRows& r, bool grad, hipStream_t s) {
  // (the copy of x on compute units that the tiles leave idle: 4 us less than a launch of its own)
  const int copies = a.copy.om ? std::min(256, a.copy.Tp) : 0;
  const dim3 grid(ceil_div(a.C, BN) * ceil_div(a.T, BM) + copies), block(64 * WM * WN);
  auto launch = [&](auto all) {
    constexpr bool ALL = decltype(all)::value;
    if (grad) hipLaunchKernelGGL((head_logits_kernel<T, BM, BN, WM, WN, true, ALL>), grid, block, 0, s, a, r);
    else hipLaunchKernelGGL((head_logits_kernel<T, BM, BN, WM, WN, false, ALL>), grid, block, 0, s, a, r);
  };
  // (fp32 models and few rows have it in the HVP too: 1e-6 of a gradient or of a loss's half difference at its
  // steps, more than is lost otherwise there)
  if constexpr (BM > 32 && sizeof(T) == 2) {
    if (head_products<T>(a.tile, a.second) == 3) return launch(std::false_type{});
  }
  launch(std::true_type{});
}

}  // namespace

// The largest tile that the rows fill and that gives most compute units a workgroup.  Loss alone, us,
// by tile (rows x columns):          256x128  128x128  64x128  64x64  32x128
//   32 x 32000 x 2048                     92       64      51     52      51
//   64 x 32000 x 2048                     93       64      55     67      71
//   128 x 32000 x 2048                    99       72      85     99     110
//   512 x 32000 x 2048                   213      242     294    344     406
//   256 x 4096 x 512                      29       21      17     16      17
//   512 x 4096 x 512                      31       24      21     22      25
//   1024 x 4096 x 512                     31       25      29     31      36
// (1 x 32000 x 2048 on weights that no cache holds: 60; 62 and 64 with tiles of 32 x 64 and 32 x 32.
// With three products 256 x 128 on four wavefronts of 128 x 64, and 128 x 256, were 1 to 5% slower than eight of
// 64 x 64 at 8192 x 32000 x 2048.  The matrix cores are busy for 78% of the cycles there, 66% with three.)
HeadTile head_tile(int T_, int C) {
  auto fills = [&](int bm, int bn) { return T_ > bm / 2 && (int64_t)ceil_div(T_, bm) * ceil_div(C, bn) >= 192; };
  if (fills(256, 128)) return {256, 128, 64};
  if (fills(128, 128)) return {128, 128, 32};
  if (fills(64, 128)) return {64, 128, 32};
  if (T_ > 32) return {64, 64, 32};
  return {32, 128, 32};
}

// fp32 models: this kernel takes the fp32 matrix instructions, the GEMM (gemm_f32.hip) split operands on the
// bf16 ones, a quarter faster, on whole tiles of 128 rows, contractions cut where tiles are few; with it
// the statistics are a launch more and the logits go through memory, 16 bytes written and read each.  Estimates
// of both in us: rounds of tiles over the compute units, each its slices of 16 k at 613 GFLOP/s and 5%, and 9
// for its epilogue, and 10 for the joining launch; 200 TFLOP/s, 5.5 TB/s and 25 for three launches.  Loss
// alone, us, here and there:
//   1 x 32000 x 2048    157  368      33 x 32000 x 2048   253  360      128 x 32000 x 2048  486  395
//   128 x 8192 x 512     44   56      512 x 8192 x 512    136  118      2047 x 8192 x 512   483  400
//   1000 x 32000 x 64   179  206      1000 x 32000 x 128  292  282      1000 x 32000 x 256  519  443
//   4096 x 8192 x 64    160  219      2000 x 4096 x 16     26   59      8192 x 1024 x 256   132  138
//   512 x 256 x 64       16   25      1 x 1024 x 1024      70   29      200 x 2048 x 512     41   40
bool head_f32_fused(int T_, int C, int d, bool second) {
  const HeadTile t = head_tile(T_, C);
  const double wgs = (double)ceil_div(T_, t.BM) * ceil_div(C, t.BN), slice = 4 * 2.0 * t.BM * t.BN * 16 / 613e3;
  const double here = std::ceil(wgs / 256) * (1.05 * ceil_div(d, 16) * slice + 9) + 10;
  const double there = (second ? 8.0 : 6.0) * ceil_div(T_, 128) * 128 * C * d / 200e6 + 16.0 * T_ * C / 5.5e6 + 25;
  return here < there;
}

template <typename T>
hipError_t launch_head_logits(const HeadLogits& a, const HeadRows& r, bool grad, hipStream_t s) {
  if (a.tile.BM == 256) launch_tile<T, 256, 128, 4, 2>(a, r, grad, s);
  else if (a.tile.BM == 128) launch_tile<T, 128, 128, 2, 4>(a, r, grad, s);
  else if (a.tile.BM == 64 && a.tile.BN == 128) launch_tile<T, 64, 128, 2, 4>(a, r, grad, s);
  else if (a.tile.BM == 64) launch_tile<T, 64, 64, 2, 2>(a, r, grad, s);
  else launch_tile<T, 32, 128, 1, 4>(a, r, grad, s);
  return hipGetLastError();
}
template hipError_t launch_head_logits<float>(const HeadLogits&, const HeadRows&, bool, hipStream_t);
template hipError_t launch_head_logits<bf16_t>(const HeadLogits&, const HeadRows&, bool, hipStream_t);

}  // namespace fdh
