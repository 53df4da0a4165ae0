// Both gradients of the vocabulary loss for a few rows (at most HEAD_THIN) in one pass over w.
//
//   dx.m = gm wm + gd wd,   dx.d = gd wm + gm wd,   dw = (gm^T xd + gd^T xm) / eps
// with the logits' gradient (gm, gd) in fp32, formed here from the logits and the rows' statistics.
// With so few rows the bytes of w (read) and dw (written) bound the work, not the products: a
// workgroup takes a run of vocabulary rows at up to 1024 columns, reads each element of w once, keeps
// x and its part of dx in registers (four columns a thread) and writes its rows of dw.  The parts of
// dx, one per run, are added by a second launch in a fixed order.  1 row of 32000 x 2048 bf16: 215 ->
// 132 us for the whole call (8 rows: 231 -> 216), with the products on the matrix cores, which round gm
// and gd to bf16, before.
#include <algorithm>
#include <type_traits>

#include "head_dev.h"

namespace fdh {

namespace {

constexpr int NT = 256, RUN = 512;   // most vocabulary rows of a workgroup

__device__ inline float4 four(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ inline float4 four(const bf16_t* p) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                     __uint_as_float(u.y & 0xffff0000u));
}
__device__ inline void put(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ inline void put(bf16_t* p, const float (&v)[4]) {
  auto two = [](float x, float y) { return (uint32_t)f32_to_bf16(x) | ((uint32_t)f32_to_bf16(y) << 16); };
  *reinterpret_cast<uint2*>(p) = make_uint2(two(v[0], v[1]), two(v[2], v[3]));
}

// T: type of x and w, O: of dw; N: rows, a power of two (those from T_ on are zeros).  `lanes`
// threads (a power of two) hold a row's columns, NT / lanes rows of w are in work at a time.
template <typename T, typename O, int N>
__global__ __launch_bounds__(NT) void head_thin_kernel(HeadThin a, HeadRows r, int lanes, int run) {
  __shared__ float gm[RUN][N], gd[RUN][N];
  __shared__ float4 sh[NT];
  const int groups = NT / lanes, grp = threadIdx.x / lanes;
  const int c = blockIdx.y * 4 * lanes + 4 * (threadIdx.x % lanes);
  const bool on = c < a.d;
  const int col = on ? c : 0;
  const int j0 = blockIdx.x * run, nj = min(run, a.V - j0);
  for (int i = threadIdx.x; i < run * N; i += NT) {
    const int jj = i % run, t = i / run;
    float m = 0.f, d = 0.f;
    if (t < a.T && jj < nj) {
      const int y = a.tgt[t];
      if (y != IGNORE_LABEL) {
        const int64_t at = (int64_t)t * a.V + j0 + jj;
        logit_grad<sizeof(T) == 4>(a.lm[at], a.ld[at], r.top[t], r.f[0][t], r.f[1][t], r.f[2][t], r.f[3][t], m, d);
        if (j0 + jj == y) m -= 1.f;
      }
    }
    gm[jj][t] = m;
    gd[jj][t] = d;
  }
  float xm[N][4], xd[N][4], dm[N][4], dd[N][4];
#pragma unroll
  for (int t = 0; t < N; ++t) {
    const bool live = on && t < a.T && a.tgt[min(t, a.T - 1)] != IGNORE_LABEL;
    const int64_t at = (int64_t)min(t, a.T - 1) * a.ldx + col;
    const float4 p = four((const T*)a.xm + at), q = four((const T*)a.xd + at);
    const float pm[4] = {p.x, p.y, p.z, p.w}, pd[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      xm[t][e] = live ? pm[e] : 0.f;
      xd[t][e] = live ? pd[e] : 0.f;
      dm[t][e] = dd[t][e] = 0.f;
    }
  }
  __syncthreads();
  constexpr int U = N == 8 ? 2 : 4;   // rows of w in flight
  for (int b = grp; b < nj; b += U * groups) {
    float4 pm[U], pd[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = (int64_t)(j0 + min(b + u * groups, nj - 1)) * a.d + col;
      pm[u] = four((const T*)a.wm + at);
      pd[u] = four((const T*)a.wd + at);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int jj = b + u * groups;
      if (jj >= nj) break;
      const float wm[4] = {pm[u].x, pm[u].y, pm[u].z, pm[u].w}, wd[4] = {pd[u].x, pd[u].y, pd[u].z, pd[u].w};
      float w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < N; ++t) {
        const float m = gm[jj][t], d = gd[jj][t];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          dm[t][e] = fmaf(d, wd[e], fmaf(m, wm[e], dm[t][e]));
          dd[t][e] = fmaf(m, wd[e], fmaf(d, wm[e], dd[t][e]));
          w[e] = fmaf(d, xm[t][e], fmaf(m, xd[t][e], w[e]));
        }
      }
      if (!on) continue;
      O* o = (O*)a.dw + (int64_t)(j0 + jj) * a.d + c;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] *= a.alpha_w;
      if constexpr (std::is_same_v<O, float>) {
        if (a.acc) {
          const float4 old = four(o);
          w[0] += old.x; w[1] += old.y; w[2] += old.z; w[3] += old.w;
        }
      }
      put(o, w);
    }
  }
  // the row groups' parts of dx, in their order
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int ch = 0; ch < 2; ++ch) {
      const float (&v)[4] = ch ? dd[t] : dm[t];
      float s[4] = {v[0], v[1], v[2], v[3]};
      if (groups > 1) {
        __syncthreads();
        sh[threadIdx.x] = make_float4(v[0], v[1], v[2], v[3]);
        __syncthreads();
        if (grp == 0)
          for (int g = 1; g < groups; ++g) {
            const float4 x = sh[g * lanes + threadIdx.x];
            s[0] += x.x; s[1] += x.y; s[2] += x.z; s[3] += x.w;
          }
      }
      if (grp == 0 && on && t < a.T) put(a.part + (((int64_t)blockIdx.x * a.T + t) * 2 + ch) * a.d + c, s);
    }
}

// dx = scale times the sum of the runs' parts [runs][T][2][d]: 64 columns of a row and channel per
// workgroup, 16 runs at a time, fp64
template <typename O>
__global__ __launch_bounds__(1024) void head_thin_sum_kernel(O* om, O* od, int64_t ldo, const float* part, int runs, int T_, int d, float scale) {
  __shared__ double sh[16][64];
  const int l = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + l, t = blockIdx.y >> 1, ch = blockIdx.y & 1;
  const int64_t step = (int64_t)T_ * 2 * d, at = ((int64_t)t * 2 + ch) * d + min(c, d - 1);
  double s = 0.0;
  constexpr int U = 8;
  for (int p = g; p < runs; p += 16 * U) {
    float x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = part[min(p + 16 * u, runs - 1) * step + at];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p + 16 * u < runs) s += (double)x[u];
  }
  sh[g][l] = s;
  __syncthreads();
  if (g != 0 || c >= d) return;
  for (int q = 1; q < 16; ++q) s += sh[q][l];
  stf(ch ? od : om, t * ldo + c, (float)(s * (double)scale));
}

// vocabulary rows per workgroup: 512 workgroups or more where there are as many, in runs of 8 to RUN
int run_of(int V, int d) {
  const int cols = (int)ceil_div(d, 1024);
  return std::min(RUN, std::max(8, V / (512 / std::min(cols, 64)) / 8 * 8));
}

template <typename T, typename O>
void launch_n(const HeadThin& a, const HeadRows& r, hipStream_t s) {
  int lanes = 2;
  while (lanes < NT && 4 * lanes < a.d) lanes *= 2;
  const int run = run_of(a.V, a.d);
  const dim3 grid(ceil_div(a.V, run), ceil_div(a.d, 4 * lanes));
  if (a.T <= 1) hipLaunchKernelGGL((head_thin_kernel<T, O, 1>), grid, dim3(NT), 0, s, a, r, lanes, run);
  else if (a.T <= 2) hipLaunchKernelGGL((head_thin_kernel<T, O, 2>), grid, dim3(NT), 0, s, a, r, lanes, run);
  else if (a.T <= 4) hipLaunchKernelGGL((head_thin_kernel<T, O, 4>), grid, dim3(NT), 0, s, a, r, lanes, run);
  else hipLaunchKernelGGL((head_thin_kernel<T, O, 8>), grid, dim3(NT), 0, s, a, r, lanes, run);
}

}  // namespace

size_t head_thin_part(int T_, int V, int d) { return (size_t)ceil_div(V, run_of(V, d)) * T_ * 2 * d * 4; }

template <typename T>
hipError_t launch_head_thin(const HeadThin& a, const HeadRows& r, bool out_f32, hipStream_t s) {
  const int runs = (int)ceil_div(a.V, run_of(a.V, a.d));
  const dim3 grid(ceil_div(a.d, 64), 2 * a.T);
  if (out_f32) {
    launch_n<T, float>(a, r, s);
    hipLaunchKernelGGL(head_thin_sum_kernel<float>, grid, dim3(1024), 0, s, (float*)a.dxm, (float*)a.dxd, a.lddx, a.part, runs, a.T, a.d, a.scale);
  } else {
    launch_n<T, T>(a, r, s);
    hipLaunchKernelGGL(head_thin_sum_kernel<T>, grid, dim3(1024), 0, s, (T*)a.dxm, (T*)a.dxd, a.lddx, a.part, runs, a.T, a.d, a.scale);
  }
  return hipGetLastError();
}
template hipError_t launch_head_thin<float>(const HeadThin&, const HeadRows&, bool, hipStream_t);
template hipError_t launch_head_thin<bf16_t>(const HeadThin&, const HeadRows&, bool, hipStream_t);

}  // namespace fdh
