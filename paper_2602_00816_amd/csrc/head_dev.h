// Device helpers of the loss over the vocabulary (head.hip, head_gemm.hip).
#pragma once
#include <type_traits>

#include "kernels.h"

namespace fdh {
namespace {

constexpr float HEAD_NEAR = 0.015625f;   // up to this |ld| the short series
constexpr float FAR_APART = 0.5f;      // from this |ld| on: p and q in the place of a and s

__device__ inline float head_ref(float lm, float ld) { return lm + fabsf(ld); }
__device__ inline bool far_apart(float ld) { return !(fabsf(ld) < FAR_APART); }
// fp32 models also take logits far below the reference in fp64: in a row whose two points are far
// apart they may be all that one of them has
__device__ inline bool far_apart_fine(float lm, float ld, float c) { return far_apart(ld) || lm - c < -60.f; }

// e^x, x <= 0, within two steps of fp32 (__expf is off by as many as |x| holds): the rounding of
// x log2 e, and what log2 e lacks in fp32, put back to first order.
__device__ inline float exp_fine(float x) {
  x = x < -200.f ? -200.f : x;   // (minus infinity, where no column is; NaN stays)
  const float hi = 1.4426950216f, lo = 1.9259630e-8f, p = x * hi;
  const float r = fmaf(x, lo, fmaf(x, hi, -p)), e = __builtin_amdgcn_exp2f(p);
  return fmaf(e, r * 0.69314718f, e);
}

// a and s of one logit, see head.hip; for |ld| < 1/2.  In fp32: the exponential is common to both
// points, to the rounding of an fp32 model with FINE.  The series' first omitted terms are below
// 3e-9 (|ld| < 1/64) and 1e-8 of the sum.
template <bool FINE>
__device__ inline void pair_exp_near(float lm, float ld, float c, float& a, float& s) {   // |ld| < 1/64
  const float e = FINE ? exp_fine(lm - c) : __expf(lm - c), b2 = ld * ld;
  a = fmaf(e, 0.5f * b2, e);
  s = e * ld * fmaf(b2, 1.f / 6, 1.f);
}
template <bool FINE>
__device__ inline void pair_exp(float lm, float ld, float c, float& a, float& s) {
  const float e = FINE ? exp_fine(lm - c) : __expf(lm - c), b2 = ld * ld;
  const bool near = fabsf(ld) < HEAD_NEAR;   // (a logit's value goes by itself alone: the short series where it serves)
  a = near ? fmaf(e, 0.5f * b2, e) : e * (1.f + b2 * (0.5f + b2 * (1.f / 24 + b2 * (1.f / 720 + b2 * (1.f / 40320)))));
  s = e * ld * (near ? fmaf(b2, 1.f / 6, 1.f) : 1.f + b2 * (1.f / 6 + b2 * (1.f / 120 + b2 * (1.f / 5040))));
}
// p and q of one logit: fp32 (bf16 models) or fp64
__device__ inline void pair_exp_far(float lm, float ld, float c, float& p, float& q) {
  p = __expf(lm - c + ld);
  q = __expf(lm - c - ld);
}
__device__ inline void pair_exp_far(float lm, float ld, float c, double& p, double& q) {
  const double x = (double)lm - (double)c;
  p = exp(x + (double)ld);
  q = exp(x - (double)ld);
}

// gradient of a row's loss with respect to one logit, but for the target's -1: c and f are the row's
// reference and factors (HeadRows)
template <bool FINE>
__device__ inline void logit_grad(float lm, float ld, float c, double f0, double f1, double f2, double f3, float& gm, float& gd) {
  if (FINE ? far_apart_fine(lm, ld, c) : far_apart(ld)) {
    typedef std::conditional_t<FINE, double, float> F;
    F p, q;
    pair_exp_far(lm, ld, c, p, q);
    gm = (float)(p * (F)f2 + q * (F)f3);
    gd = (float)(p * (F)f2 - q * (F)f3);
  } else {
    float a, s;
    pair_exp<FINE>(lm, ld, c, a, s);
    gm = a * (float)f0 - s * (float)f1;
    gd = s * (float)f0 - a * (float)f1;
  }
}

// x as the gradients' products read it: contiguous, with zeros in the rows that have no target
// (whatever stands there) and in those behind the last; workgroup `block` of `blocks`
template <typename T>
__device__ inline void copy_rows(const HeadCopy& c, int block, int blocks) {
  constexpr int VEC = 16 / sizeof(T);
  for (int64_t t = block; t < c.Tp; t += blocks) {
    const bool live = t < c.T && c.tgt[t] != IGNORE_LABEL;
    for (int j = VEC * threadIdx.x; j < c.d; j += VEC * blockDim.x) {
      const uint4 none = make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4*>((T*)c.om + t * c.d + j) = live ? *reinterpret_cast<const uint4*>((const T*)c.xm + t * c.ldx + j) : none;
      *reinterpret_cast<uint4*>((T*)c.od + t * c.d + j) = live ? *reinterpret_cast<const uint4*>((const T*)c.xd + t * c.ldx + j) : none;
    }
  }
}

}  // namespace
}  // namespace fdh
