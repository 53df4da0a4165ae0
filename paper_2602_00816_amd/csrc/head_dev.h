// Device helpers of the loss over the vocabulary (head.hip, head_gemm.hip).
#pragma once
#include "common.h"

namespace fdh {
namespace {

constexpr float HEAD_NEAR = 0.0625f;   // up to this |ld| the short series
constexpr float FAR_APART = 0.5f;      // from this |ld| on: p and q in the place of a and s

__device__ inline float head_ref(float lm, float ld) { return lm + fabsf(ld); }
__device__ inline bool far_apart(float ld) { return !(fabsf(ld) < FAR_APART); }

// a and s (or p and q) of one logit, see head.hip.  bf16 models: fp32 (the exponential is common to
// both points); fp32 models: fp64.  The series' first omitted terms are below 1e-10 (|ld| < 1/16)
// and 1e-8 (1/2) of the sum, in fp64 2^-40 / 10!.
__device__ inline void pair_exp_near(float lm, float ld, float c, float& a, float& s) {
  const float e = __expf(lm - c), b2 = ld * ld;
  a = e * (1.f + b2 * (0.5f + b2 * (1.f / 24)));
  s = e * ld * (1.f + b2 * (1.f / 6 + b2 * (1.f / 120)));
}
__device__ inline void pair_exp(float lm, float ld, float c, float& a, float& s) {
  const float x = lm - c, b = fabsf(ld);
  if (b < HEAD_NEAR) {
    pair_exp_near(lm, ld, c, a, s);
  } else if (b < FAR_APART) {
    const float e = __expf(x), b2 = ld * ld;
    a = e * (1.f + b2 * (0.5f + b2 * (1.f / 24 + b2 * (1.f / 720 + b2 * (1.f / 40320)))));
    s = e * ld * (1.f + b2 * (1.f / 6 + b2 * (1.f / 120 + b2 * (1.f / 5040))));
  } else {
    a = __expf(x + ld);
    s = __expf(x - ld);
  }
}
__device__ inline void pair_exp(float lm, float ld, float c, double& a, double& s) {
  const double x = (double)lm - (double)c, b = ld;
  if (fabs(b) < HEAD_NEAR) {
    const double e = exp(x), b2 = b * b;
    a = e * (1.0 + b2 * (1.0 / 2 + b2 * (1.0 / 24 + b2 * (1.0 / 720 + b2 * (1.0 / 40320)))));
    s = e * b * (1.0 + b2 * (1.0 / 6 + b2 * (1.0 / 120 + b2 * (1.0 / 5040 + b2 * (1.0 / 362880)))));
  } else {
    const double p = exp(x + b), q = exp(x - b);
    const bool far = far_apart(ld);
    a = far ? p : 0.5 * (p + q);
    s = far ? q : 0.5 * (p - q);
  }
}

}  // namespace
}  // namespace fdh
