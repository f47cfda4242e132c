// How a capped score is formed of a product, as hyp_attn.h says.
#pragma once

#include "common.h"

namespace hyp {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// A raw score S as an exponent of two, cap log2(e) tanh(S scale / cap).  With x = S scale / cap up to 0.4 in absolute value that is
// S r(S^2), r a polynomial fitted to an even relative error (1e-7, and 1e-7 of its evaluation), whose coefficients the host scales;
// beyond, 1 - 2 / (e^2x + 1), whose absolute error of one rounding is relative there.
__device__ __forceinline__ float cap_factor(float s, const float (&c)[4]) {
  const float y = s * s;
  float q = fmaf(y, c[3], c[2]);
  q = fmaf(y, q, c[1]);
  return fmaf(y, q, c[0]);
}
__device__ __forceinline__ float cap_any(float s, const float (&c)[4], float most, float to_cap, float cap2) {
  const float e = exp2_(2.0f * kLog2e * fabsf(s * to_cap));  // infinity: tanh is 1
  const float far = copysignf(cap2 - 2.0f * cap2 * __builtin_amdgcn_rcpf(e + 1.0f), s);
  return fabsf(s) <= most ? s * cap_factor(s, c) : far;
}

}  // namespace
}  // namespace hyp
