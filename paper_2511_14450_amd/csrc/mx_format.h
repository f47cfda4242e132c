// Numbers of 8 and 4 bits under a power of two that 32 of them share, as hyp_mx.h defines them, in gfx950's conversions.
//
// A conversion with a scale multiplies by the power of two in the float's exponent and rounds to the type it gives; every number that
// mx_write stores is a bf16 as it stands, so that none of these roundings changes anything.
#pragma once

#include "mfma_common.h"
#include "mx_kernels.h"

namespace hyp {
namespace {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ int mx_clamped(int v, int lo, int hi) { return min(max(v, lo), hi); }
__device__ __forceinline__ int mx_len(const hyp_mx_cache_t &c, int b) { return mx_clamped(c.lens[b], 0, c.most); }

__device__ __forceinline__ float mx_scale(unsigned byte) { return __uint_as_float(byte << 23); }  // 0: the conversions take an exponent of -127; 255: NaN

// numbers 2 p and 2 p + 1 of the eight that lie in word(s) w, as two bf16
template <int F> __device__ __forceinline__ unsigned mx_pair(const unsigned *w, int p, float scale) {
  bf16x2_t r;
  if constexpr (F == HYP_E4M3) {
    const unsigned x = w[p >> 1];
    r = (p & 1) ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false);
  } else {
    const unsigned x = w[0];
    r = p == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 0)
        : p == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 1)
        : p == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 2)
                 : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, 3);
  }
  return __builtin_bit_cast(unsigned, r);
}

// Largest magnitude of 32 features, as its bits (a NaN's are above infinity's), to the scale byte: the least power of two under which it does
// not pass the format's largest number, which is 1.75 * 2^8 or 1.5 * 2^2.
template <int F> __device__ __forceinline__ unsigned mx_scale_byte(unsigned bits) {
  constexpr int top = F == HYP_E4M3 ? 8 : 2, fraction = F == HYP_E4M3 ? 0x600000 : 0x400000, lo = F == HYP_E4M3 ? 127 - 117 : 127 - 125,
                hi = F == HYP_E4M3 ? 127 + 119 : 127 + 125;
  if (bits >= 0x7f800000u) return 255u;
  return (unsigned)mx_clamped((int)(bits >> 23) - top + ((int)(bits & 0x7fffffu) > fraction), lo, hi);
}

// Eight features to codes (one or two words), and the numbers that are stored in their place, as pairs of bf16.  Where a group is not finite the codes
// are NaN (HYP_E4M3) or 0, and every number NaN.
template <int F> __device__ __forceinline__ void mx_quantise(const float (&x)[8], unsigned scale, unsigned (&w)[2], unsigned (&pairs)[4]) {
  constexpr float most = F == HYP_E4M3 ? 448.f : 6.f;
  const float down = __uint_as_float((254u - scale) << 23), up = mx_scale(scale);  // scale lies in 2..252
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i] * down, -most, most);
  if constexpr (F == HYP_E4M3) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
      w[h] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], c, true);
    }
  } else {
    unsigned c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, y[0], y[1], 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], 1.0f, 2);
    w[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], 1.0f, 3);
    w[1] = 0;
  }
#pragma unroll
  for (int p = 0; p < 4; ++p) pairs[p] = mx_pair<F>(w, p, up);
  const bool bad = scale == 255u;
  if (__any(bad)) {
    w[0] = bad ? (F == HYP_E4M3 ? 0x7f7f7f7fu : 0u) : w[0];
    w[1] = bad ? (F == HYP_E4M3 ? 0x7f7f7f7fu : 0u) : w[1];
#pragma unroll
    for (int p = 0; p < 4; ++p) pairs[p] = bad ? 0x7fc07fc0u : pairs[p];
  }
}

}  // namespace
}  // namespace hyp
