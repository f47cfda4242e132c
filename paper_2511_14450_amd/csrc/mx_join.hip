// Joining what the parts of a request's keys gave for its row.
#include "mx_format.h"
#include "mx_rules.h"

namespace hyp {
namespace {

constexpr float kLn2 = 0.6931471805599453f;

// A wave for each row and query head: the weights of the parts, then their sums, a feature a lane.
template <typename T> __global__ void __launch_bounds__(256) k_mx_join(const MxTokenCall p) {
  const hyp_mx_cache_t &c = p.m.c;
  const int64_t rows = (int64_t)c.n_requests * p.q.n_q_heads, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int lane = threadIdx.x & 63, b = (int)(row / p.q.n_q_heads), h = (int)(row % p.q.n_q_heads), d = c.head_dim;
  const int runs = p.listed ? p.listed << (p.m.block_shift - 4) : (mx_len(c, b) + 15) >> 4;
  const int parts = max(1, (runs + p.runs - 1) / p.runs);
  float top = -3.402823466e38f;
  for (int i = lane; i < parts; i += 64) top = fmaxf(top, p.part_ml[2 * (i * rows + row)]);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) top = fmaxf(top, __shfl_xor(top, s));
  float sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < parts; ++i) {
    const int64_t at = i * rows + row;
    const float e = __builtin_amdgcn_exp2f(p.part_ml[2 * at] - top);
    sum = fmaf(e, p.part_ml[2 * at + 1], sum);
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (64 * x + lane < d) o[x] = fmaf(e, p.part_o[at * d + 64 * x + lane], o[x]);
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  T *out = (T *)p.out + b * p.out_rs + h * p.out_hs;
#pragma unroll
  for (int x = 0; x < 4; ++x)
    if (64 * x + lane < d) store_f32(out + 64 * x + lane, sum == 0.f ? 0.f : o[x] * inv);
  if (p.lse && lane == 0) p.lse[row] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

}  // namespace

template <typename T> hipError_t mx_join(const MxTokenCall &p, hipStream_t s) {
  k_mx_join<T><<<(unsigned)(((int64_t)p.m.c.n_requests * p.q.n_q_heads + 3) / 4), 256, 0, s>>>(p);
  return hipGetLastError();
}

template hipError_t mx_join<float>(const MxTokenCall &, hipStream_t);
template hipError_t mx_join<bf16_t>(const MxTokenCall &, hipStream_t);

}  // namespace hyp
