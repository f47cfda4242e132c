// Joining what the parts of a request's keys gave for its row.
#include "mx_format.h"
#include "mx_rules.h"

namespace hyp {
namespace {

constexpr float kLn2 = 0.6931471805599453f;

// A workgroup for each row and query head, whose waves take parts in turn, eight at a time, a feature a lane (four times): what a call waits for is
// the first read of maxima and one or two rounds of reads of sums: 4 us for 16 requests of 32 heads in four parts.
constexpr int kJoinWaves = 4;
template <typename T> __global__ void __launch_bounds__(64 * kJoinWaves) k_mx_join(const MxTokenCall p) {
  __shared__ float lds[kJoinWaves][4][64];
  const hyp_mx_cache_t &c = p.m.c;
  const int64_t rows = (int64_t)c.n_requests * p.q.n_q_heads, row = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, b = (int)(row / p.q.n_q_heads), h = (int)(row % p.q.n_q_heads), d = c.head_dim;
  const int units = p.listed ? p.listed << (p.m.block_shift - p.unit) : (int)(((int64_t)mx_len(c, b) + (1 << p.unit) - 1) >> p.unit);
  const int parts = max(1, (int)(((int64_t)units + p.units - 1) / p.units));
  const float2 *ml = (const float2 *)p.part_ml;
  float top = -3.402823466e38f, sum = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = lane; i < parts; i += 64) top = fmaxf(top, ml[i * rows + row].x);
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) top = fmaxf(top, __shfl_xor(top, s));
  for (int i0 = 0; i0 < parts; i0 += 64) {
    float e = 0.f;                       // of part i0 + lane
    if (i0 + lane < parts) {
      const float2 x = ml[(i0 + lane) * rows + row];
      e = __builtin_amdgcn_exp2f(x.x - top);
      sum = fmaf(e, x.y, sum);
    }
    // those behind the last one again the last
    const int n = min(64, parts - i0);
    for (int j = wave; j < n; j += 8 * kJoinWaves) {
      float v[8][4];
#pragma unroll
      for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int x = 0; x < 4; ++x) v[k][x] = 64 * x + lane < d ? p.part_o[((i0 + min(j + k * kJoinWaves, n - 1)) * rows + row) * d + 64 * x + lane] : 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float w = __shfl(e, min(j + k * kJoinWaves, 63));
#pragma unroll
        for (int x = 0; x < 4; ++x) o[x] = j + k * kJoinWaves < n ? fmaf(w, v[k][x], o[x]) : o[x];
      }
    }
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) sum += __shfl_xor(sum, s);
#pragma unroll
  for (int x = 0; x < 4; ++x) lds[wave][x][lane] = o[x];
  __syncthreads();
  const int f = threadIdx.x;             // a feature a thread
  if (f >= d) return;
  float all = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) all += lds[w][f >> 6][f & 63];
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  store_f32((T *)p.out + b * p.out_rs + h * p.out_hs + f, sum == 0.f ? 0.f : all * inv);
  if (p.lse && f == 0) p.lse[row] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

}  // namespace

template <typename T> hipError_t mx_join(const MxTokenCall &p, hipStream_t s) {
  k_mx_join<T><<<(unsigned)p.m.c.n_requests * p.q.n_q_heads, 64 * kJoinWaves, 0, s>>>(p);
  return hipGetLastError();
}

template hipError_t mx_join<float>(const MxTokenCall &, hipStream_t);
template hipError_t mx_join<bf16_t>(const MxTokenCall &, hipStream_t);

}  // namespace hyp
