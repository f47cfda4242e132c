// Which keys of a request stay in its cache, and moving them there.
#include "span_kernels.h"

namespace hyp {
namespace {

constexpr int kSelectThreads = 1024, kMoveRows = 32;

typedef __attribute__((__vector_size__(16))) float f32x4_t;

__device__ __forceinline__ int clamped(int v, int lo, int hi) { return min(max(v, lo), hi); }

__device__ __forceinline__ int64_t key_offset(const hyp_attn_cache_t &c, int shift, int64_t page_stride, int64_t head_stride, int64_t key_stride, int req,
                                              int kvh, int j) {
  if (!c.page_table) return (int64_t)req * page_stride + (int64_t)kvh * head_stride + (int64_t)j * key_stride;
  const int page = clamped(c.page_table[(int64_t)req * c.pages_per_request + (j >> shift)], 0, c.n_pages - 1);
  return (int64_t)page * page_stride + (int64_t)kvh * head_stride + (int64_t)(j & (c.page_keys - 1)) * key_stride;
}

// Exclusive count of `flag` over the workgroup's threads before this one; total: over all.  Two barriers.
__device__ __forceinline__ int count_before(bool flag, int *waves, int &total) {
  const unsigned long long votes = __ballot(flag);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane == 0) waves[wave] = __popcll(votes);
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kSelectThreads / 64; ++w) {
    const int n = waves[w];
    before += w < wave ? n : 0;
    sum += n;
  }
  __syncthreads();
  total = sum;
  return before + __popcll(votes & ((1ull << lane) - 1));
}

// One request and KV head.  The keep-th largest total is found by four counts of eight bits each; then one pass in the order of
// the slots says who stays (of equal totals the lowest slots), which slots become free and which keys move there.
__global__ void __launch_bounds__(kSelectThreads) k_evict_select(const EvictCall p) {
  __shared__ int hist[256], waves[kSelectThreads / 64], found[2];
  const int b = blockIdx.x / p.c.n_kv_heads, kvh = blockIdx.x % p.c.n_kv_heads, tid = threadIdx.x, K = p.keep;
  const int len = clamped(p.c.lens[b], 0, p.c.most);
  int *kept = p.kept + (int64_t)blockIdx.x * K;
  if (len <= K) {
    for (int r = tid; r < K; r += kSelectThreads) kept[r] = r < len ? r : -1;
    return;
  }
  const float *totals = p.totals.in + b * p.totals.in_request_stride + kvh * p.totals.in_head_stride;
  const int *pos = p.c.key_pos ? p.c.key_pos + b * p.c.key_pos_request_stride + kvh * p.c.key_pos_head_stride : nullptr;
  const int64_t first = (int64_t)p.c.prefix_len + p.sink;
  const int64_t newest = (p.now ? (int64_t)p.now[b] : (int64_t)p.c.prefix_len + len) - p.recent;
  // order of the keys as unsigned numbers: a NaN lowest, -0 as 0, what is always kept highest
  auto rank = [&](int j) -> unsigned {
    const int64_t at = pos ? (int64_t)pos[j] : (int64_t)p.c.prefix_len + j;
    if (at < first || at >= newest) return 0xffffffffu;
    const unsigned u = __float_as_uint(totals[j]);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0u;
    if ((u & 0x7fffffffu) == 0u) return 0x80000000u;
    return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
  };
  unsigned prefix = 0, mask = 0;
  int need = K;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < len; j += kSelectThreads) {
      const unsigned u = rank(j);
      if ((u & mask) == prefix) atomicAdd(&hist[(u >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid < 64) {  // bins 4 lane .. 4 lane + 3, counted from the highest
      int own[4], sum = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) sum += own[x] = hist[255 - (4 * tid + x)];
      int upto = sum;
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const int v = __shfl_up(upto, s);
        if (tid >= s) upto += v;
      }
      int above = upto - sum;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (above < need && need <= above + own[x]) {
          found[0] = 255 - (4 * tid + x);
          found[1] = need - above;
        }
        above += own[x];
      }
    }
    __syncthreads();
    prefix |= (unsigned)found[0] << shift;
    mask |= 255u << shift;
    need = found[1];
    __syncthreads();
  }
  int *holes = p.list + (int64_t)blockIdx.x * 2 * K, *moved = holes + K;
  int equal = 0, n_holes = 0, n_moved = 0;
  for (int j0 = 0; j0 < len; j0 += kSelectThreads) {
    const int j = j0 + tid;
    const unsigned u = j < len ? rank(j) : 0u;
    const bool same = j < len && u == prefix;
    int n;
    const int nth = equal + count_before(same, waves, n);
    equal += n;
    const bool stays = j < len && (u > prefix || (same && nth < need));
    const bool hole = j < K && !stays, mover = j >= K && stays;
    if (j0 < K) {
      const int at = n_holes + count_before(hole, waves, n);
      n_holes += n;
      if (hole) holes[at] = j;
      else if (j < K) kept[j] = j;
    }
    if (j0 + kSelectThreads > K) {
      const int at = n_moved + count_before(mover, waves, n);
      n_moved += n;
      if (mover) moved[at] = j;
    }
  }
  __threadfence_block();
  __syncthreads();
  for (int i = tid; i < n_holes; i += kSelectThreads) kept[holes[i]] = moved[i];
}

// 32 slots of one request and KV head.
template <bool VEC, int ES> __global__ void __launch_bounds__(256) k_evict_move(const EvictCall p) {
  const int per = (p.keep + kMoveRows - 1) / kMoveRows;
  const int pair = blockIdx.x / per, r0 = (blockIdx.x % per) * kMoveRows;
  const int b = pair / p.c.n_kv_heads, kvh = pair % p.c.n_kv_heads, d = p.c.head_dim, rows = min(kMoveRows, p.keep - r0);
  const int *kept = p.kept + (int64_t)pair * p.keep + r0;
  if (threadIdx.x < rows) {
    const int r = r0 + threadIdx.x, src = kept[threadIdx.x];
    if (src >= 0 && !(p.in_place && src == r)) {
      p.totals.out[b * p.totals.out_request_stride + kvh * p.totals.out_head_stride + r] =
          p.totals.in[b * p.totals.in_request_stride + kvh * p.totals.in_head_stride + src];
      if (p.to.key_pos)
        p.to.key_pos[b * p.to.key_pos_request_stride + kvh * p.to.key_pos_head_stride + r] =
            p.c.key_pos ? p.c.key_pos[b * p.c.key_pos_request_stride + kvh * p.c.key_pos_head_stride + src] : p.c.prefix_len + src;
      if (p.to.key_doc)
        p.to.key_doc[b * p.to.key_doc_request_stride + kvh * p.to.key_doc_head_stride + r] =
            p.c.key_doc ? p.c.key_doc[b * p.c.key_doc_request_stride + kvh * p.c.key_doc_head_stride + src] : -1;
    }
  }
  const int pieces = VEC ? d * ES / 16 : d;
  for (int i = threadIdx.x; i < 2 * rows * pieces; i += 256) {
    const bool v = i >= rows * pieces;
    const int x = v ? i - rows * pieces : i, row = x / pieces, at = x - row * pieces, src = kept[row];
    if (src < 0 || (p.in_place && src == r0 + row)) continue;
    const char *from = (const char *)(v ? p.c.v : p.c.k);
    char *to = (char *)(v ? p.to.v : p.to.k);
    const int64_t so = v ? key_offset(p.c, p.page_shift, p.c.v_page_stride, p.c.v_head_stride, p.c.v_key_stride, b, kvh, src)
                         : key_offset(p.c, p.page_shift, p.c.k_page_stride, p.c.k_head_stride, p.c.k_key_stride, b, kvh, src);
    const int64_t to_o = v ? key_offset(p.to, p.to_page_shift, p.to.v_page_stride, p.to.v_head_stride, p.to.v_key_stride, b, kvh, r0 + row)
                           : key_offset(p.to, p.to_page_shift, p.to.k_page_stride, p.to.k_head_stride, p.to.k_key_stride, b, kvh, r0 + row);
    if constexpr (VEC) *(f32x4_t *)(to + to_o * ES + at * 16) = *(const f32x4_t *)(from + so * ES + at * 16);
    else if constexpr (ES == 2) ((uint16_t *)to)[to_o + at] = ((const uint16_t *)from)[so + at];
    else ((uint32_t *)to)[to_o + at] = ((const uint32_t *)from)[so + at];
  }
}

// after every reader of the old lengths
__global__ void k_evict_lens(const int *lens, int *to, int n, int most, int keep) {
  const int b = blockIdx.x * blockDim.x + threadIdx.x;
  if (b < n) to[b] = min(clamped(lens[b], 0, most), keep);
}

}  // namespace

hipError_t span_evict(const EvictCall &p, hipStream_t s) {
  const unsigned pairs = (unsigned)p.c.n_requests * p.c.n_kv_heads;
  k_evict_select<<<pairs, kSelectThreads, 0, s>>>(p);
  const unsigned blocks = pairs * ((p.keep + kMoveRows - 1) / kMoveRows);
  if (p.c.dtype == HYP_BF16) {
    if (p.vec) k_evict_move<true, 2><<<blocks, 256, 0, s>>>(p);
    else k_evict_move<false, 2><<<blocks, 256, 0, s>>>(p);
  } else {
    if (p.vec) k_evict_move<true, 4><<<blocks, 256, 0, s>>>(p);
    else k_evict_move<false, 4><<<blocks, 256, 0, s>>>(p);
  }
  k_evict_lens<<<(p.c.n_requests + 255) / 256, 256, 0, s>>>(p.c.lens, p.to.lens, p.c.n_requests, p.c.most, p.keep);
  return hipGetLastError();
}

}  // namespace hyp
