// Which keys of a request stay in its cache, and moving them there.
#include "span_kernels.h"

namespace hyp {
namespace {

constexpr int kSelectThreads = kEvictThreads, kMoveRows = kEvictRows;

typedef __attribute__((__vector_size__(16))) float f32x4_t;

__device__ __forceinline__ int clamped(int v, int lo, int hi) { return min(max(v, lo), hi); }

__device__ __forceinline__ int64_t key_offset(const hyp_attn_cache_t &c, int shift, int64_t page_stride, int64_t head_stride, int64_t key_stride, int req,
                                              int kvh, int j) {
  if (!c.page_table) return (int64_t)req * page_stride + (int64_t)kvh * head_stride + (int64_t)j * key_stride;
  const int page = clamped(c.page_table[(int64_t)req * c.pages_per_request + (j >> shift)], 0, c.n_pages - 1);
  return (int64_t)page * page_stride + (int64_t)kvh * head_stride + (int64_t)(j & (c.page_keys - 1)) * key_stride;
}

// Order of the keys as unsigned numbers: a NaN lowest, -0 as 0, what is always kept highest.  Where more are always kept than there is
// room for (positions say so, which are the caller's), only those count, in the order of their totals.
__device__ __forceinline__ unsigned order_of(float total, bool always, bool crowded) {
  const unsigned x = __float_as_uint(total);
  const unsigned order = (x & 0x7fffffffu) > 0x7f800000u ? 1u : (x & 0x7fffffffu) == 0u ? 0x80000000u : x ^ ((x >> 31) ? 0xffffffffu : 0x80000000u);
  return crowded ? (always ? order : 0u) : (always ? 0xffffffffu : order);
}

// One request and KV head.  The keep-th largest total is found by three counts of 11, 11 and 10 bits; then one look at the totals in the
// order of the slots says who stays (of equal totals the lowest slots), which slots become free and which keys move there.  A thread has
// eight keys of each 8192, 1024 apart: up to so many keys are read once and stay in registers, more are read for every look.  Latency
// bounds it, of the one read and of about twenty barriers: 64 caches of 8192 keys take 16 us; a read for each of four counts and barriers for
// every 1024 keys took 27 us.
constexpr int kItems = 8, kBlock = kSelectThreads * kItems, kWaves = kSelectThreads / 64;
__global__ void __launch_bounds__(kSelectThreads) k_evict_select(const EvictCall p) {
  __shared__ int hist[2048], before[kItems * kWaves], before2[kItems * kWaves], found[2], wave_sum[kWaves];
  const int b = blockIdx.x / p.c.n_kv_heads, kvh = blockIdx.x % p.c.n_kv_heads, tid = threadIdx.x, K = p.keep, lane = tid & 63, wave = tid >> 6;
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
  unsigned u[kItems];
  bool crowded = false;
  auto read = [&](int block) {
    float t[kItems];
    int at[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int j = min(block + i * kSelectThreads + tid, len - 1);
      t[i] = totals[j];
      at[i] = pos ? pos[j] : p.c.prefix_len + j;
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) u[i] = order_of(t[i], at[i] < first || at[i] >= newest, crowded);
  };
  const bool once = len <= kBlock;
  if (once) read(0);
  unsigned prefix = 0, mask = 0;
  int need = K;
  for (int look = 0; look < 3; ++look) {
    const int shift = look == 0 ? 21 : look == 1 ? 10 : 0, bins = look == 2 ? 1024 : 2048;
    hist[tid] = hist[tid + 1024] = 0;
    __syncthreads();
    for (int block = 0; block < len; block += kBlock) {
      if (!once) read(block);
#pragma unroll
      for (int i = 0; i < kItems; ++i)
        if (block + i * kSelectThreads + tid < len && (u[i] & mask) == prefix) atomicAdd(&hist[(u[i] >> shift) & (bins - 1)], 1);
    }
    __syncthreads();
    // two bins a thread, counted from the highest; the bin in which the need is met
    const int hi = bins - 1 - 2 * tid, own0 = hi > 0 ? hist[hi] : 0, own1 = hi > 0 ? hist[hi - 1] : 0;
    int upto = own0 + own1;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const int v = __shfl_up(upto, s);
      if (lane >= s) upto += v;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    int above = upto - own0 - own1;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) above += w < wave ? wave_sum[w] : 0;
    if (above < need && need <= above + own0) {
      found[0] = hi;
      found[1] = need - above;
    } else if (above + own0 < need && need <= above + own0 + own1) {
      found[0] = hi - 1;
      found[1] = need - above - own0;
    }
    __syncthreads();
    if (look == 0 && found[0] == 2047 && !crowded) {  // only what is always kept is up there
      crowded = true;
      if (once) read(0);
      look = -1;
      continue;
    }
    prefix |= (unsigned)found[0] << shift;
    mask |= (unsigned)(bins - 1) << shift;
    need = found[1];
  }
  int *holes = p.list + (int64_t)blockIdx.x * 2 * K, *moved = holes + K;
  const unsigned long long below = (1ull << lane) - 1;
  // votes of eight flags to the count of all flags of lower slots in this block; base: of the blocks before, moved on
  auto count = [&](const unsigned long long (&votes)[kItems], int *where, int &base, int (&out)[kItems]) {
    if (lane == 0) {
#pragma unroll
      for (int i = 0; i < kItems; ++i) where[i * kWaves + wave] = __popcll(votes[i]);
    }
    __syncthreads();
    if (wave == 0) {  // 128 counts, two a lane
      const int x = where[2 * lane], y = where[2 * lane + 1];
      int upto = x + y;
#pragma unroll
      for (int s = 1; s < 64; s <<= 1) {
        const int v = __shfl_up(upto, s);
        if (lane >= s) upto += v;
      }
      where[2 * lane] = upto - x - y;
      where[2 * lane + 1] = upto - y;
      if (lane == 63) found[0] = upto;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; ++i) out[i] = base + where[i * kWaves + wave] + __popcll(votes[i] & below);
    base += found[0];
  };
  int equal = 0, n_holes = 0, n_moved = 0;
  for (int block = 0; block < len; block += kBlock) {
    if (!once) read(block);
    unsigned long long votes[kItems], hole_votes[kItems], move_votes[kItems];
    int nth[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) votes[i] = __ballot(block + i * kSelectThreads + tid < len && u[i] == prefix);
    count(votes, before, equal, nth);
    unsigned stays = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int j = block + i * kSelectThreads + tid;
      const bool s = j < len && (u[i] > prefix || (u[i] == prefix && nth[i] < need));
      stays |= (unsigned)s << i;
      hole_votes[i] = __ballot(j < K && !s);
      move_votes[i] = __ballot(j >= K && s);
    }
    int hole_at[kItems], move_at[kItems];
    __syncthreads();
    count(hole_votes, before2, n_holes, hole_at);
    __syncthreads();
    count(move_votes, before, n_moved, move_at);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int j = block + i * kSelectThreads + tid;
      const bool s = (stays >> i) & 1;
      if (j < K) {
        if (s) kept[j] = j;
        else holes[hole_at[i]] = j;
      } else if (s) {
        moved[move_at[i]] = j;
      }
    }
    __syncthreads();
  }
  __threadfence_block();
  __syncthreads();
  for (int i = tid; i < n_holes; i += kSelectThreads) kept[holes[i]] = moved[i];
}

// The same for up to 256 keys, and their move, in one launch: a key stays if fewer than `keep` come before it, counted one by one.  Latency
// bounds it, 9 us for caches of 96 keys.  A call takes 12 us for 96 keys, 17 for 256; in two launches 17 for either, and for 512 (25 in one).
constexpr int kSmall = kEvictSmall;
template <bool VEC, int ES> __device__ void move_rows(const EvictCall &p, int b, int kvh, int r0, int rows, const int *kept, int threads);

template <bool VEC, int ES> __global__ void __launch_bounds__(kSmall) k_evict_small(const EvictCall p) {
  __shared__ unsigned rank[kSmall];
  __shared__ int from[kSmall], holes[kSmall], moved[kSmall], waves[2][kSmall / 64];
  const int b = blockIdx.x / p.c.n_kv_heads, kvh = blockIdx.x % p.c.n_kv_heads, tid = threadIdx.x, K = p.keep, lane = tid & 63, wave = tid >> 6;
  const int len = clamped(p.c.lens[b], 0, p.c.most);
  int *kept = p.kept + (int64_t)blockIdx.x * K;
  for (int r = tid; r < K; r += kSmall)
    if (len <= K || r >= kSmall) kept[r] = r < len ? r : -1;
  from[tid] = tid < len && tid < K ? tid : -1;
  if (len > K) {
    unsigned u = 0;
    bool always = false;
    float total = 0.f;
    if (tid < len) {
      const int at = p.c.key_pos ? p.c.key_pos[b * p.c.key_pos_request_stride + kvh * p.c.key_pos_head_stride + tid] : p.c.prefix_len + tid;
      const int64_t newest = (p.now ? (int64_t)p.now[b] : (int64_t)p.c.prefix_len + len) - p.recent;
      total = p.totals.in[b * p.totals.in_request_stride + kvh * p.totals.in_head_stride + tid];
      always = at < (int64_t)p.c.prefix_len + p.sink || at >= newest;
      u = order_of(total, always, false);
    }
    rank[tid] = u;
    if (__syncthreads_count(always) > K) {
      u = tid < len ? order_of(total, always, true) : 0u;
      rank[tid] = u;
      __syncthreads();
    }
    int before = 0;
    for (int i = 0; i < len; i += 4) {  // ranks behind the last key are 0 and come last
      const uint4 x = *(const uint4 *)&rank[i];
      before += (x.x > u || (x.x == u && i < tid)) + (x.y > u || (x.y == u && i + 1 < tid)) + (x.z > u || (x.z == u && i + 2 < tid)) + (x.w > u || (x.w == u && i + 3 < tid));
    }
    const bool stays = tid < len && before < K, hole = tid < K && !stays, mover = tid >= K && stays;
    const unsigned long long hv = __ballot(hole), mv = __ballot(mover), below = (1ull << lane) - 1;
    if (lane == 0) {
      waves[0][wave] = __popcll(hv);
      waves[1][wave] = __popcll(mv);
    }
    __syncthreads();
    int h = __popcll(hv & below), m = __popcll(mv & below), n = 0;
#pragma unroll
    for (int w = 0; w < kSmall / 64; ++w) {
      h += w < wave ? waves[0][w] : 0;
      m += w < wave ? waves[1][w] : 0;
      n += waves[0][w];
    }
    if (hole) holes[h] = tid;
    if (mover) moved[m] = tid;
    __syncthreads();
    if (tid < n) from[holes[tid]] = moved[tid];
    __syncthreads();
    if (tid < K) kept[tid] = from[tid];
  }
  __syncthreads();
  move_rows<VEC, ES>(p, b, kvh, 0, min(K, kSmall), from, kSmall);
}

// 32 slots of one request and KV head.  Bytes bound it: 64 caches of 1024 keys of 128 bf16 features that stay take 13 us, 5.1 TB/s.
template <bool VEC, int ES> __global__ void __launch_bounds__(256) k_evict_move(const EvictCall p) {
  const int per = (p.keep + kMoveRows - 1) / kMoveRows;
  const int pair = blockIdx.x / per, r0 = (blockIdx.x % per) * kMoveRows;
  move_rows<VEC, ES>(p, pair / p.c.n_kv_heads, pair % p.c.n_kv_heads, r0, min(kMoveRows, p.keep - r0), p.kept + (int64_t)pair * p.keep + r0, 256);
}

// Rows r0 .. r0 + rows - 1 of the result: kept[r - r0] says where each comes from.
template <bool VEC, int ES> __device__ void move_rows(const EvictCall &p, int b, int kvh, int r0, int rows, const int *kept, int threads) {
  // what chose the keys was the last to read the old length
  if (kvh == 0 && r0 == 0 && threadIdx.x == 0) p.to.lens[b] = min(clamped(p.c.lens[b], 0, p.c.most), p.keep);
  if ((int)threadIdx.x < rows) {
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
  const int d = p.c.head_dim, pieces = VEC ? d * ES / 16 : d;
  for (int i = threadIdx.x; i < 2 * rows * pieces; i += threads) {
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

}  // namespace

template <bool VEC, int ES> static hipError_t evict(const EvictCall &p, hipStream_t s) {
  const unsigned pairs = (unsigned)p.c.n_requests * p.c.n_kv_heads;
  if (span_evict_once(p)) {
    k_evict_small<VEC, ES><<<pairs, kSmall, 0, s>>>(p);
    return hipGetLastError();
  }
  k_evict_select<<<pairs, kSelectThreads, 0, s>>>(p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;  // the move goes by what the selection wrote
  k_evict_move<VEC, ES><<<pairs * ((p.keep + kMoveRows - 1) / kMoveRows), 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t span_evict(const EvictCall &p, hipStream_t s) {
  if (p.c.dtype == HYP_BF16) return p.vec ? evict<true, 2>(p, s) : evict<false, 2>(p, s);
  return p.vec ? evict<true, 4>(p, s) : evict<false, 4>(p, s);
}

}  // namespace hyp
