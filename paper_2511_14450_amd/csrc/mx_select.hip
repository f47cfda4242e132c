// Which blocks of a request's keys a row reads.
#include "mx_format.h"
#include "mx_rules.h"

namespace hyp {
namespace {

constexpr int kThreads = 256, kHeads = 4;  // query heads whose scores are formed at a time
constexpr int kItems = 4;  // blocks of a thread that chooses

typedef unsigned long long u64;

// Order of scores as unsigned numbers: -0 as 0, a NaN above all numbers.  0 and the highest are no score's: blocks that are not there, and
// those that are always taken.
__device__ __forceinline__ u64 order_of(double x) {
  const u64 u = (u64)__double_as_longlong(x);
  if ((u << 1) > 0xffe0000000000000ull) return ~0ull - 1;
  if ((u << 1) == 0) return 1ull << 63;
  return u ^ ((u >> 63) ? ~0ull : 1ull << 63);
}

template <int X> __device__ __forceinline__ u64 quad_xor(u64 u) {  // of the four lanes of a quad
  constexpr int ctrl = X == 1 ? 0xb1 : 0x4e;
  const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)u, ctrl, 0xf, 0xf, true);
  const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)(u >> 32), ctrl, 0xf, 0xf, true);
  return (u64)hi << 32 | lo;
}

// Features f .. f + 7 of a row of d as 64 bits, zeros from d on.  WIDE: whole pieces of 16 bytes; no branch is in the way of requesting several.
template <typename T, bool WIDE> struct Eight {
  static constexpr int N = sizeof(T) / 2;
  uint4 w[N];
  __device__ __forceinline__ void load(const T *row, int f, int d) {
    if constexpr (WIDE) {
      const uint4 *at = (const uint4 *)(row + min(f, d - 8));
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = at[i];
    } else {
      T x[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = f + i < d ? row[f + i] : (T)0;
      __builtin_memcpy(w, x, sizeof(x));
    }
  }
  __device__ __forceinline__ void get(int f, int d, double (&x)[8]) const {
    T y[8];
    __builtin_memcpy(y, w, sizeof(y));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = !WIDE || f < d ? (double)load_f32(y + i) : 0.0;
  }
};

// Features f .. f + 7 of a block's bound, two a word, as they lie in memory, zeros from d on
template <bool WIDE> __device__ __forceinline__ uint4 load_bound(const bf16_t *row, int f, int d) {
  if constexpr (WIDE) return *(const uint4 *)(row + min(f, d - 8));
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (f + 2 * i < d ? row[f + 2 * i] : 0u) | (f + 2 * i + 1 < d ? row[f + 2 * i + 1] : 0u) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ double element(const uint4 &v, int i, bool there) {
  const unsigned w = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w, x = i & 1 ? w & 0xffff0000u : w << 16;
  return (double)__uint_as_float(there ? x : 0u);
}

// Order of the scores of blocks first + 64 t + 16 wave + 0..15, t < kTurns, as far as `end`, of one request and KV head.  The sums are formed in 64
// bits, for which products of bf16 numbers are exact for all but wide spreads of sizes, so that the choice does not hang on their order.
// The vector unit has neither the time for that (a conversion of a float takes four ordinary instructions': 22 us for 64 caches of up to 2048
// blocks of 128 features) nor for the sums over lanes; the matrix unit's 4 x 4 x 4 product does both: 16 blocks on the M axis of its four
// batches, 4 heads on the N axis, lane l holds blocks l % 16 and heads l % 4 in four pieces of features, l / 16 of them, and gets the score of
// block 4 (l / 4 % 4) + l / 16 with head l % 4.  N pieces of eight features of a lane, 64 features of a row, are held at a time: with 128 two waves
// a SIMD instead of three (23.5 us a call, 22.7).  Those 64 caches, 53 MB of bounds, take 15.5 us: without the reads 10, of which the products
// and conversions are 6; what is left is waiting, for all workgroups run at once and each goes through four turns.
constexpr int kTurns = 4, N = 2;
struct Places { int page[kTurns], in[kTurns]; };  // of the blocks of a lane
__device__ __forceinline__ Places places_of(const MxSelectCall &p, int b, int first, int turns) {
  const hyp_mx_cache_t &c = p.m.c;
  Places at;
  first += 16 * __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) + (threadIdx.x & 15);
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    at.page[t] = b;
    at.in[t] = min(first + 64 * min(t, turns - 1), p.most_blocks - 1);  // there is room for these, held or not
  }
  if (c.page_table) {
    const int s = p.m.shift - p.m.block_shift;  // log2(blocks of a page)
#pragma unroll
    for (int t = 0; t < kTurns; ++t) at.page[t] = c.page_table[(int64_t)b * c.pages_per_request + (at.in[t] >> s)];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) at.in[t] &= (1 << s) - 1;
  }
  return at;
}

template <typename T, bool WIDE, typename Put>
__device__ __forceinline__ void score_blocks(const MxSelectCall &p, const Places &where, int b, int kvh, int first, int turns, int end, Put &&put) {
  const hyp_mx_cache_t &c = p.m.c;
  const int lane = threadIdx.x & 63, chunk = lane >> 4, d = c.head_dim, group = p.q.n_q_heads / c.n_kv_heads;
  first += 16 * __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (first >= end) return;
  const bf16_t *lo = (const bf16_t *)c.lo, *hi = (const bf16_t *)c.hi;
  int64_t at[kTurns];
#pragma unroll
  for (int t = 0; t < kTurns; ++t)
    at[t] = (c.page_table ? mx_clamped(where.page[t], 0, c.n_pages - 1) : b) * c.bound_page_stride + kvh * c.bound_head_stride + where.in[t] * c.bound_block_stride;
  for (int g0 = 0; g0 < group; g0 += kHeads) {
    const T *row = (const T *)p.q.q + b * p.q.q_row_stride + (kvh * group + min(g0 + (lane & 3), group - 1)) * p.q.q_head_stride;
    double up[kTurns], down[kTurns];     // sums over features whose largest numbers count, and whose least do
#pragma unroll
    for (int t = 0; t < kTurns; ++t) up[t] = down[t] = 0.0;
    for (int from = 0; from < d; from += 32 * N) {
      Eight<T, WIDE> raw[N];
      uint4 l[2][N], u[2][N];
      auto place = [&](int n) { return from + 32 * n + 8 * chunk; };
      auto request = [&](int t) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
          u[t & 1][n] = load_bound<WIDE>(hi + at[t], place(n), d);
          l[t & 1][n] = load_bound<WIDE>(lo + at[t], place(n), d);
        }
      };
#pragma unroll
      for (int n = 0; n < N; ++n) raw[n].load(row, place(n), d);
      request(0);
      double qu[N][8], ql[N][8];         // max(q, 0) and min(q, 0)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        double q[8];
        raw[n].get(place(n), d, q);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          qu[n][e] = q[e] < 0.0 ? 0.0 : q[e];  // NaN stays one in both
          ql[n][e] = q[e] > 0.0 ? 0.0 : q[e];
        }
      }
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        if (t > 0 && (t >= turns || first + 64 * t >= end)) break;
        if (t + 1 < kTurns) request(t + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            up[t] = __builtin_amdgcn_mfma_f64_4x4x4f64(element(u[t & 1][n], e, place(n) < d), qu[n][e], up[t], 0, 0, 0);
            down[t] = __builtin_amdgcn_mfma_f64_4x4x4f64(element(l[t & 1][n], e, place(n) < d), ql[n][e], down[t], 0, 0, 0);
          }
      }
    }
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      u64 best = order_of(up[t] + down[t]);
      best = max(best, quad_xor<1>(best));
      best = max(best, quad_xor<2>(best));
      const int i = first + 64 * t + 4 * ((lane >> 2) & 3) + chunk;
      if ((lane & 3) == 0 && t < turns && i < end) put(i, best, g0 > 0);
    }
  }
}

template <typename T, bool WIDE> __global__ void __launch_bounds__(kThreads, 2) k_mx_scores(const MxSelectCall p, int tiles, int turns) {
  const int tile = blockIdx.x % tiles, pair = blockIdx.x / tiles, b = pair / p.m.c.n_kv_heads, kvh = pair % p.m.c.n_kv_heads;
  const Places where = places_of(p, b, tile * 64 * turns, turns);  // waits for no length
  const int count = (int)(((int64_t)mx_len(p.m.c, b) + (1 << p.m.block_shift) - 1) >> p.m.block_shift);
  if (count <= p.keep) return;
  u64 *order = p.order + (int64_t)pair * p.most_blocks;
  score_blocks<T, WIDE>(p, where, b, kvh, tile * 64 * turns, turns, min(count, (tile + 1) * 64 * turns), [&](int i, u64 v, bool more) { order[i] = more ? max(order[i], v) : v; });
}

// sum of v over the threads before this one, and over all; scratch: one int a wave
template <int WAVES> __device__ __forceinline__ int before_me(int v, int *scratch, int &all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = v;
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    const int x = __shfl_up(upto, s);
    if (lane >= s) upto += x;
  }
  if (lane == 63) scratch[wave] = upto;
  __syncthreads();
  int before = upto - v;
  all = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    before += w < wave ? scratch[w] : 0;
    all += scratch[w];
  }
  __syncthreads();
  return before;
}

// One request and KV head with more blocks than are kept.  Scores are sorted into kBins bins between the least and the largest; the bin in which
// the last one falls that is taken is cut into as many again until it holds few, which are then ranked one by one.  Barriers bound it, some fifteen:
// 7 us for 64 pairs of up to 2048 blocks (88 where up to 1024 were ranked one by one).
template <int THREADS> __global__ void __launch_bounds__(THREADS) k_mx_choose(const MxSelectCall p) {
  constexpr int WAVES = THREADS / 64, kMostCandidates = THREADS / 8;
  constexpr int kBins = 2 * THREADS, kBits = 31 - __builtin_clz(kBins);  // two bins a thread
  __shared__ int hist[kBins], scratch[WAVES], found[3];
  __shared__ u64 ends[2], cand[kMostCandidates];
  __shared__ int cand_at[kMostCandidates];
  const int pair = blockIdx.x, b = pair / p.m.c.n_kv_heads, tid = threadIdx.x, lane = tid & 63, K = p.keep;
  const u64 *order = p.order + (int64_t)pair * p.most_blocks;
  u64 held[kItems];                      // the first orders, which wait for no length
#pragma unroll
  for (int x = 0; x < kItems; ++x) held[x] = order[min(tid * kItems + x, p.most_blocks - 1)];
  const int count = (int)(((int64_t)mx_len(p.m.c, b) + (1 << p.m.block_shift) - 1) >> p.m.block_shift);
  int *out = p.blocks + (int64_t)pair * K;
  if (count <= K) {
    for (int r = tid; r < K; r += THREADS) out[r] = r < count ? r : -1;
    return;
  }
  const int newest = count - p.recent;
  // a thread has runs of kItems blocks, so that counts in the order of threads are counts in the order of blocks
  constexpr int STEP = THREADS * kItems;
  const bool once = count <= STEP;
  u64 u[kItems];
  auto read = [&](int base) {
#pragma unroll
    for (int x = 0; x < kItems; ++x) {
      const int i = base + tid * kItems + x;
      u[x] = i >= count ? 0 : (i < p.sink || i >= newest) ? ~0ull : base == 0 ? held[x] : order[i];
    }
  };
  auto each = [&](auto &&f) {  // f(block, its order), for those with a score of their own
    for (int base = 0; base < count; base += STEP) {
      if (!once) read(base);
#pragma unroll
      for (int x = 0; x < kItems; ++x)
        if (u[x] != 0 && u[x] != ~0ull) f(base + tid * kItems + x, u[x]);
    }
  };
  if (once) read(0);
  const int always = p.sink + p.recent;
  int need = K - always;  // of the others; no block is both, for count > K >= always
  u64 from = ~0ull, to = 0;
  if (tid == 0) {
    ends[0] = ~0ull;
    ends[1] = 0;
  }
  __syncthreads();
  each([&](int, u64 v) {
    from = min(from, v);
    to = max(to, v);
  });
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    from = min(from, (u64)__shfl_xor((long long)from, s));
    to = max(to, (u64)__shfl_xor((long long)to, s));
  }
  if (lane == 0) {
    atomicMin(&ends[0], from);
    atomicMax(&ends[1], to);
  }
  __syncthreads();
  from = ends[0];
  to = ends[1];
  // taken: all above `to`, and `need` of [from, to]
  int inside = count - always;
  while (need > 0 && need < inside && inside > kMostCandidates && from < to) {
    const int shift = max(0, 64 - __clzll((long long)(to - from)) - kBits);
    hist[tid] = hist[tid + THREADS] = 0;
    __syncthreads();
    each([&](int, u64 v) {
      if (v >= from && v <= to) atomicAdd(&hist[(int)((v - from) >> shift)], 1);
    });
    __syncthreads();
    const int hi = kBins - 1 - 2 * tid, own0 = hist[hi], own1 = hist[hi - 1];
    int all;
    const int above = before_me<WAVES>(own0 + own1, scratch, all);
    if (above < need && need <= above + own0) {
      found[0] = hi;
      found[1] = above;
      found[2] = own0;
    } else if (above + own0 < need && need <= above + own0 + own1) {
      found[0] = hi - 1;
      found[1] = above + own0;
      found[2] = own1;
    }
    __syncthreads();
    need -= found[1];
    inside = found[2];
    const u64 base = from + ((u64)found[0] << shift);
    if (to - base >= 1ull << shift) to = base + ((1ull << shift) - 1);
    from = base;
    __syncthreads();
  }
  // of [from, to] `need` are taken: none, all, the first ones where all are equal, or the best by rank
  u64 last = from;       // least order that is taken
  int equal = 0x7fffffff;  // how many of that order are, from the first block on
  if (need <= 0) {
    last = to + 1;
  } else if (need < inside) {
    if (from == to) {
      equal = need;
    } else {
      if (tid == 0) found[0] = 0;
      __syncthreads();
      each([&](int i, u64 v) {
        if (v >= from && v <= to) {
          const int x = atomicAdd(&found[0], 1);
          cand[x] = v;
          cand_at[x] = i;
        }
      });
      __syncthreads();
      // eight threads a candidate, whose counts are joined by a butterfly
      const int x0 = tid >> 3;
      const u64 mine = x0 < inside ? cand[x0] : 0;
      const int at = x0 < inside ? cand_at[x0] : 0;
      int counts = 0;  // of those before it, and of those before it that are equal, in 16 bits each
      for (int x = tid & 7; x < inside; x += 8) {
        const u64 v = cand[x];
        const bool same = v == mine && cand_at[x] < at;
        counts += (v > mine || same ? 1 : 0) + (same ? 1 << 16 : 0);
      }
#pragma unroll
      for (int x = 1; x < 8; x <<= 1) counts += __shfl_xor(counts, x);
      if ((tid & 7) == 0 && x0 < inside && (counts & 0xffff) == need - 1) {  // the last one that is taken
        ends[0] = mine;
        found[1] = (counts >> 16) + 1;
      }
      __syncthreads();
      last = ends[0];
      equal = found[1];
    }
  }
  int done = 0, equals = 0;
  for (int base = 0; base < count; base += STEP) {
    if (!once) read(base);
    int mine = 0, all;
#pragma unroll
    for (int x = 0; x < kItems; ++x) mine += u[x] == last;
    int nth = equals + before_me<WAVES>(mine, scratch, all);
    equals += all;
    int taken = 0;
    unsigned which = 0;
#pragma unroll
    for (int x = 0; x < kItems; ++x) {
      const bool is = u[x] == last;
      const bool t = u[x] == ~0ull || (u[x] != 0 && (u[x] > last || (is && nth < equal)));
      nth += is;
      which |= (unsigned)t << x;
      taken += t;
    }
    int at = done + before_me<WAVES>(taken, scratch, all);
    done += all;
#pragma unroll
    for (int x = 0; x < kItems; ++x)
      if ((which >> x) & 1) out[at++] = base + tid * kItems + x;
  }
}

// The same for requests of up to 256 blocks, scores and choice in one launch: a block is taken if fewer than `keep` come before it.
template <typename T, bool WIDE> __global__ void __launch_bounds__(kThreads, 2) k_mx_select_small(const MxSelectCall p) {
  __shared__ u64 order[kMxSmallBlocks];
  __shared__ int scratch[kThreads / 64];
  const int pair = blockIdx.x, b = pair / p.m.c.n_kv_heads, kvh = pair % p.m.c.n_kv_heads, tid = threadIdx.x, K = p.keep;
  const Places where = places_of(p, b, 0, kTurns);
  const int count = (int)(((int64_t)mx_len(p.m.c, b) + (1 << p.m.block_shift) - 1) >> p.m.block_shift);
  int *out = p.blocks + (int64_t)pair * K;
  if (count <= K) {
    for (int r = tid; r < K; r += kThreads) out[r] = r < count ? r : -1;
    return;
  }
  score_blocks<T, WIDE>(p, where, b, kvh, 0, kTurns, count, [&](int i, u64 v, bool more) { order[i] = more ? max(order[i], v) : v; });
  __syncthreads();
  if (tid >= count) order[tid] = 0;
  else if (tid < p.sink || tid >= count - p.recent) order[tid] = ~0ull;
  __syncthreads();
  const u64 mine = order[tid];
  int before = 0;
  for (int i = 0; i < count; ++i) {
    const u64 v = order[i];
    before += v > mine || (v == mine && i < tid);
  }
  const int taken = tid < count && before < K;
  int all;
  const int at = before_me<kThreads / 64>(taken, scratch, all);
  if (taken) out[at] = tid;
}

template <typename T, bool WIDE> hipError_t select(const MxSelectCall &p, hipStream_t s) {
  const unsigned pairs = (unsigned)p.m.c.n_requests * p.m.c.n_kv_heads;
  if (mx_select_once(p.most_blocks, p.keep)) {
    k_mx_select_small<T, WIDE><<<pairs, kThreads, 0, s>>>(p);
    return hipGetLastError();
  }
  const int turns = mx_score_turns(pairs, p.most_blocks), tiles = mx_score_tiles(p.most_blocks, turns);
  k_mx_scores<T, WIDE><<<pairs * tiles, kThreads, 0, s>>>(p, tiles, turns);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;  // the choice goes by the scores
  if (p.most_blocks <= kMxChooseBlocks) k_mx_choose<512><<<pairs, 512, 0, s>>>(p);
  else k_mx_choose<1024><<<pairs, 1024, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

template <typename T> hipError_t mx_select(const MxSelectCall &p, hipStream_t s) {
  return p.wide ? select<T, true>(p, s) : select<T, false>(p, s);
}

template hipError_t mx_select<float>(const MxSelectCall &, hipStream_t);
template hipError_t mx_select<bf16_t>(const MxSelectCall &, hipStream_t);

}  // namespace hyp
