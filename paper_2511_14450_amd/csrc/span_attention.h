// Kernels of attention over a shared prefix and a request's own keys (hyp_attn.h), for T = float or bf16_t.  Included by one
// translation unit per type.
#pragma once

#include <atomic>
#include <type_traits>

#include "span_core.h"
#include "span_survey.h"

namespace hyp {
namespace {

// The request of a row tile, its rows and its own keys.
struct TileRequest { int req, row0, rows, len, see_all; int64_t first; };  // first: the tile's first pair inside the request, -1: none

// Request b's tiles start at floor(q_start[b] G / tile) + b, which leaves each as many as it needs, or one more.  The lanes look at 64
// requests each, all that is to be known of them requested at once, where a bisection has a round trip to memory for each halving.
__device__ __forceinline__ TileRequest tile_request(const SpanCall &p, int t, int tile) {
  const int n = p.c.n_requests, lane = threadIdx.x & 63;
  auto cut = [&](int v) { return (int)min(max((int64_t)v, (int64_t)0), p.n_rows); };
  auto first_tile = [&](int row, int b) { return (int64_t)row * p.G / tile + b; };
  int base = 0;
  while (base + 64 < n && first_tile(uniform(cut(p.q_start[base + 64])), base + 64) <= t) base += 64;
  const int b = min(base + lane, n - 1);
  const int from = cut(p.q_start[b]), to = cut(p.q_start[b + 1]), len = span_len(p, b), all = p.see_all ? p.see_all[b] : 0;
  const unsigned long long votes = __ballot(first_tile(from, b) <= t);
  const int who = max(63 - __builtin_clzll(votes | 1), 0);
  TileRequest x;
  x.req = min(base + who, n - 1);
  x.row0 = __builtin_amdgcn_readlane(from, who);
  x.rows = max(__builtin_amdgcn_readlane(to, who) - x.row0, 0);
  x.len = __builtin_amdgcn_readlane(len, who);
  x.see_all = __builtin_amdgcn_readlane(all, who);
  const int64_t first = ((int64_t)t - first_tile(x.row0, x.req)) * tile;
  x.first = first >= 0 && first < (int64_t)x.rows * p.G ? first : -1;
  return x;
}

// Which head and item a workgroup has.  Workgroups go to the eight XCDs in turn, each with an L2 of its own: whole heads to one XCD
// while there are eight of them, so that it meets one head's keys at a time; of the r heads that are left an XCD gets every 8 / r-th
// item of one, or, where r does not divide 8, whatever comes.
__device__ __forceinline__ bool head_item(int id, int heads, int items, int &head, int &item) {
  const int x = id & 7, i = id >> 3, whole = heads >> 3, r = heads & 7;
  if (i < whole * items) {
    head = 8 * (i / items) + x;
    item = i % items;
    return true;
  }
  const int j = i - whole * items;
  if (r == 1 || r == 2 || r == 4) {
    head = 8 * whole + x % r;
    item = j * (8 / r) + x / r;
  } else {
    head = 8 * whole + (8 * j + x) % r;
    item = (8 * j + x) / r;
  }
  return item < items;
}

// attn_prompt.  A workgroup: one KV head, rows of one request (dense over the group's heads), all the keys they see or one of `splits` parts
// of them: 128 rows, 32 a wave, whose waves meet the same keys.  Two workgroups a CU, so that one's softmax runs beside the other's
// products; keys and values of the next stage are fetched straight into LDS meanwhile.  A score costs about thirteen vector instructions
// (two of them its exponential's and sum's, five a cap's) and a 16th of a matrix instruction for each 16 features: with 128 features the
// vector unit is busy for 0.55 of the time and the matrix unit for 0.3, and the two overlap less than half.  4 x 8192 causal rows of 40 heads of 128
// bf16 features: 3.7 ms capped (0.75 PFLOP/s), 3.2 ms not.  Tiles of 32 rows whose waves share the keys, for calls of few tiles:
// 920 f32 rows took 58 us, these 42, since each tile fetches the keys again.
template <typename T, int NT, bool WIDE>
__global__ void __launch_bounds__(64 * kSpanWaves, span_steps_waves(NT)) k_span_prompt(const SpanCall p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  using S = Span<T, NT, kSpanWaves, 1, span_stage_keys(NT, sizeof(T)), 2, WIDE>;
  int kvh, item;
  if (!head_item(blockIdx.x, p.c.n_kv_heads, p.tiles * p.splits, kvh, item)) return;
  const int split = p.splits > 1 ? item % p.splits : 0;
  const TileRequest q = tile_request(p, p.tiles - 1 - (p.splits > 1 ? item / p.splits : item), kSpanTile);  // the longest rows of a request first
  if (q.first < 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = threadIdx.x & 31;
  const int64_t pair = q.first + wave * 32 + col;
  const bool there = pair < (int64_t)q.rows * p.G;
  const int i = there ? (p.g_shift >= 0 ? (int)pair >> p.g_shift : (int)pair / p.G) : 0, g = there ? (int)(pair - (int64_t)i * p.G) : 0;
  const SpanRow r = span_row(p, q.row0 + i, kvh * p.G + g, q.req, q.len - q.rows + i, there);
  // the last row's reach, and the keys all of the request's rows see
  const int last_pair = (int)min(q.first + kSpanTile, (int64_t)q.rows * p.G) - 1, last = p.g_shift >= 0 ? last_pair >> p.g_shift : last_pair / p.G;
  const int end = max(q.len - q.rows + last + 1, q.see_all);
  S span(p, SpanKeys{0, p.c.prefix_len, 0, clamped(end, 0, q.len), q.req, kvh}, lds);
  const Survey<S> way(span, lds + S::LDS_ALL, r);
  typename S::State t;
  span.attend(part_start(span.stages, split, p.splits), part_start(span.stages, split + 1, p.splits), r, t, nullptr, way);
  span.store_rows(r, t, split);
}

// attn_token.  Items over the shared keys, which all requests' rows meet at once, then items of up to 32 rows of one request
// over its own keys, whose waves take turns at them.  The keys' bytes bound it: 8 requests of 9216 own keys, 8 heads of 128 bf16 features in
// pages of 128, take 54 us, 5.5 TB/s.  With one stage in LDS two workgroups fit a CU, and one's loads run beside the other's products; two
// stages and one workgroup took 86 us.  32 requests behind 8192 shared keys, 10 heads: 30 us, 2.9 TB/s - there the items are short, and a
// third of their time is the way to the first key and from the last.
template <typename T, int NT, bool WIDE> __global__ void __launch_bounds__(64 * span_token_waves(NT, sizeof(T)), span_steps_waves(NT)) k_span_token(const SpanCall p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  constexpr int NW = span_token_waves(NT, sizeof(T));
  using Own = Span<T, NT, 1, NW, 32, 1, WIDE>;
  using Pre = Span<T, NT, NW, 1, span_stage_keys(NT, sizeof(T)), 2, WIDE>;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = threadIdx.x & 31;
  int id = blockIdx.x;
  const bool pre = id < p.pre_items;
  if (!pre) id -= p.pre_items;
  const int kvh = id % p.c.n_kv_heads;
  id /= p.c.n_kv_heads;
  const int all = p.c.n_requests * p.G;  // pairs of a KV head
  if (pre) {
    const int split = id % p.pre_splits, tile = id / p.pre_splits;
    if (p.pre_wide) {
      const int pair = tile * 32 * NW + wave * 32 + col;
      const bool there = pair < all;
      const int b = there ? (p.g_shift >= 0 ? pair >> p.g_shift : pair / p.G) : 0;
      const SpanRow r = span_row(p, b, kvh * p.G + (there ? pair - b * p.G : 0), b, span_len(p, b) - 1, there);
      Pre span(p, SpanKeys{0, p.c.prefix_len, 0, 0, 0, kvh}, lds);
      typename Pre::State t;
      span.attend(part_start(span.stages, split, p.pre_splits), part_start(span.stages, split + 1, p.pre_splits), r, t, nullptr, EveryStage{0x7fffffff});
      span.store_rows(r, t, split);
      return;
    }
    const int pair = tile * 32 + col;
    const bool there = pair < all;
    const int b = there ? (p.g_shift >= 0 ? pair >> p.g_shift : pair / p.G) : 0;
    const SpanRow r = span_row(p, b, kvh * p.G + (there ? pair - b * p.G : 0), b, span_len(p, b) - 1, there);
    Own span(p, SpanKeys{0, p.c.prefix_len, 0, 0, 0, kvh}, lds);
    typename Own::State t;
    span.attend(part_start(span.stages, split, p.pre_splits), part_start(span.stages, split + 1, p.pre_splits), r, t, nullptr, EveryStage{0x7fffffff});
    span.join_waves(t, r, min(32, all - tile * 32), split);
    return;
  }
  const int split = id % p.splits;
  id /= p.splits;
  const int tile = id % p.tiles, b = id / p.tiles;
  const int g = tile * 32 + col, rows = min(32, p.G - tile * 32);
  const bool there = col < rows;
  const int len = uniform(span_len(p, b));
  const SpanRow r = span_row(p, b, kvh * p.G + (there ? g : 0), b, len - 1, there);
  Own span(p, SpanKeys{0, 0, 0, len, b, kvh}, lds);
  typename Own::State t;
  float *scores = p.scores ? p.scores + (((int64_t)b * p.c.n_kv_heads + kvh) * p.G + (there ? g : 0)) * p.score_pitch : nullptr;
  span.attend(part_start(span.stages, split, p.splits), part_start(span.stages, split + 1, p.splits), r, t, scores, EveryStage{span.has_doc ? 0 : 0x7fffffff});
  span.join_waves(t, r, rows, p.pre_splits + split);
}

// (maximum, sum) of a row's partial results, in every lane; mine: the weight of the result in slot `lane`, where there is one, over 2^maximum
__device__ __forceinline__ float2 slots_total(const SpanCall &p, int slots, int64_t pair, int lane, float &mine) {
  const int64_t all = p.n_rows * p.nq;
  const float2 *ml = (const float2 *)p.part_ml;
  const float2 first = lane < slots ? ml[lane * all + pair] : float2{-INFINITY, 0.f};
  float m = first.x;
  for (int s = lane + 64; s < slots; s += 64) m = fmaxf(m, ml[s * all + pair].x);
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
  mine = is_none(first.x) ? 0.f : exp2_(first.x - m) * first.y;
  float l = mine;
  for (int s = lane + 64; s < slots; s += 64) {
    const float2 x = ml[s * all + pair];
    if (!is_none(x.x)) l += exp2_(x.x - m) * x.y;
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) l += __shfl_xor(l, x);
  return {not_finite(l) ? l : m, l};  // a maximum passes over NaN
}

// Partial results to results, a wave a row, V features a lane; eight of a row's partial results are requested before the first is waited for.
// Bytes bound it: seven parts of 920 f32 rows of 8 heads of 128 features take 8 us, 18 of 32 bf16 requests with their totals 6.6 us.
template <typename T, int V> __device__ __forceinline__ void join_row(const SpanCall &p, int slots, int64_t pair, int lane) {
  const int d = p.c.head_dim, f = lane * V;
  const int64_t all = p.n_rows * p.nq, row = all >> 32 ? pair / p.nq : (int64_t)((unsigned)pair / (unsigned)p.nq);
  const int head = (int)(pair - row * p.nq);
  if (p.q_start && (row < p.q_start[0] || row >= p.q_start[p.c.n_requests])) return;  // no request's row
  float weight;
  const float2 ml = slots_total(p, slots, pair, lane, weight);
  const bool none = is_none(ml.x);
  if (p.lse && lane == 0) p.lse[pair] = none ? -INFINITY : (ml.x + __builtin_amdgcn_logf(ml.y)) * kLn2;
  const float inv = none ? 0.f : 1.0f / ml.y;
  float acc[V] = {};
  const bool on = f < d;  // V divides d
  // slots that hold something: those of the first 64 by a look at their weights, which all lanes have; an empty slot holds nothing, not
  // even zeros
  unsigned long long live = __ballot(!is_zero(weight));
  for (int next = 64; live || next < slots;) {
    float o[8][V], w[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      w[u] = 0.f;
      int s = slots;
      if (live) {
        s = __builtin_ctzll(live);
        live &= live - 1;
        w[u] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), s));
      } else if (next < slots) {
        s = next++;
        const float2 x = ((const float2 *)p.part_ml)[s * all + pair];
        w[u] = is_none(x.x) ? 0.f : exp2_(x.x - ml.x) * x.y;
      }
      if (s < slots) {
        const float *src = p.part_o + (s * all + pair) * d + f;
#pragma unroll
        for (int e = 0; e < V; ++e) o[u][e] = on ? src[e] : 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (!is_zero(w[u])) {
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = fmaf(w[u] * inv, o[u][e], acc[e]);
      }
  }
  if (!on) return;
  T *out = (T *)p.out + row * p.out_rs + head * p.out_hs + f;
#pragma unroll
  for (int e = 0; e < V; ++e) store_f32(out + e, acc[e]);
}

// The same for head sizes that neither two nor four features a lane fit.
template <typename T> __device__ __forceinline__ void join_odd(const SpanCall &p, int slots, int64_t pair, int lane) {
  const int d = p.c.head_dim;
  const int64_t all = p.n_rows * p.nq, row = all >> 32 ? pair / p.nq : (int64_t)((unsigned)pair / (unsigned)p.nq);
  const int head = (int)(pair - row * p.nq);
  if (p.q_start && (row < p.q_start[0] || row >= p.q_start[p.c.n_requests])) return;
  float weight;
  const float2 ml = slots_total(p, slots, pair, lane, weight);
  const bool none = is_none(ml.x);
  if (p.lse && lane == 0) p.lse[pair] = none ? -INFINITY : (ml.x + __builtin_amdgcn_logf(ml.y)) * kLn2;
  for (int f = lane; f < d; f += 64) {
    float acc = 0.f;
    for (int s = 0; s < slots; ++s) {
      const float2 x = ((const float2 *)p.part_ml)[s * all + pair];
      if (!is_none(x.x)) acc = fmaf(exp2_(x.x - ml.x) * x.y / ml.y, p.part_o[(s * all + pair) * d + f], acc);
    }
    store_f32((T *)p.out + row * p.out_rs + head * p.out_hs + f, acc);
  }
}

// ... and for attn_token the weight that own keys got, 1024 of one request and KV head to a workgroup.
template <typename T> __global__ void __launch_bounds__(256) k_span_join(const SpanCall p, int slots) {
  __shared__ float lse2[256];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, d = p.c.head_dim;
  if ((int)blockIdx.x < p.join_items) {
    const int64_t pair = (int64_t)blockIdx.x * 4 + wave;
    if (pair >= p.n_rows * p.nq) return;
    if (d <= 64) join_row<T, 1>(p, slots, pair, lane);
    else if (d <= 128 && (d & 1) == 0) join_row<T, 2>(p, slots, pair, lane);
    else if ((d & 3) == 0) join_row<T, 4>(p, slots, pair, lane);
    else join_odd<T>(p, slots, pair, lane);
    return;
  }
  const int blocks = (p.c.most + 1023) / 1024;
  int id = blockIdx.x - p.join_items;
  const int kb = id % blocks;
  id /= blocks;
  const int kvh = id % p.c.n_kv_heads, b = id / p.c.n_kv_heads;
  const int len = uniform(span_len(p, b)), j = kb * 1024 + threadIdx.x * 4;
  const float *in = p.totals.in + b * p.totals.in_request_stride + kvh * p.totals.in_head_stride;
  float *out = p.totals.out + b * p.totals.out_request_stride + kvh * p.totals.out_head_stride;
  float sum[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) sum[e] = j + e < p.c.most ? in[j + e] : 0.f;
  if (kb * 1024 < len) {
    for (int g = wave; g < p.G; g += 4) {
      float weight;
      const float2 ml = slots_total(p, slots, (int64_t)b * p.nq + kvh * p.G + g, lane, weight);
      if (lane == 0) lse2[g] = is_none(ml.x) ? INFINITY : ml.x + __builtin_amdgcn_logf(ml.y);
    }
  }
  __syncthreads();
  const float *scores = p.scores + ((int64_t)b * p.c.n_kv_heads + kvh) * p.G * p.score_pitch + j;
  if (j < len) {
    f32x4_t w = {0.f, 0.f, 0.f, 0.f};
    for (int g0 = 0; g0 < p.G; g0 += 4) {
      f32x4_t s[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (g0 + u < p.G) s[u] = *(const f32x4_t *)(scores + (g0 + u) * p.score_pitch);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (g0 + u < p.G) {
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] += exp2_(s[u][e] - lse2[g0 + u]);
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < len) sum[e] += w[e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e < p.c.most) out[j + e] = sum[e];
}

// attn_received.  A workgroup: a block of KEYS own keys of a request and KV head, or one from the front and one from the back, so
// that all workgroups have about the same number of rows to meet.  Half of its NW waves hold one half of the keys in registers, half the
// other; a head's rows pass by through LDS, ROWS at a time, from the last to the first, so that the workgroups of an XCD meet the same rows
// at about the same time.  What a key gets is summed in its lane over the rows, then over lanes and waves, in a fixed order.
// Rows come from L2 for every block of keys: 64 keys of 128 bf16 features to a block made that the bound (4.5 TB/s), and 6007 capped rows of
// 40 heads took 1.7 ms; with 128 keys they take 0.42 (0.44 PFLOP/s), the vector unit busy for 0.51 of the time, the matrix unit for 0.18, and the waves
// waiting for a third of theirs: eight waves a CU, and a barrier for every 128 rows.
// Where few rows count (8 requests, their last 32 rows, 12 K keys) there is a stage to a workgroup, 26 us for two rounds of workgroups
// that each wait for their keys.
template <typename T, int NT, bool WIDE, int ROWS, int KB, int NW> struct Received {
  using S = Span<T, NT, NW, 1, 32, 1, WIDE>;
  static constexpr int ES = sizeof(T), EPC = 16 / ES, KEYS = 64 * KB, THREADS = 64 * NW, TILE = ROWS * S::ROWB;
  static constexpr int SHARE = ((NW / 2) * KEYS * 4 + 2 * KEYS * 4 + 1023) / 1024 * 1024, LDS_ONE = SHARE + TILE, LDS = LDS_ONE + TILE;
  static constexpr int LOADS = ROWS * S::CPR / THREADS, STEP = THREADS / S::CPR;  // a lane's loads of a stage, and the rows between them
  static constexpr int TILES = ROWS / 32 / (NW / 2);                              // of a wave in a stage
  static_assert(LOADS * THREADS == ROWS * S::CPR && TILES >= 1 && LDS <= 160 * 1024, "a stage is whole loads of all waves, and whole tiles");

  const SpanCall &p;
  S span;
  char *lds;
  int wave, lane, hh, col, kvh, b, len, n, from, pairs, all;
  int64_t row0;

  __device__ __forceinline__ Received(const SpanCall &p_, char *lds_, int kvh_, int b_, int len_)
      : p(p_), span(p_, SpanKeys{0, 0, 0, len_, b_, kvh_}, lds_), lds(lds_), kvh(kvh_), b(b_), len(len_) {
    wave = span.wave; lane = span.lane; hh = span.hh; col = span.col;
    row0 = uniform((int)min(max((int64_t)p.q_start[b], (int64_t)0), p.n_rows));
    const int64_t row1 = uniform((int)max(min((int64_t)p.q_start[b + 1], p.n_rows), row0));
    n = (int)(row1 - row0);
    all = p.see_all ? clamped(uniform(p.see_all[b]), 0, len) : 0;
  }
  __device__ __forceinline__ void place(int pair, int &row, int &head) const {  // of a pair of the rows that count
    const int r = p.g_shift >= 0 ? pair >> p.g_shift : pair / p.G;
    row = (int)row0 + from + r;
    head = kvh * p.G + pair - r * p.G;
  }

  // What a lane knows of its row, as it comes from memory: looked at a stage later, or it would be waited for at once.
  struct Info {
    int doc, pos;
    float lse, slope;
  };
  __device__ __forceinline__ Info info(int pair) const {
    int row, head;
    place(min(pair, pairs - 1), row, head);
    Info x = {-1, 0, p.lse_in[(int64_t)row * p.nq + head], 0.f};
    if (p.c.key_doc) x.doc = p.q_doc[row];
    if (p.slopes) {
      x.slope = p.slopes[head];
      if (p.q_pos) x.pos = p.q_pos[row];
    }
    return x;
  }

  __device__ __forceinline__ void block(int key0, const float *in, float *out) {
    from = p.last > 0 ? max(0, n - p.last) : 0;                  // the first row that counts
    if (key0 >= all) from = max(from, key0 - (len - n));         // rows before it see none of these keys
    const int mine = key0 + (int)threadIdx.x;                    // the key whose total this thread adds up at the end
    const bool adds = threadIdx.x < KEYS && mine < p.c.most;
    const float before = adds ? in[mine] : 0.f;
    if (key0 >= len || from >= n) {
      if (adds) out[mine] = before;
      return;
    }
    pairs = (n - from) * p.G;
    const int kw = wave & 1, rw = wave >> 1, my_key0 = key0 + 32 * KB * kw;
    typename S::Rows keys[KB];
    const bool has_doc = p.c.key_doc != nullptr;
    // where this lane's pieces of a stage of rows come from; a whole stage before, the same pieces lie a fixed step back if the heads divide it
    const char *at[LOADS];
    const bool even = p.g_shift >= 0 && p.G <= ROWS;
    const int64_t step = even ? (int64_t)(ROWS >> p.g_shift) * p.q_rs * ES : 0;
    const int stages = (pairs + ROWS - 1) / ROWS;
    auto issue = [&](int s) {  // the s-th from the end
      char *dst = lds + SHARE + (s & 1) * TILE;
      const int pair0 = (stages - 1 - s) * ROWS;
      if constexpr (WIDE) {
        const int first = threadIdx.x / S::CPR, piece = threadIdx.x % S::CPR;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
          const int r = first + j * STEP, c = piece ^ S::kswz(r);
          if (even && s >= 2) at[j] -= step;
          else {
            int row, head;
            place(min(pair0 + r, pairs - 1), row, head);
            at[j] = (const char *)((const T *)p.q + row * p.q_rs + head * p.q_hs) + c * 16;
          }
          if (c < span.chunks) __builtin_amdgcn_global_load_lds((gbl_ptr_t *)at[j], (lds_ptr_t *)(dst + (j * NW + wave) * 1024), 16, 0, 0);
        }
      } else {
        const int d = p.c.head_dim;
        for (int i = threadIdx.x; i < ROWS * d; i += THREADS) {
          const int r = i / d, f = i % d, c = (f / EPC) ^ S::kswz(r);
          int row, head;
          place(min(pair0 + r, pairs - 1), row, head);
          ((T *)(dst + r * S::ROWB + c * 16))[f % EPC] = ((const T *)p.q)[row * p.q_rs + head * p.q_hs + f];
        }
      }
    };
    __syncthreads();  // the block before is done with LDS
    issue(0);
    if (threadIdx.x < KEYS) {  // ids and positions of the keys, for the rows that want them
      int *ints = (int *)lds + (NW / 2) * KEYS;
      const int key = min(mine, len - 1);
      if (has_doc) ints[threadIdx.x] = p.c.key_doc[b * p.c.key_doc_request_stride + kvh * p.c.key_doc_head_stride + key];
      if (p.slopes) ints[KEYS + threadIdx.x] = p.c.key_pos ? p.c.key_pos[b * p.c.key_pos_request_stride + kvh * p.c.key_pos_head_stride + key] : p.c.prefix_len + key;
    }
    Info next[TILES];
#pragma unroll
    for (int x = 0; x < TILES; ++x) next[x] = info((stages - 1) * ROWS + (x * (NW / 2) + rw) * 32 + col);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int first = my_key0 + 32 * kb;
      span.load_row((const T *)p.c.k + own_offset(p.c, p.page_shift, p.c.k_page_stride, p.c.k_head_stride, p.c.k_key_stride, b, kvh, min(first + col, len - 1)), true, keys[kb]);
    }
    float acc[KB][16];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[kb][i] = 0.f;
    const bool capped = p.cap2 != 0.f;
    for (int s = 0; s < stages; ++s) {
      Info these[TILES];
#pragma unroll
      for (int x = 0; x < TILES; ++x) these[x] = next[x];
      __builtin_amdgcn_s_waitcnt(0x0070);
      __syncthreads();
      if (s + 1 < stages) {
        issue(s + 1);
#pragma unroll
        for (int x = 0; x < TILES; ++x) next[x] = info((stages - 2 - s) * ROWS + (x * (NW / 2) + rw) * 32 + col);
      }
#pragma unroll
      for (int x = 0; x < TILES; ++x) {
        const int pair0 = (stages - 1 - s) * ROWS + (x * (NW / 2) + rw) * 32;
        if (pair0 < pairs) tile(lds + SHARE + (s & 1) * TILE + (x * (NW / 2) + rw) * 32 * S::ROWB, keys, these[x], pair0, my_key0, kw, capped, has_doc, acc);
      }
    }
    // the rows' lanes together, then the waves that had the same keys
    float *share = (float *)lds;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) acc[kb][i] += __shfl_xor(acc[kb][i], x);
        if (col == 0) share[rw * KEYS + 32 * (KB * kw + kb) + S::key_of(i, hh)] = acc[kb][i];
      }
    __syncthreads();
    if (adds) {
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < NW / 2; ++w) sum += share[w * KEYS + threadIdx.x];
      out[mine] = before + sum;
    }
  }

  // 32 rows meet this wave's keys
  __device__ __forceinline__ void tile(const char *rows, const typename S::Rows (&keys)[KB], const Info &now, int pair0, int my_key0, int kw, bool capped, bool has_doc,
                                       float (&acc)[KB][16]) const {
    // rows that all see all of these keys, and whose scores need no more than a cap: the first row sees least
    const int r0 = p.g_shift >= 0 ? pair0 >> p.g_shift : pair0 / p.G;
    const int reach = min(max(len - n + from + r0, all - 1), len - 1);
    const bool plain = !has_doc && !p.slopes && pair0 + 32 <= pairs && my_key0 + 32 * KB - 1 <= reach;
    // The row's log-sum-exp as an exponent of two.  What its rounding takes, up to 2^-18 from 64 on, goes to all of the row's weights as a
    // factor, by a fused sum instead of a sum: weights of scores of 0 are off by less than 5e-7 of themselves, by up to 2.6e-6 without it.
    const float hi = __uint_as_float(bits_of(now.lse * kLog2e));
    const float lse2 = is_none(now.lse) ? INFINITY : hi;  // a row that saw nothing gives nothing
    const float rest = not_finite(hi) ? 1.0f : fmaf(-kLn2, fmaf(now.lse, kLog2eLow, fmaf(now.lse, kLog2e, -hi)), 1.0f);
    f32x16_t a[KB];
    products(rows, keys, a);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      bool raw = plain;
      if (raw && capped) {
        float far = 0.f;
#pragma unroll
        for (int i = 0; i < 16; i += 2) far = fmaxf(fmaxf(far, fabsf(a[kb][i])), fabsf(a[kb][i + 1]));
        raw = !__any(!(far <= p.cap_most));
      }
      if (raw) {
        if (capped) {
#pragma unroll
          for (int i = 0; i < 16; ++i) a[kb][i] = exp2_(fmaf(a[kb][i], cap_factor(a[kb][i], p.cap_c), -lse2));
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) a[kb][i] = exp2_(fmaf(a[kb][i], p.scale2, -lse2));
        }
      } else {
        const int pair = pair0 + col, row = p.g_shift >= 0 ? pair >> p.g_shift : pair / p.G, own_index = len - n + from + row;
        const int left = (pair < pairs ? min(max(own_index, all - 1), len - 1) : -1) - my_key0 - 32 * kb - 4 * hh;
        const int pos = p.q_pos ? now.pos : p.c.prefix_len + own_index;
        const int *ints = (const int *)lds + (NW / 2) * KEYS + 32 * (KB * kw + kb) + 4 * hh;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          i32x4_t doc = {-1, -1, -1, -1}, at = {0, 0, 0, 0};
          if (has_doc) doc = *(const i32x4_t *)(ints + 8 * g);
          if (p.slopes) at = *(const i32x4_t *)(ints + KEYS + 8 * g);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * g + e;
            float s = capped ? cap_any(a[kb][i], p.cap_c, p.cap_most, p.to_cap, p.cap2) : a[kb][i] * p.scale2;
            if (p.slopes) s -= now.slope * kLog2e * fabsf((float)(pos - at[e]));
            const bool seen = S::key_of(i, 0) <= left && (doc[e] == now.doc || doc[e] < 0 || now.doc < 0);
            a[kb][i] = seen ? exp2_(s - lse2) : 0.f;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[kb][i] = fmaf(a[kb][i], rest, acc[kb][i]);
    }
  }

  // scores of 32 rows in LDS with this wave's keys: the operands of Span's products, exchanged
  __device__ __forceinline__ void products(const char *rows, const typename S::Rows (&keys)[KB], f32x16_t (&a)[KB]) const {
    constexpr int NP = S::NP, AHEAD = NP < 4 ? NP : 4;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) a[kb][r] = 0.f;
    const unsigned row = here(S::lds_at(rows) + col * S::ROWB + ((hh ^ S::kswz(col)) << 4));
    auto piece = [&](int i) { return *(const lds_f32x4_t *)(row ^ (i << 5)); };
    f32x4_t q[NP];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) q[i] = piece(i);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        if constexpr (ES == 2) {
          a[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, keys[kb].q[i]), __builtin_bit_cast(bf16x8_t, q[i]), a[kb], 0, 0, 0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) a[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(keys[kb].q[i][e], q[i][e], a[kb], 0, 0, 0);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (i + AHEAD < NP) q[i + AHEAD] = piece(i + AHEAD);
    }
  }
};

template <typename T, int NT, bool WIDE, int ROWS, int KB, int NW> __global__ void __launch_bounds__(64 * NW, NW == 4 && NT <= 8 && sizeof(T) == 2 ? 3 : NW == 4 && span_chunks(NT, sizeof(T)) > 32 ? 1 : 2) k_span_received(const SpanCall p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  using R = Received<T, NT, WIDE, ROWS, KB, NW>;
  const int blocks = (p.c.most + R::KEYS - 1) / R::KEYS, items = p.pairs_of_blocks ? (blocks + 1) / 2 : blocks;
  int kvh, item;
  if (!head_item(blockIdx.x, p.c.n_kv_heads, items * p.c.n_requests, kvh, item)) return;
  const int b = item / items, i = item % items;
  const float *in = p.totals.in + b * p.totals.in_request_stride + kvh * p.totals.in_head_stride;
  float *out = p.totals.out + b * p.totals.out_request_stride + kvh * p.totals.out_head_stride;
  R r(p, lds, kvh, b, uniform(span_len(p, b)));
  if (!WIDE || r.span.chunks < R::S::CPR) {
    const int end = p.one_stage ? R::LDS_ONE : R::LDS;
    for (int x = threadIdx.x; x < end / 16; x += R::THREADS) ((f32x4_t *)lds)[x] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  r.block(i * R::KEYS, in, out);
  if (p.pairs_of_blocks && blocks - 1 - i > i) r.block((blocks - 1 - i) * R::KEYS, in, out);
}

// most: LDS that any call of the kernel asks for; told to the device once
template <auto K> hipError_t span_launch(int lds, int most, unsigned blocks, int threads, const SpanCall &p, hipStream_t s) {
  static std::atomic<uint64_t> told{0};  // by device
  if (blocks == 0) return hipSuccess;
  int device = 0;
  hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  const uint64_t bit = 1ull << (device & 63);
  if (device > 63 || !(told.load(std::memory_order_relaxed) & bit)) {
    e = hipFuncSetAttribute((const void *)K, hipFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e != hipSuccess) return e;
    told.fetch_or(bit, std::memory_order_relaxed);
  }
  K<<<blocks, threads, lds, s>>>(p);
  return hipGetLastError();
}

// f(steps, wide) with both as types
template <typename F> hipError_t span_pick(int d, bool wide, F &&f) {
  using std::integral_constant;
  if (!wide) return d <= 128 ? f(integral_constant<int, 8>(), std::false_type()) : f(integral_constant<int, 16>(), std::false_type());
  switch (span_steps(d, true)) {
    case 4: return f(integral_constant<int, 4>(), std::true_type());
    case 6: return f(integral_constant<int, 6>(), std::true_type());
    case 8: return f(integral_constant<int, 8>(), std::true_type());
    default: return f(integral_constant<int, 16>(), std::true_type());
  }
}

}  // namespace

template <typename T> hipError_t span_prompt(const SpanCall &p, bool wide, hipStream_t s) {
  return span_pick(p.c.head_dim, wide, [&](auto nt, auto w) {
    constexpr int NT = decltype(nt)::value;
    constexpr bool W = decltype(w)::value;
    using S = Span<T, NT, kSpanWaves, 1, span_stage_keys(NT, sizeof(T)), 2, W>;
    return span_launch<k_span_prompt<T, NT, W>>(S::LDS_ALL + (p.c.key_doc ? Survey<S>::LDS : 0), S::LDS_ALL + Survey<S>::LDS,
                                                (unsigned)span_head_items(p.c.n_kv_heads, p.tiles * p.splits), 64 * kSpanWaves, p, s);
  });
}

template <typename T> hipError_t span_token(const SpanCall &p, bool wide, hipStream_t s) {
  return span_pick(p.c.head_dim, wide, [&](auto nt, auto w) {
    constexpr int NT = decltype(nt)::value;
    constexpr bool W = decltype(w)::value;
    constexpr int NW = span_token_waves(NT, sizeof(T));
    constexpr int own = Span<T, NT, 1, NW, 32, 1, W>::LDS_ALL, pre = Span<T, NT, NW, 1, span_stage_keys(NT, sizeof(T)), 2, W>::LDS_ALL;
    constexpr int lds = own > pre ? own : pre;
    return span_launch<k_span_token<T, NT, W>>(lds, lds,
                              (unsigned)p.pre_items + (unsigned)p.c.n_requests * p.tiles * p.splits * p.c.n_kv_heads, 64 * NW, p, s);
  });
}

template <typename T> hipError_t span_received(const SpanCall &p, bool wide, hipStream_t s) {
  return span_pick(p.c.head_dim, wide, [&](auto nt, auto w) {
    constexpr int NT = decltype(nt)::value;
    constexpr bool W = decltype(w)::value;
    SpanCall call = p;
    auto go = [&](auto pairs) {
      constexpr SpanReceived F = span_received_form(NT, sizeof(T), decltype(pairs)::value);
      using R = Received<T, NT, W, F.rows, F.keys / 64, F.waves>;
      call.one_stage = p.last > 0 && (int64_t)p.last * p.G <= F.rows;
      return span_launch<k_span_received<T, NT, W, F.rows, F.keys / 64, F.waves>>(call.one_stage ? R::LDS_ONE : R::LDS, R::LDS,
                                                                                 (unsigned)span_head_items(p.c.n_kv_heads, span_received_items(p, F.keys)), 64 * F.waves, call, s);
    };
    return p.pairs_of_blocks ? go(std::true_type()) : go(std::false_type());
  });
}

template <typename T> hipError_t span_join(const SpanCall &p, hipStream_t s) {
  const int slots = p.pre_splits + p.splits;
  unsigned blocks = p.join_items;
  if (p.scores) blocks += (unsigned)((p.c.most + 1023) / 1024) * p.c.n_kv_heads * p.c.n_requests;
  if (blocks == 0) return hipSuccess;
  k_span_join<T><<<blocks, 256, 0, s>>>(p, slots);
  return hipGetLastError();
}

}  // namespace hyp
