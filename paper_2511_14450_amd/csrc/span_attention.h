// Kernels of attention over a shared prefix and a request's own keys (hyp_attn.h), for T = float or bf16_t.  Included by one
// translation unit per type.
#pragma once

#include "span_core.h"
#include "span_survey.h"

namespace hyp {
namespace {

// The request of row tile `t`: request b's tiles start at floor(q_start[b] G / tile) + b, which leaves each as many as it
// needs, or one more.  Returns the tile's first pair inside the request, or -1 if there is none.
__device__ __forceinline__ int64_t tile_request(const SpanCall &p, int t, int tile, int &req, int64_t &row0, int &rows) {
  const int n = p.c.n_requests;
  auto start = [&](int b) { return min(max((int64_t)p.q_start[b], (int64_t)0), p.n_rows); };
  int lo = 0, hi = n - 1;  // the last request whose first tile is <= t
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start(mid) * p.G / tile + mid <= t) lo = mid;
    else hi = mid - 1;
  }
  req = uniform(lo);
  row0 = uniform((int)start(req));
  rows = uniform((int)max(start(req + 1) - row0, (int64_t)0));
  const int64_t first = ((int64_t)t - (row0 * p.G / tile + req)) * tile;
  return first >= 0 && first < (int64_t)rows * p.G ? first : -1;
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

// attn_prompt.  A workgroup: one KV head, 128 rows of one request (dense over the group's heads), all the keys they see or one
// of `splits` parts of them.
template <typename T, int NT, bool WIDE> __global__ void __launch_bounds__(64 * kSpanWaves, span_steps_waves(NT)) k_span_prompt(const SpanCall p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  using S = Span<T, NT, kSpanWaves, 1, span_stage_keys(NT, sizeof(T)), WIDE>;
  int kvh, item;
  if (!head_item(blockIdx.x, p.c.n_kv_heads, p.tiles * p.splits, kvh, item)) return;
  const int split = item % p.splits;
  const int tile = p.tiles - 1 - item / p.splits;  // the longest rows of a request first
  int req, n;
  int64_t row0;
  const int64_t first = tile_request(p, tile, kSpanTile, req, row0, n);
  if (first < 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = threadIdx.x & 31;
  const int len = uniform(span_len(p, req));
  const int64_t pair = first + wave * 32 + col;
  const bool there = pair < (int64_t)n * p.G;
  const int i = there ? (int)(pair / p.G) : 0, g = there ? (int)(pair - (int64_t)i * p.G) : 0;
  const SpanRow r = span_row(p, (int)row0 + i, kvh * p.G + g, req, len - n + i, there);
  // the last row's reach, and the keys all of the request's rows see
  const int last = (int)(min(first + kSpanTile, (int64_t)n * p.G) - 1) / p.G;
  int end = len - n + last + 1;
  if (p.see_all) end = max(end, uniform(p.see_all[req]));
  const SpanKeys keys{0, p.c.prefix_len, 0, clamped(end, 0, len), req, kvh};
  typename S::State t;
  auto part = [&](int stages, int x) { return (int)((int64_t)stages * x / p.splits); };
  S span(p, keys, lds);
  const Survey<S> way(span, lds + S::LDS_ALL, r);
  span.attend(part(span.stages, split), part(span.stages, split + 1), r, t, nullptr, way);
  span.store_rows(r, t, split);
}

// attn_token.  Items over the shared keys, which all requests' rows meet at once, then items of up to 32 rows of one request
// over its own keys, whose waves take turns at them.
template <typename T, int NT, bool WIDE> __global__ void __launch_bounds__(64 * span_token_waves(NT, sizeof(T))) k_span_token(const SpanCall p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  constexpr int NW = span_token_waves(NT, sizeof(T));
  using Own = Span<T, NT, 1, NW, 32, WIDE>;
  using Pre = Span<T, NT, NW, 1, span_stage_keys(NT, sizeof(T)), WIDE>;
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
      const int b = there ? pair / p.G : 0;
      const SpanRow r = span_row(p, b, kvh * p.G + (there ? pair - b * p.G : 0), b, span_len(p, b) - 1, there);
      Pre span(p, SpanKeys{0, p.c.prefix_len, 0, 0, 0, kvh}, lds);
      typename Pre::State t;
      span.attend((int)((int64_t)span.stages * split / p.pre_splits), (int)((int64_t)span.stages * (split + 1) / p.pre_splits), r, t, nullptr, EveryStage{0x7fffffff});
      span.store_rows(r, t, split);
      return;
    }
    const int pair = tile * 32 + col;
    const bool there = pair < all;
    const int b = there ? pair / p.G : 0;
    const SpanRow r = span_row(p, b, kvh * p.G + (there ? pair - b * p.G : 0), b, span_len(p, b) - 1, there);
    Own span(p, SpanKeys{0, p.c.prefix_len, 0, 0, 0, kvh}, lds);
    typename Own::State t;
    span.attend((int)((int64_t)span.stages * split / p.pre_splits), (int)((int64_t)span.stages * (split + 1) / p.pre_splits), r, t, nullptr, EveryStage{0x7fffffff});
    span.join_waves(t, min(32, all - tile * 32), tile * 32, split);
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
  span.attend((int)((int64_t)span.stages * split / p.splits), (int)((int64_t)span.stages * (split + 1) / p.splits), r, t, scores, EveryStage{span.has_doc ? 0 : 0x7fffffff});
  span.join_waves(t, rows, (int64_t)b * p.G + tile * 32, p.pre_splits + split);
}

// The weight of a row's partial results: (maximum, sum) over the slots, in every lane.
__device__ __forceinline__ float2 slots_total(const SpanCall &p, int slots, int64_t pair, int lane) {
  const int64_t all = p.n_rows * p.nq;
  float m = -INFINITY;
  for (int s = lane; s < slots; s += 64) m = fmaxf(m, p.part_ml[2 * (s * all + pair)]);
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
  float l = 0.f;
  for (int s = lane; s < slots; s += 64) {
    const float ms = p.part_ml[2 * (s * all + pair)];
    if (!is_none(ms)) l += exp2_(ms - m) * p.part_ml[2 * (s * all + pair) + 1];
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) l += __shfl_xor(l, x);
  return {m, l};
}

// Partial results to results, a wave a row; then, for attn_token, the weight that own keys got.
template <typename T> __global__ void __launch_bounds__(256) k_span_join(const SpanCall p, int slots) {
  __shared__ float lse2[256];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, d = p.c.head_dim;
  const int64_t all = p.n_rows * p.nq;
  if ((int)blockIdx.x < p.join_items) {
    const int64_t pair = (int64_t)blockIdx.x * 4 + wave;
    if (pair >= all) return;
    const int64_t row = pair / p.nq;
    if (p.q_start && (row < p.q_start[0] || row >= p.q_start[p.c.n_requests])) return;  // no request's row
    const float2 ml = slots_total(p, slots, pair, lane);
    const int head = (int)(pair - row * p.nq);
    T *out = (T *)p.out + row * p.out_rs + head * p.out_hs;
    const bool none = is_none(ml.x);
    if (p.lse && lane == 0) p.lse[pair] = none ? -INFINITY : (ml.x + __builtin_amdgcn_logf(ml.y)) * kLn2;
    const float inv = none ? 0.f : 1.0f / ml.y;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < slots; ++s) {
      const float ms = p.part_ml[2 * (s * all + pair)];
      if (is_none(ms)) continue;
      const float a = exp2_(ms - ml.x) * p.part_ml[2 * (s * all + pair) + 1] * inv;
      const float *o = p.part_o + (s * all + pair) * d;
#pragma unroll
      for (int x = 0; x < 4; ++x)
        if (lane + 64 * x < d) acc[x] = fmaf(a, o[lane + 64 * x], acc[x]);
    }
#pragma unroll
    for (int x = 0; x < 4; ++x)
      if (lane + 64 * x < d) store_f32(out + lane + 64 * x, acc[x]);
    return;
  }
  // 1024 keys of one request and KV head
  const int blocks = (p.c.most + 1023) / 1024;
  int id = blockIdx.x - p.join_items;
  const int kb = id % blocks;
  id /= blocks;
  const int kvh = id % p.c.n_kv_heads, b = id / p.c.n_kv_heads;
  const int len = uniform(span_len(p, b));
  const float *in = p.totals.in + b * p.totals.in_request_stride + kvh * p.totals.in_head_stride;
  float *out = p.totals.out + b * p.totals.out_request_stride + kvh * p.totals.out_head_stride;
  if (kb * 1024 < len) {
    for (int g = wave; g < p.G; g += 4) {
      const float2 ml = slots_total(p, slots, (int64_t)b * p.nq + kvh * p.G + g, lane);
      if (lane == 0) lse2[g] = is_none(ml.x) ? INFINITY : ml.x + __builtin_amdgcn_logf(ml.y);
    }
  }
  __syncthreads();
  const float *scores = p.scores + ((int64_t)b * p.c.n_kv_heads + kvh) * p.G * p.score_pitch;
  for (int j = kb * 1024 + threadIdx.x; j < min(p.c.most, kb * 1024 + 1024); j += 256) {
    float w = 0.f;
    if (j < len)
      for (int g = 0; g < p.G; ++g) w += exp2_(scores[g * p.score_pitch + j] - lse2[g]);
    out[j] = in[j] + w;
  }
}

// attn_received.  A workgroup: one KV head and 128 own keys of a request, 32 a wave, which stay in registers; the rows that see
// them pass by in tiles of 32 through LDS, as the keys do above.
template <typename T, int NT, bool WIDE> __global__ void __launch_bounds__(256) k_span_received(const SpanCall p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  using S = Span<T, NT, 4, 1, 32, WIDE>;
  constexpr int ES = sizeof(T), EPC = 16 / ES;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hh = lane >> 5, col = lane & 31;
  int id = blockIdx.x;
  const int kvh = id % p.c.n_kv_heads;
  id /= p.c.n_kv_heads;
  const int b = id % p.c.n_requests, kb = id / p.c.n_requests;
  const int len = uniform(span_len(p, b)), key0 = kb * kSpanReceivedKeys;
  const float *in = p.totals.in + b * p.totals.in_request_stride + kvh * p.totals.in_head_stride;
  float *out = p.totals.out + b * p.totals.out_request_stride + kvh * p.totals.out_head_stride;
  const int64_t row0 = min(max((int64_t)p.q_start[b], (int64_t)0), p.n_rows), row1 = max(min((int64_t)p.q_start[b + 1], p.n_rows), row0);
  const int n = (int)(row1 - row0);
  int from = p.last > 0 ? max(0, n - p.last) : 0;               // the first row that counts
  const int all = p.see_all ? clamped(p.see_all[b], 0, len) : 0;
  if (key0 >= all) from = max(from, key0 - (len - n));          // rows before it see none of these keys
  if (key0 >= len || from >= n) {
    for (int j = key0 + threadIdx.x; j < min(p.c.most, key0 + kSpanReceivedKeys); j += 256) out[j] = in[j];
    return;
  }
  S span(p, SpanKeys{0, 0, 0, len, b, kvh}, lds);
  const int my_key0 = key0 + wave * 32;
  // this wave's keys as the other operand: lane = key my_key0 + col
  typename S::Rows keys;
  {
    const int key = min(my_key0 + col, len - 1);
    span.load_row((const T *)p.c.k + own_offset(p.c, p.page_shift, p.c.k_page_stride, p.c.k_head_stride, p.c.k_key_stride, b, kvh, key), true, keys);
  }
  int key_doc[16], key_pos[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int key = min(my_key0 + S::key_of(i, hh), len - 1);
    key_doc[i] = p.c.key_doc ? p.c.key_doc[b * p.c.key_doc_request_stride + kvh * p.c.key_doc_head_stride + key] : -1;
    key_pos[i] = p.slopes ? (p.c.key_pos ? p.c.key_pos[b * p.c.key_pos_request_stride + kvh * p.c.key_pos_head_stride + key] : p.c.prefix_len + key) : 0;
  }
  const int pairs = (n - from) * p.G;
  auto row_of = [&](int pair) { return row0 + from + pair / p.G; };
  auto head_of = [&](int pair) { return kvh * p.G + pair % p.G; };
  constexpr int TILE = 32 * S::ROWB;
  if (!WIDE || span.chunks < S::CPR) {
    for (int i = threadIdx.x; i < 2 * TILE / 16; i += 256) ((f32x4_t *)lds)[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    __syncthreads();
  }
  auto issue = [&](int tile, int buf) {
    char *dst = lds + buf * TILE;
    if constexpr (WIDE) {
      constexpr int LOADS = (32 * S::CPR + 255) / 256;
#pragma unroll
      for (int j = 0; j < LOADS; ++j) {
        const int at = (j * 4 + wave) * 64 + lane, row = at / S::CPR, c = (at % S::CPR) ^ S::kswz(row);
        const int pair = min(tile * 32 + row, pairs - 1);
        const char *src = (const char *)((const T *)p.q + row_of(pair) * p.q_rs + head_of(pair) * p.q_hs) + c * 16;
        if (at < 32 * S::CPR && c < span.chunks) __builtin_amdgcn_global_load_lds((gbl_ptr_t *)src, (lds_ptr_t *)(dst + (j * 4 + wave) * 1024), 16, 0, 0);
      }
    } else {
      const int d = p.c.head_dim;
      for (int i = threadIdx.x; i < 32 * d; i += 256) {
        const int row = i / d, f = i % d, c = (f / EPC) ^ S::kswz(row);
        const int pair = min(tile * 32 + row, pairs - 1);
        ((T *)(dst + row * S::ROWB + c * 16))[f % EPC] = ((const T *)p.q)[row_of(pair) * p.q_rs + head_of(pair) * p.q_hs + f];
      }
    }
  };
  struct Info { SpanRow r; float lse2; };
  auto info = [&](int tile) {
    const int pair = tile * 32 + col;
    const bool there = pair < pairs;
    const int64_t row = row_of(there ? pair : 0);
    Info x;
    x.r = span_row(p, (int)row, head_of(there ? pair : 0), b, len - n + (int)(row - row0), there);
    const float lse = there ? p.lse_in[row_pair(p, x.r)] : -INFINITY;
    x.lse2 = is_none(lse) ? INFINITY : lse * kLog2e;
    return x;
  };
  float acc[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) acc[i] = 0.f;
  const int tiles = (pairs + 31) / 32;
  issue(0, 0);
  Info next = info(0);
  for (int tile = 0; tile < tiles; ++tile) {
    const Info now = next;
    __builtin_amdgcn_s_waitcnt(0x0070);
    __syncthreads();
    if (tile + 1 < tiles) {
      issue(tile + 1, (tile + 1) & 1);
      next = info(tile + 1);
    }
    f32x16_t a;
#pragma unroll
    for (int r = 0; r < 16; ++r) a[r] = 0.f;
    const char *row = lds + (tile & 1) * TILE + col * S::ROWB;
    const int x = S::kswz(col);
#pragma unroll
    for (int i = 0; i < S::NP; ++i) {
      const f32x4_t q = *(const f32x4_t *)(row + (((2 * i + hh) ^ x) << 4));
      if constexpr (ES == 2) {
        a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, keys.q[i]), __builtin_bit_cast(bf16x8_t, q), a, 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) a = __builtin_amdgcn_mfma_f32_32x32x2f32(keys.q[i][e], q[e], a, 0, 0, 0);
      }
    }
    float s[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = a[i];
    if (p.cap2 != 0.f) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = cap_any(s[i], p.cap_c, p.cap_most, p.to_cap, p.cap2);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] *= p.scale2;
    }
    if (p.slopes) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] -= now.r.slope2 * fabsf((float)(now.r.pos - key_pos[i]));
    }
    const int last = min(now.r.lim, len - 1);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      bool seen = my_key0 + S::key_of(i, hh) <= last;
      if (p.c.key_doc) seen = seen && (key_doc[i] == now.r.doc || key_doc[i] < 0 || now.r.doc < 0);
      acc[i] += seen ? exp2_(s[i] - now.lse2) : 0.f;
    }
  }
  // the rows' lanes together
#pragma unroll
  for (int i = 0; i < 16; ++i) {
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) acc[i] += __shfl_xor(acc[i], x);
    const int key = my_key0 + S::key_of(i, hh);
    if (col == 0 && key < p.c.most) out[key] = in[key] + acc[i];
  }
}

inline unsigned head_items(int heads, int items) { return 8u * ((unsigned)(heads >> 3) * items + ((unsigned)(heads & 7) * items + 7) / 8); }

template <int NT, bool WIDE, typename K> hipError_t span_launch(K kernel, int lds, unsigned blocks, int threads, const SpanCall &p, hipStream_t s) {
  if (blocks == 0) return hipSuccess;
  hipError_t e = hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return e;
  kernel<<<blocks, threads, lds, s>>>(p);
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
    using S = Span<T, NT, kSpanWaves, 1, span_stage_keys(NT, sizeof(T)), W>;
    const int lds = S::LDS_ALL + (p.c.key_doc ? Survey<S>::LDS : 0);
    return span_launch<NT, W>(k_span_prompt<T, NT, W>, lds,
                              head_items(p.c.n_kv_heads, p.tiles * p.splits), 64 * kSpanWaves, p, s);
  });
}

template <typename T> hipError_t span_token(const SpanCall &p, bool wide, hipStream_t s) {
  return span_pick(p.c.head_dim, wide, [&](auto nt, auto w) {
    constexpr int NT = decltype(nt)::value;
    constexpr bool W = decltype(w)::value;
    constexpr int NW = span_token_waves(NT, sizeof(T));
    constexpr int own = Span<T, NT, 1, NW, 32, W>::LDS_ALL, pre = Span<T, NT, NW, 1, span_stage_keys(NT, sizeof(T)), W>::LDS_ALL;
    return span_launch<NT, W>(k_span_token<T, NT, W>, own > pre ? own : pre,
                              (unsigned)p.pre_items + (unsigned)p.c.n_requests * p.tiles * p.splits * p.c.n_kv_heads, 64 * NW, p, s);
  });
}

template <typename T> hipError_t span_received(const SpanCall &p, bool wide, hipStream_t s) {
  return span_pick(p.c.head_dim, wide, [&](auto nt, auto w) {
    constexpr int NT = decltype(nt)::value;
    constexpr bool W = decltype(w)::value;
    const unsigned blocks = (unsigned)((p.c.most + kSpanReceivedKeys - 1) / kSpanReceivedKeys) * p.c.n_requests * p.c.n_kv_heads;
    return span_launch<NT, W>(k_span_received<T, NT, W>, 2 * 32 * span_chunks(NT, sizeof(T)) * 16, blocks, 256, p, s);
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
