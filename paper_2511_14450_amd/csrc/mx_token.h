// Attention of one row a request over its cached codes, for T = float or bf16_t rows.
//
// A wave takes two runs of 16 keys at a time, and up to 16 query heads of one KV head.  S^T = K Q^T has keys on the M axis of the matrix
// instruction and heads on the N axis, with the 32 features of a step in whatever order the codes come best: a lane holds 8 to 32 adjacent
// features of one key, which is 8 or 16 bytes.  Lane l then owns head l % 16 and keys 4 (l / 16) .. + 3 of either run, so that a head's scale,
// cap, distance and mask stay in its four lanes, and its probabilities are the operand of O^T += V^T P^T as they stand, if that product's
// keys are taken in the same order: a lane holds 2 to 8 adjacent features of those eight keys, converted as pairs of features and exchanged to
// pairs of keys.  Codes go from memory to registers; nothing of the keys passes through LDS.  The codes' numbers are bf16 as they stand, so that
// products of bf16 rows are exact; float rows and probabilities are three bf16 that add up to them.
#pragma once

#include <type_traits>

#include "attn_score.h"
#include "mx_format.h"
#include "mx_rules.h"

namespace hyp {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kFollow = 8.0f;     // the running maximum moves when a score passes it by more than 2^8
constexpr float kLowest = -3.402823466e38f;  // the maximum of no score: finite, so that a score of -infinity has the weight 0 beside it

// Pieces of a row of G groups, for keys (4 lanes a row) and values (16 lanes a row): a piece has `feats` adjacent features a lane.
struct Piece { int base, feats; };
constexpr int key_feats(int format, int left) { return format == HYP_E2M1 && left >= 4 ? 32 : left >= 2 ? 16 : 8; }
constexpr int value_feats(int left) { return left >= 4 ? 8 : left >= 2 ? 4 : 2; }
template <int G, int F, bool KEY> struct Pieces {
  int n = 0;
  Piece at[8] = {};
  constexpr Pieces() {
    for (int done = 0; done < G; ++n) {
      at[n].base = 32 * done;
      at[n].feats = KEY ? key_feats(F, G - done) : value_feats(G - done);
      done += KEY ? at[n].feats / 8 : at[n].feats / 2;
    }
  }
};
constexpr int piece_bytes(int format, int feats) { return format == HYP_E4M3 ? feats : feats / 2; }

template <int BYTES> __device__ __forceinline__ void load_bytes(const uint8_t *p, unsigned *w) {
  if constexpr (BYTES == 16) {
    const uint4 x = *(const uint4 *)p;
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  } else if constexpr (BYTES == 8) {
    const uint2 x = *(const uint2 *)p;
    w[0] = x.x; w[1] = x.y;
  } else if constexpr (BYTES == 4) {
    w[0] = *(const unsigned *)p;
  } else if constexpr (BYTES == 2) {
    w[0] = *(const uint16_t *)p;
  } else {
    w[0] = *p;
  }
}
constexpr int words(int bytes) { return (bytes + 3) / 4; }

__device__ __forceinline__ bf16x8_t as_bf16x8(const unsigned (&w)[4]) {
  uint4 x = make_uint4(w[0], w[1], w[2], w[3]);
  return __builtin_bit_cast(bf16x8_t, x);
}

// x as one bf16 (rounded), or as the sum of three: the first and the second are x and the rest cut to 8 bits, the third is what is left.
template <int PARTS> __device__ __forceinline__ void split8(const float (&x)[8], bf16x8_t (&out)[PARTS]) {
  if constexpr (PARTS == 1) {
#pragma unroll
    for (int i = 0; i < 8; ++i) out[0][i] = (__bf16)x[i];
  } else {
    unsigned w[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      unsigned a[2], b[2], c[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float v = x[2 * i + h];
        a[h] = __float_as_uint(v) & 0xffff0000u;
        const bool whole = (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u;  // infinities and NaN have no rest
        if (whole) a[h] = (__float_as_uint(v) | ((__float_as_uint(v) & 0xffffu) ? 0x400000u : 0u)) & 0xffff0000u;
        const float r = whole ? 0.f : v - __uint_as_float(a[h]);
        b[h] = __float_as_uint(r) & 0xffff0000u;
        c[h] = __float_as_uint(r - __uint_as_float(b[h])) & 0xffff0000u;
      }
      w[0][i] = a[0] >> 16 | a[1];
      w[1][i] = b[0] >> 16 | b[1];
      w[2][i] = c[0] >> 16 | c[1];
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) out[k] = as_bf16x8(w[k]);
  }
}

template <typename T, int G, int KF, int VF> struct Token {
  static constexpr int QP = sizeof(T) == 4 ? 3 : 1;  // parts of rows and probabilities
  static constexpr Pieces<G, KF, true> KP{};
  static constexpr Pieces<G, VF, false> VP{};
  static constexpr int VW = [] { int n = 0; for (int i = 0; i < VP.n; ++i) n += words(piece_bytes(VF, VP.at[i].feats)); return n; }();
  static constexpr int KW = [] { int n = 0; for (int i = 0; i < KP.n; ++i) n += words(piece_bytes(KF, KP.at[i].feats)); return n; }();
  static constexpr int D = 32 * G;

  struct Run {                 // of 16 keys, as a lane holds it
    unsigned k[KW], ks[KP.n];
    unsigned v[4][VW], vs[VP.n];
    int valid;                 // keys that are there; 0: none
    int first;                 // their first key
  };

  const MxTokenCall &p;
  const int lane, col, quarter;
  int kvh;
  bf16x8_t q[QP][G];
  f32x4_t o[2 * G];
  float m, l;

  __device__ __forceinline__ Token(const MxTokenCall &call) : p(call), lane(threadIdx.x & 63), col(lane & 15), quarter(lane >> 4) {}

  // Row of head `head` (of q), as the N operand of the steps of K's pieces; zeros where there is no such head
  __device__ __forceinline__ void load_q(int b, int head, bool there) {
    const T *row = (const T *)p.q.q + b * p.q.q_row_stride + head * p.q.q_head_stride;
    const int d = p.m.c.head_dim;
    int step = 0;
#pragma unroll
    for (int i = 0; i < KP.n; ++i) {
#pragma unroll
      for (int s = 0; s < KP.at[i].feats / 8; ++s, ++step) {
        const int f = KP.at[i].base + KP.at[i].feats * quarter + 8 * s;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
        if (there) {
          if (p.wide_q && f < d) {
            if constexpr (sizeof(T) == 2) {
              const u16x8_t v = *(const u16x8_t *)(row + f);
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = bf16_to_f32(v.v[e]);
            } else {
              const f32x4_t a = *(const f32x4_t *)(row + f), z = *(const f32x4_t *)(row + f + 4);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                x[e] = a[e];
                x[4 + e] = z[e];
              }
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (f + e < d) x[e] = load_f32(row + f + e);
          }
        }
        bf16x8_t part[QP];
        split8<QP>(x, part);
#pragma unroll
        for (int t = 0; t < QP; ++t) q[t][step] = part[t];
      }
    }
  }

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 2 * G; ++i) o[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m = kLowest;
    l = 0.f;
  }

  // place: page (or request), place in it of the run's first key, keys that are there, first key.  Keys beyond the last one that is there are read
  // as that one, of which nothing is used.
  __device__ __forceinline__ void fetch(Run &r, int4 place) {
    const hyp_mx_cache_t &c = p.m.c;
    const int page = __builtin_amdgcn_readfirstlane(place.x), at = __builtin_amdgcn_readfirstlane(place.y);
    r.valid = __builtin_amdgcn_readfirstlane(place.z);
    r.first = __builtin_amdgcn_readfirstlane(place.w);
    const int last = max(r.valid, 1) - 1;
    const uint8_t *k = c.k + (int64_t)page * c.k_page_stride + (int64_t)kvh * c.k_head_stride + (int64_t)at * c.k_key_stride;
    const uint8_t *v = c.v + (int64_t)page * c.v_page_stride + (int64_t)kvh * c.v_head_stride + (int64_t)at * c.v_key_stride;
    const uint8_t *ks = c.k_scale + (int64_t)page * c.k_scale_page_stride + (int64_t)kvh * c.k_scale_head_stride + at;
    const uint8_t *vs = c.v_scale + (int64_t)page * c.v_scale_page_stride + (int64_t)kvh * c.v_scale_head_stride + at;
    const int key = min(col, last);
    const uint8_t *row = k + (unsigned)key * (unsigned)c.k_key_stride;
    int w = 0;
#pragma unroll
    for (int i = 0; i < KP.n; ++i) {
      constexpr auto P = KP;
      const int feats = P.at[i].feats, base = P.at[i].base;
      const int bytes = piece_bytes(KF, feats);
      const uint8_t *from = row + piece_bytes(KF, base) + bytes * quarter;
      if (bytes == 16) load_bytes<16>(from, &r.k[w]);
      else if (bytes == 8) load_bytes<8>(from, &r.k[w]);
      else load_bytes<4>(from, &r.k[w]);
      w += words(bytes);
      r.ks[i] = ks[(int64_t)((base + feats * quarter) >> 5) * c.k_scale_group_stride + key];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint8_t *vrow = v + (unsigned)min(4 * quarter + j, last) * (unsigned)c.v_key_stride;
      w = 0;
#pragma unroll
      for (int i = 0; i < VP.n; ++i) {
        constexpr auto P = VP;
        const int bytes = piece_bytes(VF, P.at[i].feats);
        const uint8_t *from = vrow + piece_bytes(VF, P.at[i].base) + bytes * col;
        if (bytes == 8) load_bytes<8>(from, &r.v[j][w]);
        else if (bytes == 4) load_bytes<4>(from, &r.v[j][w]);
        else if (bytes == 2) load_bytes<2>(from, &r.v[j][w]);
        else load_bytes<1>(from, &r.v[j][w]);
        w += words(bytes);
      }
    }
    // four keys' scales at once; the room of a request or page is a multiple of 16
#pragma unroll
    for (int i = 0; i < VP.n; ++i) {
      constexpr auto P = VP;
      r.vs[i] = *(const unsigned *)(vs + (int64_t)((P.at[i].base + P.at[i].feats * col) >> 5) * c.v_scale_group_stride + 4 * quarter);
    }
  }

  // Raw scores of a run: keys 4 quarter + i of it with this lane's head
  __device__ __forceinline__ f32x4_t scores(const Run &r) {
    f32x4_t s = {0.f, 0.f, 0.f, 0.f};
    int step = 0, w = 0;
#pragma unroll
    for (int i = 0; i < KP.n; ++i) {
      constexpr auto P = KP;
      const float scale = mx_scale(r.ks[i]);
#pragma unroll
      for (int x = 0; x < P.at[i].feats / 8; ++x, ++step) {
        unsigned a[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) a[t] = mx_pair<KF>(&r.k[w], t, scale);
        w += KF == HYP_E4M3 ? 2 : 1;
        const bf16x8_t key = as_bf16x8(a);
#pragma unroll
        for (int t = 0; t < QP; ++t) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[t][step], s, 0, 0, 0);
      }
    }
    return s;
  }

  // Scores of keys first + 4 quarter + i as exponents of two, -infinity where there is no such key
  __device__ __forceinline__ void shape(f32x4_t &s, const Run &r, float slope2, int len) {
    if (p.cap2 != 0.f) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = cap_any(s[i], p.cap_c, p.cap_most, p.to_cap, p.cap2);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] *= p.scale2;
    }
    if (p.slopes) {
      const int far = len - 1 - r.first - 4 * quarter;
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] -= slope2 * (float)(far - i);
    }
    if (r.valid < 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = 4 * quarter + i < r.valid ? s[i] : -INFINITY;
    }
  }

  __device__ __forceinline__ void step(Run &a, Run &b, float slope2, int len) {
    f32x4_t s0 = scores(a), s1 = scores(b);
    shape(s0, a, slope2, len);
    shape(s1, b, slope2, len);
    float top = fmaxf(fmaxf(fmaxf(s0[0], s0[1]), fmaxf(s0[2], s0[3])), fmaxf(fmaxf(s1[0], s1[1]), fmaxf(s1[2], s1[3])));
    if (__any(top > m + kFollow)) {
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float now = fmaxf(m, top), f = exp2_(m - now);
#pragma unroll
      for (int i = 0; i < 2 * G; ++i) o[i] *= f;
      l *= f;
      m = now;
    }
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = exp2_(s0[i] - m);
      x[4 + i] = exp2_(s1[i] - m);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) l += x[i];
    bf16x8_t prob[QP];
    split8<QP>(x, prob);
    if (a.valid < 16) mend(a);
    if (b.valid < 16) mend(b);
    int w = 0, at = 0;
#pragma unroll
    for (int i = 0; i < VP.n; ++i) {
      constexpr auto P = VP;
      float scale[8];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        scale[j] = mx_scale((a.vs[i] >> (8 * j)) & 255u);
        scale[4 + j] = mx_scale((b.vs[i] >> (8 * j)) & 255u);
      }
#pragma unroll
      for (int t = 0; t < P.at[i].feats / 2; ++t) {
        unsigned pair[8], even[4], odd[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          pair[j] = mx_pair<VF>(&a.v[j][w], t, scale[j]);
          pair[4 + j] = mx_pair<VF>(&b.v[j][w], t, scale[4 + j]);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          even[j] = __builtin_amdgcn_perm(pair[2 * j + 1], pair[2 * j], 0x05040100u);
          odd[j] = __builtin_amdgcn_perm(pair[2 * j + 1], pair[2 * j], 0x07060302u);
        }
#pragma unroll
        for (int x = 0; x < QP; ++x) {
          o[at] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(even), prob[x], o[at], 0, 0, 0);
          o[at + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(odd), prob[x], o[at + 1], 0, 0, 0);
        }
        at += 2;
      }
      w += words(piece_bytes(VF, P.at[i].feats));
    }
  }

  // Values of keys that are not there, whose weight is 0, may not be NaN.  Behind the last key that is there its codes were read, under scales of
  // places that hold anything: a 1 instead of those.  A run without keys was read at a place that may not be seen: zeros.
  __device__ __forceinline__ void mend(Run &r) {
#pragma unroll
    for (int i = 0; i < VP.n; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (4 * quarter + j >= r.valid) r.vs[i] = (r.vs[i] & ~(255u << (8 * j))) | 127u << (8 * j);
    if (r.valid) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int w = 0; w < VW; ++w) r.v[j][w] = 0;
  }
};

// One part of a request's keys, of one KV head and up to 16 of its query heads: the waves take pairs of runs in turn, and join what they have in
// LDS.
template <typename T, int G, int KF, int VF> __global__ void __launch_bounds__(kThreads, 2) k_mx_token(const MxTokenCall p) {
  using Tk = Token<T, G, KF, VF>;
  extern __shared__ char lds[];
  int4 *places = (int4 *)lds;
  __shared__ int used;
  const hyp_mx_cache_t &c = p.m.c;
  const int part = blockIdx.x % p.parts, item = blockIdx.x / p.parts, ht = item % p.head_tiles, pair = item / p.head_tiles;
  const int b = pair / c.n_kv_heads, kvh = pair % c.n_kv_heads, wave = threadIdx.x >> 6;
  const int len = mx_len(c, b);
  const int per = p.m.block_shift - 4;   // log2(runs of a block)
  const int runs = p.listed ? p.listed << per : (len + 15) >> 4;
  const int r0 = part * p.runs, n = min(p.runs, runs - r0);
  if (!p.listed && n <= 0 && part > 0) return;  // the join does not look at it
  if (threadIdx.x == 0) used = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int r = r0 + i;
    int4 at = make_int4(b, 0, 0, 0);
    if (p.listed) {
      const int block = p.blocks[(int64_t)pair * p.listed + (r >> per)];
      if (block >= 0 && block <= (len - 1) >> p.m.block_shift && len > 0) {
        at.w = (block << p.m.block_shift) + ((r & ((1 << per) - 1)) << 4);
        at.z = mx_clamped(len - at.w, 0, 16);
      }
    } else {
      at.w = r << 4;
      at.z = min(len - at.w, 16);
    }
    if (at.z > 0) {
      at.y = at.w;
      if (c.page_table) {
        at.x = mx_clamped(c.page_table[(int64_t)b * c.pages_per_request + (at.w >> p.m.shift)], 0, c.n_pages - 1);
        at.y = at.w & (c.page_keys - 1);
      }
      atomicMax(&used, i + 1);
    } else if (c.page_table) {
      at.x = 0;
    }
    places[i] = at;
  }
  __syncthreads();
  const int end = used;                  // runs behind the last one that holds keys are left out
  Tk t(p);
  t.kvh = kvh;
  const int head = ht * 16 + t.col;      // of the group
  const bool there = head < p.G;
  const int qh = kvh * p.G + (there ? head : 0);
  t.load_q(b, qh, there);
  t.clear();
  const float slope2 = p.slopes && there ? p.slopes[qh] * kLog2e : 0.f;
  const int4 none = make_int4(c.page_table ? 0 : b, 0, 0, 0);
  auto place = [&](int i) { return i < end ? places[i] : none; };
  typename Tk::Run a, z;
  for (int i = 2 * wave; i < end; i += 2 * kWaves) {
    t.fetch(a, place(i));
    t.fetch(z, place(i + 1));
    t.step(a, z, slope2, len);
  }
  // join the waves: O^T is features x heads, lane (head, quarter) has features base + (4 quarter + r) feats + x
  t.l += __shfl_xor(t.l, 16);
  t.l += __shfl_xor(t.l, 32);
  __syncthreads();                       // places are done with
  constexpr int PITCH = Tk::D + 4;       // floats of a head; four more keep the sixteen heads off one another's banks
  float *ml = (float *)lds, *os = ml + 2 * kWaves * 16;
  const int heads = min(16, p.G - ht * 16);
  if (t.quarter == 0) {
    ml[(wave * 16 + t.col) * 2] = t.m;
    ml[(wave * 16 + t.col) * 2 + 1] = t.l;
  }
  if (there) {
    float *to = os + (wave * heads + t.col) * PITCH;
    int at = 0;
#pragma unroll
    for (int i = 0; i < Tk::VP.n; ++i) {
      constexpr auto P = Tk::VP;
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int x = 0; x < P.at[i].feats; x += 2) {
          float2 v = make_float2(t.o[at + x][r], t.o[at + x + 1][r]);
          *(float2 *)(to + P.at[i].base + (4 * t.quarter + r) * P.at[i].feats + x) = v;
        }
      at += P.at[i].feats;
    }
  }
  __syncthreads();
  const int d = c.head_dim;
  for (int x = threadIdx.x; x < heads * (Tk::D / 2); x += kThreads) {
    const int h = x / (Tk::D / 2), f = 2 * (x % (Tk::D / 2));
    if (f >= d) continue;
    float top = kLowest;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[(w * 16 + h) * 2]);
    float sum = 0.f, s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float e = exp2_(ml[(w * 16 + h) * 2] - top);
      const float2 v = *(const float2 *)(os + (w * heads + h) * PITCH + f);
      sum = fmaf(e, ml[(w * 16 + h) * 2 + 1], sum);
      s0 = fmaf(e, v.x, s0);
      s1 = fmaf(e, v.y, s1);
    }
    const int g = kvh * p.G + ht * 16 + h;
    const int64_t row = (int64_t)b * p.q.n_q_heads + g;
    if (p.parts > 1) {
      const int64_t at = (int64_t)part * c.n_requests * p.q.n_q_heads + row;
      p.part_o[at * d + f] = s0;
      if (f + 1 < d) p.part_o[at * d + f + 1] = s1;
      if (f == 0) {
        p.part_ml[2 * at] = top;
        p.part_ml[2 * at + 1] = sum;
      }
    } else {
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      T *out = (T *)p.out + b * p.out_rs + g * p.out_hs + f;
      store_f32(out, sum == 0.f ? 0.f : s0 * inv);
      if (f + 1 < d) store_f32(out + 1, sum == 0.f ? 0.f : s1 * inv);
      if (f == 0 && p.lse) p.lse[row] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
}

template <int G, typename T> constexpr int token_lds(int heads) {
  const int joined = 2 * kWaves * 16 * 4 + kWaves * heads * (32 * G + 4) * 4, places = kMxMostRuns * 16;
  return joined > places ? joined : places;
}

template <typename T, int KF, int VF, int G> hipError_t token_of(const MxTokenCall &p, hipStream_t s) {
  constexpr int most = token_lds<G, T>(16);
  static_assert(most <= 160 * 1024, "LDS of a CU");
  const int lds = token_lds<G, T>(p.G < 16 ? p.G : 16);
  if (lds > 64 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void *)k_mx_token<T, G, KF, VF>, hipFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e != hipSuccess) return e;
  }
  k_mx_token<T, G, KF, VF><<<(unsigned)p.m.c.n_requests * p.m.c.n_kv_heads * p.head_tiles * p.parts, kThreads, lds, s>>>(p);
  return hipGetLastError();
}

}  // namespace

template <typename T, int KF, int VF> hipError_t mx_token(const MxTokenCall &p, hipStream_t s) {
  switch (p.m.groups) {
    case 1: return token_of<T, KF, VF, 1>(p, s);
    case 2: return token_of<T, KF, VF, 2>(p, s);
    case 3: return token_of<T, KF, VF, 3>(p, s);
    case 4: return token_of<T, KF, VF, 4>(p, s);
    case 5: return token_of<T, KF, VF, 5>(p, s);
    case 6: return token_of<T, KF, VF, 6>(p, s);
    case 7: return token_of<T, KF, VF, 7>(p, s);
    default: return token_of<T, KF, VF, 8>(p, s);
  }
}

}  // namespace hyp
