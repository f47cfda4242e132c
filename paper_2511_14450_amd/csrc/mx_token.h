// Attention of one row a request over its cached codes, for T = float or bf16_t rows.
//
// A wave takes two runs of 16 keys at a time, and up to 16 query heads of one KV head.  S^T = K Q^T has keys on the M axis of the matrix
// instruction and heads on the N axis, with the 32 features of a step in whatever order the codes come best: a lane holds 8 to 32 adjacent
// features of one key, which is 8 or 16 bytes.  Lane l then owns head l % 16 and keys 4 (l / 16) .. + 3 of either run, so that a head's scale,
// cap, distance and mask stay in its four lanes, and its probabilities are the operand of O^T += V^T P^T as they stand, if that product's
// keys are taken in the same order: a lane holds 2 to 8 adjacent features of those eight keys, converted as pairs of features and exchanged to
// pairs of keys.  Codes go from memory to registers; nothing of the keys passes through LDS.  The codes' numbers are bf16 as they stand, so that
// products of bf16 rows are exact; float rows and the probabilities beside them are three bf16 that add up to them.  Beside bf16 rows a probability is
// the sum of two, which hold it to 2^-16: as one, results were 2.0e-3 from the formula in 64 bits where rounding the results to bf16 costs
// 1.6e-3 - 1.7e-3, and sums in which values cancel were off by as much as their terms' 2^-8.
//
// Bytes bound 8 bits: 8 x 32768 keys of 8 heads of 128 features 90.5 us, of which the keys take 86 (6.4 TB/s; a streaming read reaches 6.45) and the
// join 4.8; capped scores that fall with the distance make it 95.  4 bits have half as many and are bound by the issue of instructions and by waiting:
// 58 us, 68 capped.  What it took, in steps that were each measured over the capped ones with one bf16 a probability: no clamped places in the loop
// (whole runs lie in the room; lengths count where codes are used), bytes to a unit of keys in LDS, where 64-bit products on the scalar unit were
// (together 105 -> 96), streaming loads (-7 us; a cache that fits the memory-side one, of 19 MB, takes 1 us more), the next pair of runs requested before
// one is worked on (4 bits: 59 -> 54; without it, at four waves a SIMD, 8 bits are as fast), one workgroup a CU for 8 bits.  Eight waves a workgroup
// were slower (32 requests of 101 - 608 keys: 18.7 instead of 12).  Two bf16 a probability took 3 % (listed blocks) to 9 % (4 bits) more.
#pragma once

#include <atomic>
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

typedef unsigned u32x4_t __attribute__((ext_vector_type(4)));
typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
template <int BYTES> __device__ __forceinline__ void load_bytes(const uint8_t *p, unsigned *w) {
  auto get = [](auto *at) { return __builtin_nontemporal_load(at); };  // read once, and more of them than the caches hold
  if constexpr (BYTES == 16) {
    const u32x4_t x = get((const u32x4_t *)p);
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  } else if constexpr (BYTES == 8) {
    const u32x2_t x = get((const u32x2_t *)p);
    w[0] = x.x; w[1] = x.y;
  } else if constexpr (BYTES == 4) {
    w[0] = get((const unsigned *)p);
  } else if constexpr (BYTES == 2) {
    w[0] = get((const uint16_t *)p);
  } else {
    w[0] = get(p);
  }
}
constexpr int words(int bytes) { return (bytes + 3) / 4; }

__device__ __forceinline__ bf16x8_t as_bf16x8(const unsigned (&w)[4]) {
  uint4 x = make_uint4(w[0], w[1], w[2], w[3]);
  return __builtin_bit_cast(bf16x8_t, x);
}

// x as the sum of two bf16, x and the rest rounded, or of three: the first and the second are x and the rest cut to 8 bits, the third is what is left.
template <int PARTS> __device__ __forceinline__ void split8(const float (&x)[8], bf16x8_t (&out)[PARTS]) {
  static_assert(PARTS == 2 || PARTS == 3, "two or three");
  if constexpr (PARTS == 2) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      out[0][i] = (__bf16)x[i];
      out[1][i] = (__bf16)(x[i] - (float)out[0][i]);
    }
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

// HT: tiles of 16 query heads of a wave
template <typename T, int G, int KF, int VF, int HT> struct Token {
  static constexpr int QP = sizeof(T) == 4 ? 3 : 1, PP = sizeof(T) == 4 ? 3 : 2;  // parts of rows, and of probabilities
  static constexpr Pieces<G, KF, true> KP{};
  static constexpr Pieces<G, VF, false> VP{};
  static constexpr int VW = [] { int n = 0; for (int i = 0; i < VP.n; ++i) n += words(piece_bytes(VF, VP.at[i].feats)); return n; }();
  static constexpr int KW = [] { int n = 0; for (int i = 0; i < KP.n; ++i) n += words(piece_bytes(KF, KP.at[i].feats)); return n; }();
  static constexpr int D = 32 * G;

  struct Run {                 // of 16 keys, as a lane holds it
    unsigned k[KW], ks[KP.n];
    unsigned v[4][VW], vs[VP.n];
    int valid;                 // keys that are there: none below 1, all from 16 on
    int first;                 // their first key
  };

  const MxTokenCall &p;
  const int lane, col, quarter;
  // bytes from a run's first key to this lane's keys and values, and to their scales (key strides are below 2^24, group strides below 2^28)
  unsigned k_at, v_at[4], ks_at[KP.n], vs_at[VP.n];
  bf16x8_t q[HT][QP][G];
  f32x4_t o[HT][2 * G];
  float m[HT], l[HT];

  __device__ __forceinline__ Token(const MxTokenCall &call) : p(call), lane(threadIdx.x & 63), col(lane & 15), quarter(lane >> 4) {}

  // First feature of the steps of K's pieces: base + feats * quarter
  struct Steps {
    int base[G] = {}, feats[G] = {};
    constexpr Steps() {
      int s = 0;
      for (int i = 0; i < KP.n; ++i)
        for (int x = 0; x < KP.at[i].feats; x += 8, ++s) {
          base[s] = KP.at[i].base + x;
          feats[s] = KP.at[i].feats;
        }
    }
  };
  __device__ __forceinline__ int feature(int s) const {
    constexpr Steps S{};
    return S.base[s] + S.feats[s] * quarter;
  }

  // Row of head `head` (of q), as tile ht's N operand of the steps of K's pieces; zeros where there is no such head
  __device__ __forceinline__ void load_q(int ht, int b, int head, bool there) {
    const T *row = (const T *)p.q.q + b * p.q.q_row_stride + head * p.q.q_head_stride;
    const int d = p.m.c.head_dim;
    constexpr int W = 2 * sizeof(T);     // words of eight features
    unsigned x[G][W];
    if (p.wide_q) {  // all pieces are requested before one is looked at
#pragma unroll
      for (int s = 0; s < G; ++s) {
        const uint4 *from = (const uint4 *)(row + min(feature(s), d - 8));
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
          const uint4 v = from[i];
          x[s][4 * i] = v.x; x[s][4 * i + 1] = v.y; x[s][4 * i + 2] = v.z; x[s][4 * i + 3] = v.w;
        }
      }
#pragma unroll
      for (int s = 0; s < G; ++s)
#pragma unroll
        for (int i = 0; i < W; ++i) x[s][i] = there && feature(s) < d ? x[s][i] : 0u;
    } else {
#pragma unroll
      for (int s = 0; s < G; ++s)
#pragma unroll
        for (int i = 0; i < W; ++i) {
          x[s][i] = 0;
#pragma unroll
          for (int e = 0; e < 4 / (int)sizeof(T); ++e) {
            const int f = feature(s) + i * 4 / (int)sizeof(T) + e;
            unsigned v = 0;
            __builtin_memcpy(&v, row + min(f, d - 1), sizeof(T));
            x[s][i] |= (there && f < d ? v : 0u) << (16 * e);
          }
        }
    }
#pragma unroll
    for (int s = 0; s < G; ++s) {
      if constexpr (QP == 1) {
        q[ht][0][s] = as_bf16x8(x[s]);
      } else {
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = __uint_as_float(x[s][e]);
        bf16x8_t part[QP];
        split8<QP>(y, part);
#pragma unroll
        for (int t = 0; t < QP; ++t) q[ht][t][s] = part[t];
      }
    }
  }

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int h = 0; h < HT; ++h) {
#pragma unroll
      for (int i = 0; i < 2 * G; ++i) o[h][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      m[h] = kLowest;
      l[h] = 0.f;
    }
  }

  __device__ __forceinline__ void aim() {
    const hyp_mx_cache_t &c = p.m.c;
    k_at = (unsigned)col * (unsigned)c.k_key_stride + piece_bytes(KF, KP.at[0].feats) * quarter;
#pragma unroll
    for (int j = 0; j < 4; ++j) v_at[j] = (unsigned)(4 * quarter + j) * (unsigned)c.v_key_stride;
#pragma unroll
    for (int i = 0; i < KP.n; ++i) ks_at[i] = (unsigned)((KP.at[i].base + KP.at[i].feats * quarter) >> 5) * (unsigned)c.k_scale_group_stride + col;
#pragma unroll
    for (int i = 0; i < VP.n; ++i) vs_at[i] = (unsigned)((VP.at[i].base + VP.at[i].feats * col) >> 5) * (unsigned)c.v_scale_group_stride + 4 * quarter;
  }

  // The codes of a run from its first key's places on.  All sixteen keys lie in the room of their request or page, whether they are there or not:
  // lengths are looked at when the codes are used.
  __device__ __forceinline__ void fetch(Run &r, const uint8_t *k, const uint8_t *v, const uint8_t *ks, const uint8_t *vs, int valid, int first) {
    r.valid = valid;
    r.first = first;
    int w = 0;
#pragma unroll
    for (int i = 0; i < KP.n; ++i) {
      constexpr auto P = KP;
      const int bytes = piece_bytes(KF, P.at[i].feats);
      // the pieces behind the first may be shorter, and a lane's place in them with it
      const unsigned at = k_at - (unsigned)((piece_bytes(KF, P.at[0].feats) - bytes) * quarter);
      const uint8_t *from = k + piece_bytes(KF, P.at[i].base) + at;
      if (bytes == 16) load_bytes<16>(from, &r.k[w]);
      else if (bytes == 8) load_bytes<8>(from, &r.k[w]);
      else load_bytes<4>(from, &r.k[w]);
      w += words(bytes);
      r.ks[i] = ks[ks_at[i]];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w = 0;
#pragma unroll
      for (int i = 0; i < VP.n; ++i) {
        constexpr auto P = VP;
        const int bytes = piece_bytes(VF, P.at[i].feats);
        const uint8_t *from = v + piece_bytes(VF, P.at[i].base) + (v_at[j] + (unsigned)(bytes * col));
        if (bytes == 8) load_bytes<8>(from, &r.v[j][w]);
        else if (bytes == 4) load_bytes<4>(from, &r.v[j][w]);
        else if (bytes == 2) load_bytes<2>(from, &r.v[j][w]);
        else load_bytes<1>(from, &r.v[j][w]);
        w += words(bytes);
      }
    }
    // four keys' scales at once; the room of a request or page is a multiple of 16
#pragma unroll
    for (int i = 0; i < VP.n; ++i) r.vs[i] = *(const unsigned *)(vs + vs_at[i]);
  }

  // Raw scores of a run: keys 4 quarter + i of it with this lane's heads
  __device__ __forceinline__ void scores(const Run &r, f32x4_t (&s)[HT]) {
#pragma unroll
    for (int h = 0; h < HT; ++h) s[h] = f32x4_t{0.f, 0.f, 0.f, 0.f};
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
        for (int h = 0; h < HT; ++h)
#pragma unroll
          for (int t = 0; t < QP; ++t) s[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key, q[h][t][step], s[h], 0, 0, 0);
      }
    }
  }

  __device__ __forceinline__ void clear_behind(f32x4_t &s, const Run &r) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = 4 * quarter + i < r.valid ? s[i] : 0.f;
  }

  // Scores of keys first + 4 quarter + i as exponents of two, -infinity where there is no such key; raw: all lie where the polynomial of a cap holds
  __device__ __forceinline__ void shape(f32x4_t &s, const Run &r, float slope2, int len, bool raw) {
    float factor[4];
    if (p.cap2 == 0.f) {
#pragma unroll
      for (int i = 0; i < 4; ++i) factor[i] = p.scale2;
    } else if (raw) {
#pragma unroll
      for (int i = 0; i < 4; ++i) factor[i] = cap_factor(s[i], p.cap_c);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[i] = cap_any(s[i], p.cap_c, p.cap_most, p.to_cap, p.cap2);
        factor[i] = 1.0f;
      }
    }
    if (p.slopes) {
      const float far = slope2 * (float)(len - 1 - r.first - 4 * quarter);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = fmaf(s[i], factor[i], fmaf(slope2, (float)i, -far));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] *= factor[i];
    }
    if (r.valid < 16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = 4 * quarter + i < r.valid ? s[i] : -INFINITY;
    }
  }

  __device__ __forceinline__ void step(Run &a, Run &b, const float (&slope2)[HT], int len) {
    f32x4_t s0[HT], s1[HT];
    scores(a, s0);
    scores(b, s1);
    bf16x8_t prob[HT][PP];
#pragma unroll
    for (int h = 0; h < HT; ++h) {
      // what is behind the last key has no part in which form of the cap is taken either, whose roundings differ
      if (a.valid < 16) clear_behind(s0[h], a);
      if (b.valid < 16) clear_behind(s1[h], b);
      bool raw = false;
      if (p.cap2 != 0.f) {
        const float far = fmaxf(fmaxf(fmaxf(fabsf(s0[h][0]), fabsf(s0[h][1])), fmaxf(fabsf(s0[h][2]), fabsf(s0[h][3]))),
                                fmaxf(fmaxf(fabsf(s1[h][0]), fabsf(s1[h][1])), fmaxf(fabsf(s1[h][2]), fabsf(s1[h][3]))));
        raw = !__any(!(far <= p.cap_most));  // a NaN stays one by either way
      }
      shape(s0[h], a, slope2[h], len, raw);
      shape(s1[h], b, slope2[h], len, raw);
      float top = fmaxf(fmaxf(fmaxf(s0[h][0], s0[h][1]), fmaxf(s0[h][2], s0[h][3])), fmaxf(fmaxf(s1[h][0], s1[h][1]), fmaxf(s1[h][2], s1[h][3])));
      if (__any(top > m[h] + kFollow)) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(m[h], top), f = exp2_(m[h] - now);
#pragma unroll
        for (int i = 0; i < 2 * G; ++i) o[h][i] *= f;
        l[h] *= f;
        m[h] = now;
      }
      float x[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = exp2_(s0[h][i] - m[h]);
        x[4 + i] = exp2_(s1[h][i] - m[h]);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) l[h] += x[i];
      split8<PP>(x, prob[h]);
    }
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
        for (int h = 0; h < HT; ++h)
#pragma unroll
          for (int x = 0; x < PP; ++x) {
            o[h][at] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(even), prob[h][x], o[h][at], 0, 0, 0);
            o[h][at + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(odd), prob[h][x], o[h][at + 1], 0, 0, 0);
          }
        at += 2;
      }
      w += words(piece_bytes(VF, P.at[i].feats));
    }
  }

  // Values of keys that are not there, whose weight is 0, may not be NaN: zeros under a scale of 1.
  __device__ __forceinline__ void mend(Run &r) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool gone = 4 * quarter + j >= r.valid;
#pragma unroll
      for (int w = 0; w < VW; ++w) r.v[j][w] = gone ? 0u : r.v[j][w];
#pragma unroll
      for (int i = 0; i < VP.n; ++i) r.vs[i] = gone ? (r.vs[i] & ~(255u << (8 * j))) | 127u << (8 * j) : r.vs[i];
    }
  }
};

// Where a unit of 16 or 32 keys lies, which is one or two runs: bytes from the tensors' beginnings, its first key, and, of a listed block, how many
// are there.
struct __attribute__((aligned(16))) Place {
  int64_t k, v, ks, vs;
  int first, valid, pad[2];
};

__device__ __forceinline__ int64_t uniform64(int64_t v) {
  const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)v), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

// One part of a request's keys, of one KV head and up to 16 HT of its query heads: the waves take pairs of runs in turn, and join what they have in
// LDS.
template <typename T, int G, int KF, int VF, int HT> __global__ void __launch_bounds__(kThreads, mx_token_two_workgroups(G, sizeof(T) == 4) ? 2 : 1) k_mx_token(const MxTokenCall p) {
  using Tk = Token<T, G, KF, VF, HT>;
  extern __shared__ char lds[];
  __shared__ int held[kWaves];           // units up to the last one that holds keys, among each wave's
  Place *places = (Place *)lds;
  const hyp_mx_cache_t &c = p.m.c;
  const int part = blockIdx.x % p.parts, item = blockIdx.x / p.parts, ht = item % p.head_tiles, pair = item / p.head_tiles;
  const int b = pair / c.n_kv_heads, kvh = pair % c.n_kv_heads, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int per = p.m.block_shift - p.unit;  // log2(units of a block); a unit has 16 or 32 keys
  const int unit = 1 << p.unit, u0 = part * p.units;
  const int len = mx_len(c, b), most = p.listed ? p.listed << per : (int)(((int64_t)c.most + unit - 1) >> p.unit);
  Tk t(p);
  const int head0 = ht * 16 * HT;        // of the group
  float slope2[HT];
#pragma unroll
  for (int h = 0; h < HT; ++h) {
    const int head = head0 + 16 * h + t.col, qh = kvh * p.G + (head < p.G ? head : 0);
    t.load_q(h, b, qh, head < p.G);
    slope2[h] = p.slopes && head < p.G ? p.slopes[qh] * kLog2e : 0.f;
  }
  // all units that the part can have, so that nothing waits for the length; those behind the last one that holds keys are left out below
  static_assert(kMxMostUnits <= kThreads, "a unit a thread");
  int end = min(p.units, most - u0);
  bool holds = false;                    // of listed ones
  if ((int)threadIdx.x < end) {
    const int i = threadIdx.x, u = u0 + i;
    Place at = {};
    at.first = u << p.unit;
    if (p.listed) {
      const int block = p.blocks[(int64_t)pair * p.listed + (u >> per)];
      const bool its = len > 0 && block >= 0 && block <= (len - 1) >> p.m.block_shift;
      at.first = its ? (block << p.m.block_shift) + ((u & ((1 << per) - 1)) << p.unit) : 0;  // else a place that may be read
      at.valid = its ? mx_clamped(len - at.first, 0, unit) : 0;
      if (at.valid == 0) at.first = 0;
      holds = at.valid > 0;
    }
    int page = b, in = at.first;
    if (c.page_table) {
      page = mx_clamped(c.page_table[(int64_t)b * c.pages_per_request + (at.first >> p.m.shift)], 0, c.n_pages - 1);
      in = at.first & (c.page_keys - 1);
    }
    at.k = page * c.k_page_stride + kvh * c.k_head_stride + in * c.k_key_stride;
    at.v = page * c.v_page_stride + kvh * c.v_head_stride + in * c.v_key_stride;
    at.ks = page * c.k_scale_page_stride + kvh * c.k_scale_head_stride + in;
    at.vs = page * c.v_scale_page_stride + kvh * c.v_scale_head_stride + in;
    places[i] = at;
  }
  if (p.listed) {
    const unsigned long long votes = __ballot(holds);
    if (t.lane == 0) held[wave] = votes ? 64 * wave + 64 - __clzll((long long)votes) : 0;
  } else {
    end = min(end, (int)(((int64_t)len + unit - 1) >> p.unit) - u0);
    if (end <= 0 && part > 0) return;    // the join does not look at it
  }
  __syncthreads();
  if (p.listed) {
    end = held[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) end = max(end, held[w]);
    end = __builtin_amdgcn_readfirstlane(end);
  }
  t.aim();
  t.clear();
  auto fetch = [&](typename Tk::Run &a, typename Tk::Run &z, int i) {
    const Place at = places[i];
    const int first = __builtin_amdgcn_readfirstlane(at.first), valid = p.listed ? __builtin_amdgcn_readfirstlane(at.valid) : len - first;
    const uint8_t *k = c.k + uniform64(at.k), *v = c.v + uniform64(at.v), *ks = c.k_scale + uniform64(at.ks), *vs = c.v_scale + uniform64(at.vs);
    t.fetch(a, k, v, ks, vs, valid, first);
    if (p.unit == 5) {
      t.fetch(z, k + 16 * c.k_key_stride, v + 16 * c.v_key_stride, ks + 16, vs + 16, valid - 16, first + 16);
    } else {
      const bool more = i + 1 < end;
      const Place of = places[more ? i + 1 : i];
      const int from = __builtin_amdgcn_readfirstlane(of.first);
      t.fetch(z, c.k + uniform64(of.k), c.v + uniform64(of.v), c.k_scale + uniform64(of.ks), c.v_scale + uniform64(of.vs),
              !more ? 0 : p.listed ? __builtin_amdgcn_readfirstlane(of.valid) : len - from, from);
    }
  };
  const int each = p.unit == 5 ? 1 : 2, STEP = kWaves * each;
  int i = wave * each;
  if constexpr (HT == 1 && G <= (sizeof(T) == 4 ? 3 : 4)) {
    // the next pair of runs is on its way while one is worked on
    typename Tk::Run a[2], z[2];
    if (i < end) {
      fetch(a[0], z[0], i);
      for (;;) {
        if (i + STEP >= end) {
          t.step(a[0], z[0], slope2, len);
          break;
        }
        fetch(a[1], z[1], i + STEP);
        t.step(a[0], z[0], slope2, len);
        i += 2 * STEP;
        if (i >= end) {
          t.step(a[1], z[1], slope2, len);
          break;
        }
        fetch(a[0], z[0], i);
        t.step(a[1], z[1], slope2, len);
      }
    }
  } else {
    for (; i < end; i += STEP) {
      typename Tk::Run a, z;
      fetch(a, z, i);
      t.step(a, z, slope2, len);
    }
  }
  // join the waves: O^T is features x heads, lane (head, quarter) has features base + (4 quarter + r) feats + x
  __syncthreads();                       // places are done with
  constexpr int PITCH = Tk::D + 4;       // floats of a head; four more keep the sixteen heads off one another's banks
  constexpr int HEADS = 16 * HT;
  float *ml = (float *)lds, *os = ml + 2 * kWaves * HEADS;
  const int heads = min(HEADS, p.G - head0);
#pragma unroll
  for (int h = 0; h < HT; ++h) {
    t.l[h] += __shfl_xor(t.l[h], 16);
    t.l[h] += __shfl_xor(t.l[h], 32);
    const int mine = 16 * h + t.col;
    if (t.quarter == 0) {
      ml[(wave * HEADS + mine) * 2] = t.m[h];
      ml[(wave * HEADS + mine) * 2 + 1] = t.l[h];
    }
    if (mine < heads) {
      float *to = os + (wave * heads + mine) * PITCH;
      int at = 0;
#pragma unroll
      for (int i = 0; i < Tk::VP.n; ++i) {
        constexpr auto P = Tk::VP;
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int x = 0; x < P.at[i].feats; x += 2) {
            float2 v = make_float2(t.o[h][at + x][r], t.o[h][at + x + 1][r]);
            *(float2 *)(to + P.at[i].base + (4 * t.quarter + r) * P.at[i].feats + x) = v;
          }
        at += P.at[i].feats;
      }
    }
  }
  __syncthreads();
  const int d = c.head_dim;
  for (int x = threadIdx.x; x < heads * (Tk::D / 2); x += kThreads) {
    const int h = x / (Tk::D / 2), f = 2 * (x % (Tk::D / 2));
    if (f >= d) continue;
    float top = kLowest;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[(w * HEADS + h) * 2]);
    float sum = 0.f, s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float e = exp2_(ml[(w * HEADS + h) * 2] - top);
      const float2 v = *(const float2 *)(os + (w * heads + h) * PITCH + f);
      sum = fmaf(e, ml[(w * HEADS + h) * 2 + 1], sum);
      s0 = fmaf(e, v.x, s0);
      s1 = fmaf(e, v.y, s1);
    }
    const int g = kvh * p.G + head0 + h;
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

template <int G, int HT> constexpr int token_lds(int heads) {
  const int joined = 2 * kWaves * 16 * HT * 4 + kWaves * heads * (32 * G + 4) * 4, places = kMxMostUnits * (int)sizeof(Place);
  return joined > places ? joined : places;
}

template <typename T, int KF, int VF, int G, int HT> hipError_t token_of(const MxTokenCall &p, hipStream_t s) {
  constexpr int most = token_lds<G, HT>(16 * HT);
  constexpr int own = kWaves * 4;        // what the kernel has beside it
  static_assert(most + own <= 80 * 1024, "LDS of two workgroups of a CU");
  const int lds = token_lds<G, HT>(std::min(p.G, 16 * HT));
  if (lds + own > 64 * 1024) {  // sixteen heads of more than 224 features, or 32 of more than 96: each device is told once
    static std::atomic<uint64_t> told{0};
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (device & 63);
    if (device > 63 || !(told.load(std::memory_order_relaxed) & bit)) {
      e = hipFuncSetAttribute((const void *)k_mx_token<T, G, KF, VF, HT>, hipFuncAttributeMaxDynamicSharedMemorySize, most);
      if (e != hipSuccess) return e;
      told.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  k_mx_token<T, G, KF, VF, HT><<<(unsigned)p.m.c.n_requests * p.m.c.n_kv_heads * p.head_tiles * p.parts, kThreads, lds, s>>>(p);
  return hipGetLastError();
}

template <typename T, int KF, int VF, int G> hipError_t token_tiles(const MxTokenCall &p, hipStream_t s) {
  if constexpr (mx_token_two_tiles(G, sizeof(T) == 4))
    if (p.tiles == 2) return token_of<T, KF, VF, G, 2>(p, s);
  return token_of<T, KF, VF, G, 1>(p, s);
}

}  // namespace

template <typename T, int KF, int VF> hipError_t mx_token(const MxTokenCall &p, hipStream_t s) {
  switch (p.m.groups) {
    case 1: return token_tiles<T, KF, VF, 1>(p, s);
    case 2: return token_tiles<T, KF, VF, 2>(p, s);
    case 3: return token_tiles<T, KF, VF, 3>(p, s);
    case 4: return token_tiles<T, KF, VF, 4>(p, s);
    case 5: return token_tiles<T, KF, VF, 5>(p, s);
    case 6: return token_tiles<T, KF, VF, 6>(p, s);
    case 7: return token_tiles<T, KF, VF, 7>(p, s);
    default: return token_tiles<T, KF, VF, 8>(p, s);
  }
}

}  // namespace hyp
