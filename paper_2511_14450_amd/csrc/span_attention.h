// Kernels of attention over a shared prefix and a request's own keys (hyp_attn.h), for T = float or bf16_t.  Included by one
// translation unit per type.
//
// A wave works on 32 rows, (row of q, head of the group) pairs, and forms S^T = K Q^T with keys on the M axis of the matrix
// instruction and rows on the N axis: lane l owns row l % 32 and, of a block of 32 keys, keys 8 (i / 4) + 4 (l / 32) + i % 4 in
// register i.  A row's cap, bias, mask, maximum and sum then stay in its two lanes, and the probabilities leave the score
// registers in the order in which O^T += V^T P^T wants them, if that product's keys are taken in the same order.
#pragma once

#include "mfma_common.h"
#include "span_kernels.h"

namespace hyp {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFollow = 8.0f;  // the running maximum moves when a score passes it by more than 2^8

typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16v4_t;
typedef __attribute__((address_space(3))) bf16v4_t lds_bf16v4_t;
typedef int i32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float half_max(float v) {
  const unsigned u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float v) {
  const unsigned u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
// This file is compiled as if no number were NaN, so that a maximum is one instruction.  Where a NaN may stand it is looked at
// as an integer, which the compiler is kept from seeing through.
__device__ __forceinline__ unsigned bits_of(float x) {
  unsigned u = __float_as_uint(x);
  asm("" : "+v"(u));
  return u;
}
__device__ __forceinline__ bool not_finite(float x) { return (bits_of(x) & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool is_zero(float x) { return bits_of(x) == 0u; }
__device__ __forceinline__ bool is_none(float x) { return bits_of(x) == 0xff800000u; }  // the maximum of no score
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) v = min(v, __shfl_xor(v, s));
  return v;
}
__device__ __forceinline__ int wave_max(int v) { return -wave_min(-v); }
__device__ __forceinline__ int clamped(int v, int lo, int hi) { return min(max(v, lo), hi); }

// A raw score S as an exponent of two, cap log2(e) tanh(S scale / cap).  With x = S scale / cap up to 0.625 in absolute value that is
// S r(S^2), r a polynomial fitted to an even relative error (4e-9; 1e-7 as evaluated), whose coefficients the host scales;
// beyond, 1 - 2 / (e^2x + 1), whose absolute error of one rounding is relative there.
__device__ __forceinline__ float cap_factor(float s, const float (&c)[6]) {
  const float y = s * s;
  float q = fmaf(y, c[5], c[4]);
  q = fmaf(y, q, c[3]);
  q = fmaf(y, q, c[2]);
  q = fmaf(y, q, c[1]);
  return fmaf(y, q, c[0]);
}
__device__ __forceinline__ float cap_any(float s, const float (&c)[6], float most, float to_cap, float cap2) {
  const float e = exp2_(2.0f * kLog2e * fabsf(s * to_cap));  // infinity: tanh is 1
  const float far = copysignf(cap2 - 2.0f * cap2 * __builtin_amdgcn_rcpf(e + 1.0f), s);
  return fabsf(s) <= most ? s * cap_factor(s, c) : far;
}

__device__ __forceinline__ float load_val(const float *p) { return *p; }
__device__ __forceinline__ float load_val(const bf16_t *p) { return bf16_to_f32(*p); }

// What a wave's lane knows of its row.
struct SpanRow {
  const void *q;
  int64_t at;      // (row of q) * nq + head
  int64_t out;     // offset of its first feature in `out`
  int lim;         // own keys up to this index are seen; -1: none
  int doc, pos;
  float slope2;    // slope * log2(e)
  bool there;
};

// The keys of an item: shared ones [a0, a1), own ones [b0, b1) of a request.
struct SpanKeys { int a0, a1, b0, b1, req, kvh; };

template <typename T> __device__ __forceinline__ SpanRow span_row(const SpanCall &p, int64_t row, int head, int req, int own_index, bool there) {
  SpanRow r;
  r.there = there;
  r.at = row * p.nq + head;
  r.out = row * p.out_rs + head * p.out_hs;
  r.q = (const T *)p.q + row * p.q_rs + head * p.q_hs;
  r.lim = own_index;
  if (there && p.see_all && p.q_start) r.lim = max(r.lim, p.see_all[req] - 1);
  r.doc = there && p.c.key_doc && p.q_doc ? p.q_doc[row] : -1;
  r.pos = there && p.q_pos ? p.q_pos[row] : p.c.prefix_len + own_index;
  r.slope2 = there && p.slopes ? p.slopes[head] * kLog2e : 0.f;
  if (!there) r.lim = -1;
  return r;
}

__device__ __forceinline__ int span_len(const SpanCall &p, int b) { return clamped(p.c.lens[b], 0, p.c.most); }

__device__ __forceinline__ int64_t own_offset(const hyp_attn_cache_t &c, int page_shift, int64_t page_stride, int64_t head_stride, int64_t key_stride,
                                              int req, int kvh, int j) {
  if (!c.page_table) return (int64_t)req * page_stride + (int64_t)kvh * head_stride + (int64_t)j * key_stride;
  const int page = clamped(c.page_table[(int64_t)req * c.pages_per_request + (j >> page_shift)], 0, c.n_pages - 1);
  return (int64_t)page * page_stride + (int64_t)kvh * head_stride + (int64_t)(j & (c.page_keys - 1)) * key_stride;
}

// pair i of KV head c, counted from `first` over (row of q, head of the group), as (row of q) * nq + head
__device__ inline int64_t pair_at(const SpanCall &p, int64_t first, int kvh, int i) {
  const int64_t x = first + i, row = x / p.G;
  return row * p.nq + kvh * p.G + (x - row * p.G);
}

// RW waves of 32 rows each, KW waves that take turns at the keys; SKW keys of a wave in a stage.
template <typename T, int NT, int RW, int KW, int SKW, bool WIDE> struct Span {
  static constexpr int ES = sizeof(T), NW = RW * KW, THREADS = 64 * NW;
  static constexpr int CPR = span_chunks(NT, ES), ROWB = CPR * 16;  // an LDS row
  static constexpr int EPC = 16 / ES;                               // elements of a piece
  static constexpr int NP = NT * ES / 2;                            // pairs of pieces of a row's features
  static constexpr int NDB = NT / 2;                                // 32-feature blocks of the output
  static constexpr int SKEYS = KW * SKW, NKB = SKW / 32;
  static constexpr int TILE = SKEYS * ROWB, BUF = 2 * TILE;         // keys, then values
  static constexpr int INTS = 2 * BUF;                              // ids and positions of the stages' keys, after two buffers
  static constexpr int LDS = INTS + 2 * 2 * SKEYS * 4;
  static constexpr int JOIN = KW > 1 ? KW * (NDB * 32 * 33 + 64) * 4 : 0;
  static constexpr int LDS_ALL = LDS > JOIN ? LDS : JOIN;
  static_assert(LDS_ALL <= 160 * 1024, "LDS of a CU");

  // LDS has 64 banks of 4 bytes: rows of 16 pieces or more fill them all, rows of 8 half of them.  The pieces of a row are exchanged by the
  // row's number, so that the 16 rows that 16 lanes read a piece of, and the two pieces of four value rows that 32 lanes read, meet in
  // no bank.
  static constexpr int KM = CPR >= 16 ? 15 : 7;
  static __device__ __forceinline__ int kswz(int row) { return row & KM; }
  static __device__ __forceinline__ int vswz(int row) {
    if constexpr (ES == 4) return ((row >> 2) & 1) << 3;
    return CPR >= 16 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
  }

  const SpanCall &p;
  const SpanKeys sg;
  char *lds;
  int wave, lane, hh, col;
  int pre_stages, stages;
  bool has_doc, has_pos, small_page;
  int chunks;  // pieces of a row that hold features

  __device__ __forceinline__ Span(const SpanCall &p_, const SpanKeys &sg_, char *lds_) : p(p_), sg(sg_), lds(lds_) {
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lane = threadIdx.x & 63;
    hh = lane >> 5;
    col = lane & 31;
    pre_stages = (sg.a1 - sg.a0 + SKEYS - 1) / SKEYS;
    stages = pre_stages + (sg.b1 - sg.b0 + SKEYS - 1) / SKEYS;
    has_doc = p.c.key_doc != nullptr && sg.b1 > sg.b0;
    has_pos = p.slopes != nullptr && p.c.key_pos != nullptr;
    small_page = p.c.page_table && p.c.page_keys < SKEYS;
    chunks = p.c.head_dim * ES / 16;
  }

  struct Stage { int base, end; bool own; };
  __device__ __forceinline__ Stage stage_of(int st) const {
    const bool own = st >= pre_stages;
    return {own ? sg.b0 + (st - pre_stages) * SKEYS : sg.a0 + st * SKEYS, own ? sg.b1 : sg.a1, own};
  }

  // Pieces of a row behind the features count as zero in every product; they are never written after this.
  __device__ __forceinline__ void clear_padding() {
    if (!WIDE || chunks < CPR) {
      for (int i = threadIdx.x; i < 2 * BUF / 16; i += THREADS) ((f32x4_t *)lds)[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      __syncthreads();
    }
  }

  // One stage's keys (or values) into LDS.  A whole stage that lies in one page or in none is addressed by a uniform base and a
  // lane offset in 32 bits; else each lane forms its row's address, the rows behind the last key being that key's again.
  template <bool VALUES> __device__ __forceinline__ void load_tile(const Stage &s, char *dst) {
    const T *base = (const T *)(s.own ? (VALUES ? p.c.v : p.c.k) : (VALUES ? p.c.prefix_v : p.c.prefix_k));
    const int64_t ks = s.own ? (VALUES ? p.c.v_key_stride : p.c.k_key_stride) : (VALUES ? p.c.prefix_v_key_stride : p.c.prefix_k_key_stride);
    const int64_t hs = s.own ? (VALUES ? p.c.v_head_stride : p.c.k_head_stride) : (VALUES ? p.c.prefix_v_head_stride : p.c.prefix_k_head_stride);
    const int64_t ps = VALUES ? p.c.v_page_stride : p.c.k_page_stride;
    auto offset = [&](int key) -> int64_t {
      return s.own ? own_offset(p.c, p.page_shift, ps, hs, ks, sg.req, sg.kvh, key) : (int64_t)sg.kvh * hs + (int64_t)key * ks;
    };
    if constexpr (WIDE) {
      constexpr int LOADS = SKEYS * CPR / 64 / NW, ROWS = NW * 64 / CPR;  // rows between a lane's loads
      static_assert(LOADS * 64 * NW == SKEYS * CPR, "a stage is whole loads of all waves");
      const int first = (wave * 64 + lane) / CPR, piece = (wave * 64 + lane) % CPR;
      const bool one_page = s.base + SKEYS <= s.end && !(s.own && small_page);
      if (one_page) {
        const T *start = base + offset(s.base);
        constexpr bool SAME = ROWS % (KM + 1) == 0;  // all of a lane's rows exchange alike
        const unsigned step = (unsigned)(ROWS * ks * ES);
        const int c0 = piece ^ (VALUES ? vswz(first) : kswz(first));
        const unsigned off0 = (unsigned)(first * ks * ES) + c0 * 16;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
          unsigned off = off0;
          int c = c0;
          if constexpr (!SAME) {
            const int row = first + j * ROWS;
            c = piece ^ (VALUES ? vswz(row) : kswz(row));
            off = (unsigned)(first * ks * ES) + c * 16;
          }
          const char *src = (const char *)start + (size_t)j * step;
          if (NT != 6 && chunks == CPR)
            __builtin_amdgcn_global_load_lds((gbl_ptr_t *)(src + off), (lds_ptr_t *)(dst + (j * NW + wave) * 1024), 16, 0, 0);
          else if (c < chunks)
            __builtin_amdgcn_global_load_lds((gbl_ptr_t *)(src + off), (lds_ptr_t *)(dst + (j * NW + wave) * 1024), 16, 0, 0);
        }
      } else {
#pragma unroll 1
        for (int j = 0; j < LOADS; ++j) {
          const int row = first + j * ROWS, c = piece ^ (VALUES ? vswz(row) : kswz(row));
          const char *src = (const char *)(base + offset(min(s.base + row, s.end - 1))) + c * 16;
          if (c < chunks) __builtin_amdgcn_global_load_lds((gbl_ptr_t *)src, (lds_ptr_t *)(dst + (j * NW + wave) * 1024), 16, 0, 0);
        }
      }
    } else {
      const int d = p.c.head_dim;
      for (int i = threadIdx.x; i < SKEYS * d; i += THREADS) {
        const int row = i / d, f = i % d, c = (f / EPC) ^ (VALUES ? vswz(row) : kswz(row));
        ((T *)(dst + row * ROWB + c * 16))[f % EPC] = base[offset(min(s.base + row, s.end - 1)) + f];
      }
    }
  }

  __device__ __forceinline__ void issue(int st, int buf) {
    const Stage s = stage_of(st);
    load_tile<false>(s, lds + buf * BUF);
    load_tile<true>(s, lds + buf * BUF + TILE);
    if (s.own && (has_doc || has_pos)) {
      constexpr int PIECES = SKEYS < 64 ? 1 : SKEYS / 64;
#pragma unroll
      for (int x = 0; x < (2 * PIECES + NW - 1) / NW; ++x) {
        const int i = x * NW + wave;  // piece of 64 (or all SKEYS) ints of one array
        const bool pos = i / PIECES == 1;
        const int j = (i % PIECES) * 64 + lane;
        if (i < 2 * PIECES && j < SKEYS && (pos ? has_pos : has_doc)) {
          const int key = min(s.base + j, s.end - 1);
          const int *src = pos ? p.c.key_pos + sg.req * p.c.key_pos_request_stride + sg.kvh * p.c.key_pos_head_stride + key
                               : p.c.key_doc + sg.req * p.c.key_doc_request_stride + sg.kvh * p.c.key_doc_head_stride + key;
          __builtin_amdgcn_global_load_lds((gbl_ptr_t *)src, (lds_ptr_t *)(lds + INTS + ((buf * 2 + pos) * SKEYS + (i % PIECES) * 64) * 4), 4, 0, 0);
        }
      }
    }
  }

  // A row's features, the operand of the score product that it stays in.
  struct Rows {
    f32x4_t q[NP];  // piece 2 i + hh of the row
  };
  __device__ __forceinline__ void load_rows(const SpanRow &r, Rows &rows) const {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      f32x4_t x = {0.f, 0.f, 0.f, 0.f};
      const int c = 2 * i + hh;
      if (r.there) {
        if constexpr (WIDE) {
          if (c < chunks) x = *(const f32x4_t *)((const char *)r.q + c * 16);
        } else {
          union { f32x4_t v; T t[EPC]; } u = {x};
#pragma unroll
          for (int e = 0; e < EPC; ++e)
            if (c * EPC + e < p.c.head_dim) u.t[e] = ((const T *)r.q)[c * EPC + e];
          x = u.v;
        }
      }
      rows.q[i] = x;
    }
  }

  // scores of one block of 32 keys in LDS
  static __device__ __forceinline__ void block_scores(const char *keys, const Rows &rows, int col, int hh, float *s /*16*/) {
    f32x16_t a;
#pragma unroll
    for (int r = 0; r < 16; ++r) a[r] = 0.f;
    const char *row = keys + col * ROWB;
    const int x = kswz(col);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const f32x4_t k = *(const f32x4_t *)(row + (((2 * i + hh) ^ x) << 4));
      if constexpr (ES == 2) {
        a = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, rows.q[i]), a, 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) a = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], rows.q[i][e], a, 0, 0, 0);
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = a[r];
  }

  static __device__ __forceinline__ int key_of(int i, int hh) { return 8 * (i >> 2) + 4 * hh + (i & 3); }

  // cap and bias of one block of 32 keys from `base` on; kpos: positions of its keys in LDS, or null
  __device__ __forceinline__ void rule(float (&s)[16], const SpanRow &r, int first_pos, const int *kpos) const {
    if (p.cap2 != 0.f) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = cap_any(s[i], p.cap_c, p.cap_most, p.to_cap, p.cap2);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] *= p.scale2;
    }
    if (p.slopes) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        i32x4_t at;
        if (kpos) at = *(const i32x4_t *)(kpos + 8 * g + 4 * hh);
        else
#pragma unroll
          for (int e = 0; e < 4; ++e) at[e] = first_pos + 8 * g + 4 * hh + e;
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * g + e] -= r.slope2 * fabsf((float)(r.pos - at[e]));
      }
    }
  }

  struct State {
    f32x16_t o[NDB];
    float m, l;
  };
  static __device__ __forceinline__ void clear(State &t) {
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) t.o[db][r] = 0.f;
    t.m = -INFINITY;
    t.l = 0.f;
  }

  // One stage's share of a wave.  score_out: where given, this row's scores (key j of the request at [j]).
  __device__ __forceinline__ void compute(const Stage &sta, int buf, const Rows &rows, const SpanRow &r, int lim_lo, int lim_hi, State &t, float *score_out) const {
    const int kw = KW > 1 ? wave / RW : 0;
    const int base = sta.base + kw * SKW;
    if (base >= sta.end || (sta.own && base > lim_hi)) return;
    const char *keys = lds + buf * BUF + kw * SKW * ROWB, *values = lds + buf * BUF + TILE;
    const int *ints = (const int *)(lds + INTS) + buf * 2 * SKEYS + kw * SKW;
    const bool edge = base + SKW > sta.end || (sta.own && base + SKW - 1 > lim_lo), docs = sta.own && has_doc;
    float s[NKB][16];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) block_scores(keys + kb * 32 * ROWB, rows, col, hh, s[kb]);
    // Scores that all rows see and that no distance moves stay raw: cap and scale do not change their order, so the maximum is
    // taken of them as they are, and the last step of either is one instruction with the subtraction of the maximum.
    const bool capped = p.cap2 != 0.f;
    bool raw = !(edge || docs || p.slopes || score_out);
    float mx = -INFINITY;
    if (raw) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, s[kb][i]), s[kb][i + 1]);
      if (capped) {
        float far = 0.f;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; i += 2) far = fmaxf(fmaxf(far, fabsf(s[kb][i])), fabsf(s[kb][i + 1]));
        raw = !__any(!(far <= p.cap_most));
        mx *= cap_factor(mx, p.cap_c);
      } else {
        mx *= p.scale2;
      }
    }
    if (!raw) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
        rule(s[kb], r, (sta.own ? p.c.prefix_len : 0) + base + kb * 32, sta.own && has_pos ? ints + SKEYS + kb * 32 : nullptr);
      if (edge) {
        const int last = sta.own ? min(r.lim, sta.end - 1) : sta.end - 1;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (base + kb * 32 + key_of(i, hh) > last) s[kb][i] = -INFINITY;
      }
      if (docs) {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const i32x4_t id = *(const i32x4_t *)(ints + kb * 32 + 8 * g + 4 * hh);
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (id[e] != r.doc && id[e] >= 0 && r.doc >= 0) s[kb][4 * g + e] = -INFINITY;
          }
      }
      if (score_out && sta.own && r.there) {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int g = 0; g < 4; ++g)  // up to the row's pitch, a multiple of the stage
            *(f32x4_t *)(score_out + base + kb * 32 + 8 * g + 4 * hh) = f32x4_t{s[kb][4 * g], s[kb][4 * g + 1], s[kb][4 * g + 2], s[kb][4 * g + 3]};
      }
      mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; i += 2) mx = fmaxf(fmaxf(mx, s[kb][i]), s[kb][i + 1]);
    }
    const float m_new = fmaxf(t.m, half_max(mx));
    if (__any(m_new - t.m > kFollow)) {
      const float alpha = m_new == -INFINITY ? 1.0f : exp2_(t.m - m_new);
      t.l *= alpha;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) t.o[db][i] *= alpha;
      t.m = m_new;
    }
    const float m = t.m == -INFINITY ? 0.f : t.m;  // a row that has seen nothing yet: all its probabilities are 2^-inf
    if (raw && capped) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = exp2_(fmaf(s[kb][i], cap_factor(s[kb][i], p.cap_c), -m));
    } else {
      const float c = raw ? p.scale2 : 1.0f;
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[kb][i] = exp2_(fmaf(s[kb][i], c, -m));
    }
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += s[kb][i];
      t.l += sum;
    }
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
      const int row0 = kw * SKW + kb * 32;
      if constexpr (ES == 2) {
#pragma unroll
        for (int m2 = 0; m2 < 2; ++m2) {
          bf16x8_t pf;
#pragma unroll
          for (int e = 0; e < 8; ++e) pf[e] = (__bf16)s[kb][8 * m2 + e];
          // 16 lanes read four rows of 16 features and get a feature's four rows each
          const int g16 = (lane >> 4) & 1, i16 = lane & 15;
          const int ra = row0 + 16 * m2 + 4 * hh + (i16 >> 2), rb = ra + 8;
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            const int c = 4 * db + 2 * g16 + ((i16 & 3) >> 1);
            const bf16v4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16v4_t *)(values + ra * ROWB + ((c ^ vswz(ra)) << 4) + (i16 & 1) * 8));
            const bf16v4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16v4_t *)(values + rb * ROWB + ((c ^ vswz(rb)) << 4) + (i16 & 1) * 8));
            const bf16x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            t.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf, t.o[db], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = row0 + key_of(i, hh);
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            const float v = *(const float *)(values + row * ROWB + (((8 * db + (col >> 2)) ^ vswz(row)) << 4) + (col & 3) * 4);
            t.o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[kb][i], t.o[db], 0, 0, 0);
          }
        }
      }
    }
  }

  // A value that a row does not see is multiplied by a probability of zero; if it is an infinity or a NaN that is no zero.  Then, as
  // where a sum leaves the range of a float although the result does not, a wave's rows are summed again one key at a time, with
  // their final weights, from memory.  Slow, and right.  The result is the one of a sum of one.
  __device__ __forceinline__ void careful(int st0, int st1, const SpanRow &r, State &t) const {
    const int kw = KW > 1 ? wave / RW : 0, d = p.c.head_dim;
    if (!is_zero(t.l)) {
      t.m += __builtin_amdgcn_logf(t.l);
      t.l = 1.0f;
    }
    const float m = t.m;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) t.o[db][i] = 0.f;
    for (int st = st0; st < st1; ++st) {
      const Stage sta = stage_of(st);
      const int base = sta.base + kw * SKW, end = min(base + SKW, sta.end);
      for (int key = base; key < end; ++key) {
        bool seen = r.there && (!sta.own || key <= r.lim);
        int64_t ko, vo;
        int pos = key;
        if (sta.own) {
          ko = own_offset(p.c, p.page_shift, p.c.k_page_stride, p.c.k_head_stride, p.c.k_key_stride, sg.req, sg.kvh, key);
          vo = own_offset(p.c, p.page_shift, p.c.v_page_stride, p.c.v_head_stride, p.c.v_key_stride, sg.req, sg.kvh, key);
          pos = p.c.prefix_len + key;
          if (has_pos) pos = p.c.key_pos[sg.req * p.c.key_pos_request_stride + sg.kvh * p.c.key_pos_head_stride + key];
          if (has_doc) {
            const int id = p.c.key_doc[sg.req * p.c.key_doc_request_stride + sg.kvh * p.c.key_doc_head_stride + key];
            if (id != r.doc && id >= 0 && r.doc >= 0) seen = false;
          }
        } else {
          ko = sg.kvh * p.c.prefix_k_head_stride + key * p.c.prefix_k_key_stride;
          vo = sg.kvh * p.c.prefix_v_head_stride + key * p.c.prefix_v_key_stride;
        }
        if (!seen || is_zero(t.l)) continue;
        const T *k = (const T *)(sta.own ? p.c.k : p.c.prefix_k) + ko, *v = (const T *)(sta.own ? p.c.v : p.c.prefix_v) + vo;
        float dot = 0.f;
        for (int f = 0; f < d; ++f) dot = fmaf(load_val((const T *)r.q + f), load_val(k + f), dot);
        dot = p.cap2 != 0.f ? cap_any(dot, p.cap_c, p.cap_most, p.to_cap, p.cap2) : dot * p.scale2;
        if (p.slopes) dot -= r.slope2 * fabsf((float)(r.pos - pos));
        const float pr = exp2_(dot - m);
        if (is_zero(pr)) continue;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int f = 32 * db + key_of(i, hh);
            if (f < d) t.o[db][i] = fmaf(pr, load_val(v + f), t.o[db][i]);
          }
      }
    }
  }

  __device__ __forceinline__ void attend(int st0, int st1, const SpanRow &r, State &t, float *score_out) {
    clear(t);
    if (st0 >= st1) return;
    clear_padding();
    issue(st0, 0);
    Rows rows;
    load_rows(r, rows);
    const int lim_lo = __builtin_amdgcn_readfirstlane(wave_min(r.there ? r.lim : 0x7fffffff)), lim_hi = __builtin_amdgcn_readfirstlane(wave_max(r.lim));
    int buf = 0;
    for (int st = st0; st < st1; ++st) {
      __builtin_amdgcn_s_waitcnt(0x0070);  // this wave's share of the stage has landed
      __syncthreads();                     // all shares have, and the other buffer is free
      if (st + 1 < st1) issue(st + 1, buf ^ 1);
      compute(stage_of(st), buf, rows, r, lim_lo, lim_hi, t, score_out);
      buf ^= 1;
    }
    t.l = half_sum(t.l);
    bool odd = false;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd |= not_finite(t.o[db][i]);
    if (__any(odd && r.there)) careful(st0, st1, r, t);
  }

  // A row's result straight from its registers: normalised, or as partial result of `slot`.
  __device__ __forceinline__ void store_rows(const SpanRow &r, const State &t, int slot) const {
    if (!r.there) return;
    const int d = p.c.head_dim;
    const bool none = is_zero(t.l);
    const float inv = none ? 0.f : 1.0f / t.l;
    if (p.part_o) {
      const int64_t at = (int64_t)slot * p.n_rows * p.nq + r.at;
      if (hh == 0) {
        p.part_ml[2 * at] = none ? -INFINITY : t.m;
        p.part_ml[2 * at + 1] = t.l;
      }
      if (none) return;
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int f = 32 * db + 8 * g + 4 * hh;
          float *dst = p.part_o + at * d + f;
          f32x4_t x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = t.o[db][4 * g + e] * inv;
          if ((d & 3) == 0) {
            if (f < d) *(f32x4_t *)dst = x;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (f + e < d) dst[e] = x[e];
          }
        }
      return;
    }
    if (p.lse && hh == 0) p.lse[r.at] = none ? -INFINITY : (t.m + __builtin_amdgcn_logf(t.l)) * kLn2;
    T *out = (T *)p.out + r.out;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int f = 32 * db + 8 * g + 4 * hh;
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = none ? 0.f : t.o[db][4 * g + e] * inv;
        if (p.out_vec) {
          if (f < d) {
            if constexpr (ES == 2) *(bf16x4_t *)(out + f) = pack4(x[0], x[1], x[2], x[3]);
            else *(f32x4_t *)(out + f) = f32x4_t{x[0], x[1], x[2], x[3]};
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (f + e < d) store_f32(out + f + e, x[e]);
        }
      }
  }

  // The waves that took turns at the keys of the same 32 rows, joined through LDS; rows: how many there are, row r being the
  // pair (r / G, r % G) from `first` on.
  __device__ __forceinline__ void join_waves(const State &t, int rows, int64_t first, int slot) const {
    static_assert(RW == 1, "rows of one wave");
    constexpr int PER = NDB * 32 * 33 + 64;
    float *mine = (float *)lds + wave * PER;
    __syncthreads();  // the stages are done with
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) mine[64 + (32 * db + key_of(i, hh)) * 33 + col] = t.o[db][i];
    if (hh == 0) {
      mine[col] = is_zero(t.l) ? -INFINITY : t.m;
      mine[32 + col] = t.l;
    }
    __syncthreads();
    const int d = p.c.head_dim;
    for (int i = threadIdx.x; i < rows * d; i += THREADS) {
      const int row = i / d, f = i - row * d;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < KW; ++w) m = fmaxf(m, ((float *)lds)[w * PER + row]);
      float l = 0.f, o = 0.f, a[KW];
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float *x = (float *)lds + w * PER;
        a[w] = is_none(x[row]) ? 0.f : exp2_(x[row] - m);
        if (!is_zero(a[w])) l += a[w] * x[32 + row];
      }
      const float inv = 1.0f / l;
#pragma unroll
      for (int w = 0; w < KW; ++w)
        if (!is_zero(a[w])) o += a[w] * inv * ((float *)lds)[w * PER + 64 + f * 33 + row];
      const int64_t pair = pair_at(p, first, sg.kvh, row), r = pair / p.nq;
      const int head = (int)(pair - r * p.nq);
      if (p.part_o) {
        const int64_t to = (int64_t)slot * p.n_rows * p.nq + pair;
        p.part_o[to * d + f] = o;
        if (f == 0) {
          p.part_ml[2 * to] = is_zero(l) ? -INFINITY : m;
          p.part_ml[2 * to + 1] = l;
        }
      } else {
        store_f32((T *)p.out + r * p.out_rs + head * p.out_hs + f, o);
        if (f == 0 && p.lse) p.lse[pair] = is_zero(l) ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
      }
    }
  }
};

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
  req = lo;
  row0 = start(lo);
  rows = (int)max(start(lo + 1) - row0, (int64_t)0);
  const int64_t first = ((int64_t)t - (row0 * p.G / tile + lo)) * tile;
  return first >= 0 && first < (int64_t)rows * p.G ? first : -1;
}

// attn_prompt.  A workgroup: one KV head, 128 rows of one request (dense over the group's heads), all the keys they see or one
// of `splits` parts of them.
template <typename T, int NT, bool WIDE> __global__ void __launch_bounds__(64 * kSpanWaves, span_steps_waves(NT)) k_span_prompt(const SpanCall p) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  using S = Span<T, NT, kSpanWaves, 1, span_stage_keys(NT, sizeof(T)), WIDE>;
  int id = blockIdx.x;
  const int kvh = id % p.c.n_kv_heads;
  id /= p.c.n_kv_heads;
  const int split = id % p.splits;
  const int tile = p.tiles - 1 - id / p.splits;
  int req, n;
  int64_t row0;
  const int64_t first = tile_request(p, tile, kSpanTile, req, row0, n);
  if (first < 0) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = threadIdx.x & 31;
  const int len = span_len(p, req);
  const int64_t pair = first + wave * 32 + col;
  const bool there = pair < (int64_t)n * p.G;
  const int i = there ? (int)(pair / p.G) : 0, g = there ? (int)(pair - (int64_t)i * p.G) : 0;
  const SpanRow r = span_row<T>(p, row0 + i, kvh * p.G + g, req, len - n + i, there);
  // the last row's reach, and the keys all of the request's rows see
  const int last = (int)(min(first + kSpanTile, (int64_t)n * p.G) - 1) / p.G;
  int end = len - n + last + 1;
  if (p.see_all) end = max(end, p.see_all[req]);
  S span(p, SpanKeys{0, p.c.prefix_len, 0, clamped(end, 0, len), req, kvh}, lds);
  const int st0 = (int)((int64_t)span.stages * split / p.splits), st1 = (int)((int64_t)span.stages * (split + 1) / p.splits);
  typename S::State t;
  span.attend(st0, st1, r, t, nullptr);
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
      const SpanRow r = span_row<T>(p, b, kvh * p.G + (there ? pair - b * p.G : 0), b, span_len(p, b) - 1, there);
      Pre span(p, SpanKeys{0, p.c.prefix_len, 0, 0, 0, kvh}, lds);
      typename Pre::State t;
      span.attend((int)((int64_t)span.stages * split / p.pre_splits), (int)((int64_t)span.stages * (split + 1) / p.pre_splits), r, t, nullptr);
      span.store_rows(r, t, split);
      return;
    }
    const int pair = tile * 32 + col;
    const bool there = pair < all;
    const int b = there ? pair / p.G : 0;
    const SpanRow r = span_row<T>(p, b, kvh * p.G + (there ? pair - b * p.G : 0), b, span_len(p, b) - 1, there);
    Own span(p, SpanKeys{0, p.c.prefix_len, 0, 0, 0, kvh}, lds);
    typename Own::State t;
    span.attend((int)((int64_t)span.stages * split / p.pre_splits), (int)((int64_t)span.stages * (split + 1) / p.pre_splits), r, t, nullptr);
    span.join_waves(t, min(32, all - tile * 32), tile * 32, split);
    return;
  }
  const int split = id % p.splits;
  id /= p.splits;
  const int tile = id % p.tiles, b = id / p.tiles;
  const int g = tile * 32 + col, rows = min(32, p.G - tile * 32);
  const bool there = col < rows;
  const int len = span_len(p, b);
  const SpanRow r = span_row<T>(p, b, kvh * p.G + (there ? g : 0), b, len - 1, there);
  Own span(p, SpanKeys{0, 0, 0, len, b, kvh}, lds);
  typename Own::State t;
  float *scores = p.scores ? p.scores + (((int64_t)b * p.c.n_kv_heads + kvh) * p.G + (there ? g : 0)) * p.score_pitch : nullptr;
  span.attend((int)((int64_t)span.stages * split / p.splits), (int)((int64_t)span.stages * (split + 1) / p.splits), r, t, scores);
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
  const int len = span_len(p, b);
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
  const int len = span_len(p, b), key0 = kb * kSpanReceivedKeys;
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
    SpanRow r;
    r.there = true;
    r.q = (const T *)p.c.k + own_offset(p.c, p.page_shift, p.c.k_page_stride, p.c.k_head_stride, p.c.k_key_stride, b, kvh, key);
    span.load_rows(r, keys);
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
    x.r = span_row<T>(p, row, head_of(there ? pair : 0), b, len - n + (int)(row - row0), there);
    const float lse = there ? p.lse_in[x.r.at] : -INFINITY;
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
    return span_launch<NT, W>(k_span_prompt<T, NT, W>, Span<T, NT, kSpanWaves, 1, span_stage_keys(NT, sizeof(T)), W>::LDS_ALL,
                              (unsigned)p.tiles * p.splits * p.c.n_kv_heads, 64 * kSpanWaves, p, s);
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
