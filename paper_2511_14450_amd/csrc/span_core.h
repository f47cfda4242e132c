// What the kernels of attention over a shared prefix and a request's own keys (hyp_attn.h) are made of, for T = float or bf16_t.
//
// A wave works on 32 rows, (row of q, head of the group) pairs, and forms S^T = K Q^T with keys on the M axis of the matrix
// instruction and rows on the N axis: lane l owns row l % 32 and, of a block of 32 keys, keys 8 (i / 4) + 4 (l / 32) + i % 4 in
// register i.  A row's cap, bias, mask, maximum and sum then stay in its two lanes, and the probabilities leave the score
// registers in the order in which O^T += V^T P^T wants them, if that product's keys are taken in the same order.
#pragma once

#include "attn_score.h"
#include "mfma_common.h"
#include "span_kernels.h"

namespace hyp {
namespace {

constexpr float kLog2eLow = (float)(1.4426950408889634 - (double)kLog2e), kLn2 = 0.6931471805599453f;
constexpr float kFollow = 8.0f;  // the running maximum moves when a score passes it by more than 2^8

typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16v4_t;
typedef __attribute__((address_space(3))) f32x4_t lds_f32x4_t;
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
// This file is compiled as if no number were NaN, so that a maximum is one instruction.  Where a NaN may stand it is looked at
// as an integer, which the compiler is kept from seeing through.
__device__ __forceinline__ unsigned bits_of(float x) {
  unsigned u = __float_as_uint(x);
  asm("" : "+v"(u));
  return u;
}
__device__ __forceinline__ bool not_finite(float x) { return (bits_of(x) & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool is_nan(float x) { return (bits_of(x) & 0x7fffffffu) > 0x7f800000u; }
__device__ __forceinline__ bool is_zero(float x) { return bits_of(x) == 0u; }
__device__ __forceinline__ bool is_none(float x) { return bits_of(x) == 0xff800000u; }  // the maximum of no score
// A value the compiler does not know to be the same in the next trip of a loop: what is formed of it is formed again there, instead of
// staying in registers throughout.
__device__ __forceinline__ unsigned here(unsigned v) {
  asm volatile("" : "+v"(v));
  return v;
}
// a value that is the same in all lanes, which the compiler does not see where it comes from memory
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) v = min(v, __shfl_xor(v, s));
  return v;
}
__device__ __forceinline__ int wave_max(int v) {  // not the negated minimum: -2^31, which is an id as well, has no negative
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) v = max(v, __shfl_xor(v, s));
  return v;
}
__device__ __forceinline__ int clamped(int v, int lo, int hi) { return min(max(v, lo), hi); }

__device__ __forceinline__ float load_val(const float *p) { return *p; }
__device__ __forceinline__ float load_val(const bf16_t *p) { return bf16_to_f32(*p); }

// What a wave's lane knows of its row.
struct SpanRow {
  int row, head;   // of q
  int lim;         // own keys up to this index are seen; -1: none
  int doc, pos;
  float slope2;    // slope * log2(e)
  bool there;
};

// All stages in turn.
struct EveryStage {
  int own_from;     // ids, where there are any, may hide keys from here on
  __device__ __forceinline__ int next(int st, int st1) const { return min(st, st1); }
  __device__ __forceinline__ bool hides(int st) const { return st >= own_from; }
};

// The keys of an item: shared ones [a0, a1), own ones [b0, b1) of a request.
struct SpanKeys { int a0, a1, b0, b1, req, kvh; };

__device__ __forceinline__ SpanRow span_row(const SpanCall &p, int row, int head, int req, int own_index, bool there) {
  SpanRow r;
  r.there = there;
  r.row = row;
  r.head = head;
  r.lim = own_index;
  if (there && p.see_all && p.q_start) r.lim = max(r.lim, max(p.see_all[req], 0) - 1);  // no less than none: -2^31 has no predecessor
  r.doc = there && p.c.key_doc && p.q_doc ? p.q_doc[row] : -1;
  r.pos = there && p.q_pos ? p.q_pos[row] : p.c.prefix_len + own_index;
  r.slope2 = there && p.slopes ? p.slopes[head] * kLog2e : 0.f;
  if (!there) r.lim = -1;
  return r;
}
__device__ __forceinline__ int64_t row_pair(const SpanCall &p, const SpanRow &r) { return (int64_t)r.row * p.nq + r.head; }
template <typename T> __device__ __forceinline__ const T *row_q(const SpanCall &p, const SpanRow &r) {
  return (const T *)p.q + (int64_t)r.row * p.q_rs + (int64_t)r.head * p.q_hs;
}

__device__ __forceinline__ int span_len(const SpanCall &p, int b) { return clamped(p.c.lens[b], 0, p.c.most); }

__device__ __forceinline__ int64_t own_offset(const hyp_attn_cache_t &c, int page_shift, int64_t page_stride, int64_t head_stride, int64_t key_stride,
                                              int req, int kvh, int j) {
  if (!c.page_table) return (int64_t)req * page_stride + (int64_t)kvh * head_stride + (int64_t)j * key_stride;
  const int page = clamped(c.page_table[(int64_t)req * c.pages_per_request + (j >> page_shift)], 0, c.n_pages - 1);
  return (int64_t)page * page_stride + (int64_t)kvh * head_stride + (int64_t)(j & (c.page_keys - 1)) * key_stride;
}

// stages [at(part), at(part + 1)) of `stages` are part `part` of `parts`
__device__ __forceinline__ int part_start(int stages, int part, int parts) {
  if (parts == 1) return part ? stages : 0;
  const int each = stages / parts, more = stages - each * parts;
  return part * each + min(part, more);
}

// RW waves of 32 rows each, KW waves that take turns at the keys; SKW keys of a wave in a stage; NBUF stages in LDS: with one, another
// workgroup of the CU computes while this one loads.
template <typename T, int NT, int RW, int KW, int SKW, int NBUF, bool WIDE> struct Span {
  static constexpr int ES = sizeof(T), NW = RW * KW, THREADS = 64 * NW;
  static constexpr int CPR = span_chunks(NT, ES), ROWB = CPR * 16;  // an LDS row
  static constexpr int EPC = 16 / ES;                               // elements of a piece
  static constexpr int NP = NT * ES / 2;                            // pairs of pieces of a row's features
  static constexpr int NDB = NT / 2;                                // 32-feature blocks of the output
  static constexpr int SKEYS = KW * SKW, NKB = SKW / 32;
  static constexpr int TILE = SKEYS * ROWB, BUF = 2 * TILE;         // keys, then values
  static constexpr int INTS = NBUF * BUF;                           // ids and positions of the stages' keys, after the buffers
  static constexpr int LDS = INTS + NBUF * 2 * SKEYS * 4;
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

  // where the first row of a stage in one page starts, in scalar registers
  template <bool VALUES> __device__ __forceinline__ int64_t uniform_offset(const Stage &s) const {
    const int64_t ks = s.own ? (VALUES ? p.c.v_key_stride : p.c.k_key_stride) : (VALUES ? p.c.prefix_v_key_stride : p.c.prefix_k_key_stride);
    const int64_t hs = s.own ? (VALUES ? p.c.v_head_stride : p.c.k_head_stride) : (VALUES ? p.c.prefix_v_head_stride : p.c.prefix_k_head_stride);
    const int64_t ps = VALUES ? p.c.v_page_stride : p.c.k_page_stride;
    if (!s.own) return (int64_t)sg.kvh * hs + (int64_t)s.base * ks;
    if (!p.c.page_table) return (int64_t)sg.req * ps + (int64_t)sg.kvh * hs + (int64_t)s.base * ks;
    // a scalar load: a vector one would be waited for together with the keys and values in flight
    const int page = clamped(((const __attribute__((address_space(4))) int *)(uintptr_t)p.c.page_table)[(int64_t)sg.req * p.c.pages_per_request + (s.base >> p.page_shift)], 0, p.c.n_pages - 1);
    return (int64_t)page * ps + (int64_t)sg.kvh * hs + (int64_t)(s.base & (p.c.page_keys - 1)) * ks;
  }

  // Pieces of a row behind the features count as zero in every product; they are never written after this.
  __device__ __forceinline__ void clear_padding() {
    if (!WIDE || chunks < CPR) {
      for (int i = threadIdx.x; i < NBUF * BUF / 16; i += THREADS) ((f32x4_t *)lds)[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
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
      constexpr bool SAME = ROWS % (KM + 1) == 0;  // all of a lane's rows exchange alike
      auto fetch = [&](const char *src, int j, bool on) {
        if (on) __builtin_amdgcn_global_load_lds((gbl_ptr_t *)src, (lds_ptr_t *)(dst + (j * NW + wave) * 1024), 16, 0, 0);
      };
      const bool one_page = !(s.own && small_page), whole = s.base + SKEYS <= s.end;
      const unsigned row_bytes = (unsigned)(ks * ES);
      if (one_page && whole) {
        const char *start = (const char *)(base + uniform_offset<VALUES>(s));
        const unsigned step = ROWS * row_bytes, here = (unsigned)first * row_bytes;
        const int c0 = piece ^ (VALUES ? vswz(first) : kswz(first));
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
          const int c = SAME ? c0 : piece ^ (VALUES ? vswz(first + j * ROWS) : kswz(first + j * ROWS));
          const char *src = start + (size_t)j * step + (here + (unsigned)c * 16u);
          if (NT != 6 && chunks == CPR) fetch(src, j, true);
          else fetch(src, j, c < chunks);
        }
      } else if (KW > 1 && one_page) {
        // the rows behind the last key are that key again, up to the end of its wave's block
        const char *start = (const char *)(base + uniform_offset<VALUES>(s));
        const int last = s.end - 1 - s.base, need = (last / SKW + 1) * SKW;
#pragma unroll(LOADS > 8 ? 4 : LOADS)  // the widest rows have 32 loads, whose addresses do not fit the registers
        for (int j = 0; j < LOADS; ++j) {
          const int row = first + j * ROWS, c = piece ^ (VALUES ? vswz(row) : kswz(row));
          fetch(start + ((unsigned)min(row, last) * row_bytes + (unsigned)c * 16u), j, c < chunks && row < need);
        }
      } else {
#pragma unroll 1
        for (int j = 0; j < LOADS; ++j) {
          const int row = first + j * ROWS, c = piece ^ (VALUES ? vswz(row) : kswz(row));
          fetch((const char *)(base + offset(min(s.base + row, s.end - 1))) + c * 16, j, c < chunks);
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
  __device__ __forceinline__ void load_rows(const SpanRow &r, Rows &rows) const { load_row(row_q<T>(p, r), r.there, rows); }
  __device__ __forceinline__ void load_row(const T *q, bool there, Rows &rows) const {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      f32x4_t x = {0.f, 0.f, 0.f, 0.f};
      const int c = 2 * i + hh;
      if (there) {
        if constexpr (WIDE) {
          if (c < chunks) x = *(const f32x4_t *)((const char *)q + c * 16);
        } else {
          union { f32x4_t v; T t[EPC]; } u = {x};
#pragma unroll
          for (int e = 0; e < EPC; ++e)
            if (c * EPC + e < p.c.head_dim) u.t[e] = q[c * EPC + e];
          x = u.v;
        }
      }
      rows.q[i] = x;
    }
  }

  static __device__ __forceinline__ unsigned lds_at(const char *at) { return (unsigned)(uintptr_t)(lds_ptr_t *)(void *)at; }

  // scores of the stage's blocks of 32 keys; products of the blocks in turn, each operand requested AHEAD products before its own
  static __device__ __forceinline__ void block_scores(const char *keys, const Rows &rows, int col, int hh, f32x16_t (&a)[NKB]) {
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) a[kb][r] = 0.f;
    constexpr int ALL = NP * NKB, AHEAD = ES == 2 ? (ALL < 6 ? ALL : 6) : 2;
    const unsigned row = here(lds_at(keys) + col * ROWB + ((hh ^ kswz(col)) << 4));  // pieces of a row lie an exclusive or apart
    auto piece = [&](int i) { return *(const lds_f32x4_t *)((row ^ ((i / NKB) << 5)) + (i % NKB) * 32 * ROWB); };
    f32x4_t k[ALL];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) k[i] = piece(i);
#pragma unroll
    for (int i = 0; i < ALL; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      f32x16_t &x = a[i % NKB];
      const f32x4_t &q = rows.q[i / NKB];
      if constexpr (ES == 2) {
        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, k[i]), __builtin_bit_cast(bf16x8_t, q), x, 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(k[i][e], q[e], x, 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (i + AHEAD < ALL) k[i + AHEAD] = piece(i + AHEAD);
    }
    __builtin_amdgcn_sched_barrier(0);
  }

  // 16 lanes read four rows of 16 features of a block's values, and get a feature's four rows each
  __device__ __forceinline__ unsigned value_address(const char *values) const {
    const int i16 = lane & 15, row = 4 * hh + (i16 >> 2);
    return lds_at(values) + row * ROWB + (((2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ vswz(row)) << 4) + (i16 & 1) * 8;
  }
  // The operands of 16 keys' values, all feature blocks.  Not the builtin: the compiler has it wait for the next stage's loads to LDS, which
  // it cannot know apart.  The reads are waited for here.
  typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));
  template <int AT> static __device__ __forceinline__ void read_values(unsigned at, bf16x8_t (&v)[NDB]) {
    static_assert(NDB == 2 || NDB == 3 || NDB == 4 || NDB == 8, "feature blocks");
    constexpr int LO = AT * 16 * ROWB, HI = LO + 8 * ROWB;
    static_assert(HI < 65536, "offset field");
    u32x2_t r[2 * NDB];
    if constexpr (NDB == 2) {
      asm volatile("ds_read_b64_tr_b16 %0, %4 offset:%6\n\tds_read_b64_tr_b16 %1, %4 offset:%7\n\tds_read_b64_tr_b16 %2, %5 offset:%6\n\t"
                   "ds_read_b64_tr_b16 %3, %5 offset:%7\n\ts_waitcnt lgkmcnt(0)"
                   : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]) : "v"(at), "v"(at ^ 64), "n"(LO), "n"(HI) : "memory");
    } else if constexpr (NDB == 3) {
      asm volatile("ds_read_b64_tr_b16 %0, %6 offset:%9\n\tds_read_b64_tr_b16 %1, %6 offset:%10\n\tds_read_b64_tr_b16 %2, %7 offset:%9\n\t"
                   "ds_read_b64_tr_b16 %3, %7 offset:%10\n\tds_read_b64_tr_b16 %4, %8 offset:%9\n\tds_read_b64_tr_b16 %5, %8 offset:%10\n\ts_waitcnt lgkmcnt(0)"
                   : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5])
                   : "v"(at), "v"(at ^ 64), "v"(at ^ 128), "n"(LO), "n"(HI) : "memory");
    } else {
#pragma unroll
      for (int h = 0; h < NDB; h += 4)
        asm volatile("ds_read_b64_tr_b16 %0, %8 offset:%12\n\tds_read_b64_tr_b16 %1, %8 offset:%13\n\tds_read_b64_tr_b16 %2, %9 offset:%12\n\t"
                     "ds_read_b64_tr_b16 %3, %9 offset:%13\n\tds_read_b64_tr_b16 %4, %10 offset:%12\n\tds_read_b64_tr_b16 %5, %10 offset:%13\n\t"
                     "ds_read_b64_tr_b16 %6, %11 offset:%12\n\tds_read_b64_tr_b16 %7, %11 offset:%13\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(r[2 * h]), "=&v"(r[2 * h + 1]), "=&v"(r[2 * h + 2]), "=&v"(r[2 * h + 3]), "=&v"(r[2 * h + 4]), "=&v"(r[2 * h + 5]),
                       "=&v"(r[2 * h + 6]), "=&v"(r[2 * h + 7])
                     : "v"(at ^ (h << 6)), "v"(at ^ ((h + 1) << 6)), "v"(at ^ ((h + 2) << 6)), "v"(at ^ ((h + 3) << 6)), "n"(LO), "n"(HI) : "memory");
    }
#pragma unroll
    for (int db = 0; db < NDB; ++db)
      v[db] = __builtin_shufflevector(__builtin_bit_cast(bf16v4_t, r[2 * db]), __builtin_bit_cast(bf16v4_t, r[2 * db + 1]), 0, 1, 2, 3, 4, 5, 6, 7);
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
      const int h4 = here(4 * hh);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        i32x4_t at;
        if (kpos) at = *(const i32x4_t *)(kpos + 8 * g + h4);
        else
#pragma unroll
          for (int e = 0; e < 4; ++e) at[e] = first_pos + 8 * g + h4 + e;
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

  // One stage's share of a wave.  docs: ids may hide some of its keys; score_out: where given, this row's scores (key j of the request at [j]).
  __device__ __forceinline__ void compute(const Stage &sta, int buf, const Rows &rows, const SpanRow &r, int lim_lo, int lim_hi, bool docs, State &t, float *score_out) const {
    const int kw = KW > 1 ? wave / RW : 0;
    const int base = sta.base + kw * SKW;
    if (base >= sta.end || (sta.own && base > lim_hi)) return;
    const char *keys = lds + buf * BUF + kw * SKW * ROWB, *values = lds + buf * BUF + TILE + kw * SKW * ROWB;
    const int *ints = (const int *)(lds + INTS) + buf * 2 * SKEYS + kw * SKW;
    const bool edge = base + SKW > sta.end || (sta.own && base + SKW - 1 > lim_lo);
    f32x16_t a[NKB];
    block_scores(keys, rows, col, hh, a);
    // the first values' operands come while the last scores are formed
    bf16x8_t v[2][NDB];
    const unsigned va = here(value_address(values));
    if constexpr (ES == 2) read_values<0>(va, v[0]);
    float s[NKB][16];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kb][i] = a[kb][i];
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
        const int left = (int)here((sta.own ? min(r.lim, sta.end - 1) : sta.end - 1) - base - 4 * hh);
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (kb * 32 + key_of(i, 0) > left) s[kb][i] = -INFINITY;
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
    if constexpr (ES == 2) {
      // Probabilities are rounded to the matrix instruction's bf16, their sum is not: results of 128 bf16 features are 2.3e-3 from 64 bits
      // instead of 1.7e-3, which rounding them alone takes.  In two parts of eight bits they would cost these products twice.
      auto add = [&](auto at) {  // 16 keys: their probabilities rounded, their values added, the next ones' operands fetched behind the products
        constexpr int AT = decltype(at)::value;
        bf16x8_t pf;
#pragma unroll
        for (int e = 0; e < 8; ++e) pf[e] = (__bf16)s[AT / 2][8 * (AT & 1) + e];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int db = 0; db < NDB; ++db) t.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[AT & 1][db], pf, t.o[db], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (AT + 1 < 2 * NKB) read_values<AT + 1>(va, v[(AT + 1) & 1]);
      };
      add(std::integral_constant<int, 0>());
      add(std::integral_constant<int, 1>());
      if constexpr (NKB > 1) {
        add(std::integral_constant<int, 2>());
        add(std::integral_constant<int, 3>());
      }
    } else {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int row = kb * 32 + key_of(i, hh);
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            const float x = *(const float *)(values + row * ROWB + (((8 * db + (col >> 2)) ^ vswz(row)) << 4) + (col & 3) * 4);
            t.o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[kb][i], t.o[db], 0, 0, 0);
          }
        }
    }
  }

  // A value that a row does not see is multiplied by a probability of zero; if it is an infinity or a NaN that is no zero.  Then, as
  // where a sum leaves the range of a float although the result does not, those features of a wave's rows that are not finite are summed
  // again one key at a time, with the rows' final weights, from memory: slow, and right.  It ends as soon as all of them are NaN, which
  // no key undoes; a row whose sum of weights is none has only NaN from the start.  The result is the one of a sum of one.
  template <typename Way> __device__ __forceinline__ void careful(int st0, int st1, const SpanRow &r, State &t, const Way &way) const {
    const int kw = KW > 1 ? wave / RW : 0, d = p.c.head_dim;
    const bool none = is_zero(t.l), lost = not_finite(t.l);
    if (lost) t.m = t.l;  // whatever this part is joined with
    const bool sums = r.there && !none && !lost;
    const float inv = sums ? 1.0f / t.l : 1.0f;
    if (sums) {
      t.m += __builtin_amdgcn_logf(t.l);
      t.l = 1.0f;
    }
    unsigned again[NDB];  // a bit for each feature that is summed again
    bool open = false;    // whether some of them is not NaN yet
#pragma unroll
    for (int db = 0; db < NDB; ++db) {
      again[db] = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const bool odd = sums && not_finite(t.o[db][i]);
        if (odd && 32 * db + key_of(i, hh) < d) again[db] |= 1u << i;
        t.o[db][i] = odd || none ? 0.f : t.o[db][i] * inv;
      }
      open |= again[db] != 0;
    }
    const float m = t.m;
    const T *q = row_q<T>(p, r);
    for (int st = way.next(st0, st1); st < st1; st = way.next(st + 1, st1)) {
      const Stage sta = stage_of(st);
      const int base = sta.base + kw * SKW, end = min(base + SKW, sta.end);
      for (int key = base; key < end; ++key) {
        if (!__any(open)) return;
        bool seen = open && (!sta.own || key <= r.lim);
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
        if (seen) {
          const T *k = (const T *)(sta.own ? p.c.k : p.c.prefix_k) + ko, *v = (const T *)(sta.own ? p.c.v : p.c.prefix_v) + vo;
          float dot = 0.f;
#pragma unroll 8  // so many features' loads at once; the values' would not find registers
          for (int f = 0; f < d; ++f) dot = fmaf(load_val(q + f), load_val(k + f), dot);
          dot = p.cap2 != 0.f ? cap_any(dot, p.cap_c, p.cap_most, p.to_cap, p.cap2) : dot * p.scale2;
          if (p.slopes) dot -= r.slope2 * fabsf((float)(r.pos - pos));
          const float pr = exp2_(dot - m);
          if (!is_zero(pr)) {
            open = false;
#pragma unroll
            for (int db = 0; db < NDB; ++db)
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (again[db] >> i & 1) {
                  t.o[db][i] = fmaf(pr, load_val(v + 32 * db + key_of(i, hh)), t.o[db][i]);
                  open |= !is_nan(t.o[db][i]);
                }
          }
        }
      }
    }
  }

  // way.next(st): the first stage from st on that is to be looked at; way.hides(st): whether ids may hide some of its keys
  template <typename Way> __device__ __forceinline__ void attend(int st0, int st1, const SpanRow &r, State &t, float *score_out, const Way &way) {
    clear(t);
    int st = way.next(st0, st1);
    if (st >= st1) return;
    clear_padding();
    issue(st, 0);
    Rows rows;
    load_rows(r, rows);
    const int lim_lo = uniform(wave_min(r.there ? r.lim : 0x7fffffff)), lim_hi = uniform(wave_max(r.lim));
    int buf = 0;
    while (st < st1) {
      const int then = way.next(st + 1, st1);
      __builtin_amdgcn_s_waitcnt(0x0070);  // this wave's share of the stage has landed
      __syncthreads();                     // all shares have, and the other buffer is free
      if (NBUF > 1 && then < st1) issue(then, buf ^ 1);
      compute(stage_of(st), buf, rows, r, lim_lo, lim_hi, way.hides(st), t, score_out);
      if constexpr (NBUF > 1) buf ^= 1;
      else if (then < st1) {
        __syncthreads();
        issue(then, 0);
      }
      st = then;
    }
    t.l = half_sum(t.l);
    bool odd = false;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) odd |= not_finite(t.o[db][i]);
    if (__any(odd && r.there)) careful(st0, st1, r, t, way);
  }

  // A row's result straight from its registers: normalised, or as partial result of `slot`.
  __device__ __forceinline__ void store_rows(const SpanRow &r, const State &t, int slot) const {
    if (!r.there) return;
    const int d = p.c.head_dim;
    const bool none = is_zero(t.l);
    const float inv = none ? 0.f : 1.0f / t.l;
    if (p.part_o) {
      const int64_t at = (int64_t)slot * p.n_rows * p.nq + row_pair(p, r);
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
    if (p.lse && hh == 0) p.lse[row_pair(p, r)] = none ? -INFINITY : (t.m + __builtin_amdgcn_logf(t.l)) * kLn2;
    T *out = (T *)p.out + (int64_t)r.row * p.out_rs + (int64_t)r.head * p.out_hs;
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

  // The waves that took turns at the keys of the same rows, the lanes' r, joined through LDS.  rows: how many there are.
  __device__ __forceinline__ void join_waves(const State &t, const SpanRow &info, int rows, int slot) const {
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
    for (int row = wave; row < rows; row += NW) {  // a wave a row, a lane a feature
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < KW; ++w) m = fmaxf(m, ((float *)lds)[w * PER + row]);
      float l = 0.f, a[KW];
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float *x = (float *)lds + w * PER;
        a[w] = is_none(x[row]) ? 0.f : exp2_(x[row] - m);
        if (!is_zero(a[w])) l += a[w] * x[32 + row];
      }
      const float inv = 1.0f / l;
      const int64_t r = __builtin_amdgcn_readlane(info.row, row);
      const int head = __builtin_amdgcn_readlane(info.head, row);
      const int64_t pair = r * p.nq + head, to = (int64_t)slot * p.n_rows * p.nq + pair;
      if (lane == 0) {
        if (p.part_o) {
          p.part_ml[2 * to] = is_zero(l) ? -INFINITY : not_finite(l) ? l : m;  // a maximum passes over NaN
          p.part_ml[2 * to + 1] = l;
        } else if (p.lse) {
          p.lse[pair] = is_zero(l) ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
        }
      }
      for (int f = lane; f < d; f += 64) {
        float o = 0.f;
#pragma unroll
        for (int w = 0; w < KW; ++w)
          if (!is_zero(a[w])) o += a[w] * inv * ((float *)lds)[w * PER + 64 + f * 33 + row];
        if (p.part_o) p.part_o[to * d + f] = o;
        else store_f32((T *)p.out + r * p.out_rs + head * p.out_hs + f, o);
      }
    }
  }
};

}  // namespace
}  // namespace hyp
