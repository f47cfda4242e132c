// Attention over a shared prefix and a request's own keys: what the host side and the kernels agree on.
#pragma once

#include "common.h"
#include "hyp_attn.h"

namespace hyp {

// One call, as its kernels see it.  Rows of a KV head are (row of q, head of the group) pairs, the head running fastest, so that
// a tile of 32 or 128 of them is dense whatever the group's size is.
struct SpanCall {
  hyp_attn_cache_t c;
  int page_shift;             // log2(page_keys)
  int G, nq;
  int g_shift;                // log2(G), -1: G is no power of two
  float scale2;               // scale * log2(e): scores are held as exponents of two
  float to_cap, cap2;         // scale / cap, cap * log2(e); cap2 0: not capped
  float cap_c[4], cap_most;   // polynomial of the capped score, and the largest raw score it is for
  const float *slopes;
  const void *q;
  int64_t q_rs, q_hs;
  int64_t n_rows;
  const int *q_start, *see_all, *q_pos, *q_doc;
  void *out;
  int64_t out_rs, out_hs;
  float *lse;
  int out_vec;                // four features of a row may be stored at once
  // attn_prompt: row tiles over all requests; attn_token: items over the prefix (tiles of all requests' rows), then own items
  int tiles, splits;          // own items: row tiles a request, splits of its keys
  int pre_tiles, pre_splits, pre_wide;  // pre_wide: a wave for each 32 rows of a tile; else the waves share the keys
  int pre_items;
  // partial results: slot s of row r (all q heads) at (s * n_rows * nq + r): d normalised sums, and (maximum, sum)
  float *part_o, *part_ml;
  float *scores;              // attn_token with totals: [b][c][g][score_pitch], exponents of two
  int64_t score_pitch;
  hyp_attn_totals_t totals;
  const float *lse_in;        // attn_received
  int last;
  int pairs_of_blocks;        // a workgroup has a block of keys from the front and one from the back, or one block
  int one_stage;              // the rows that count fit one stage
  int join_items;             // workgroups of the join that merge rows; the others add totals
};

struct EvictCall {
  hyp_attn_cache_t c, to;
  int page_shift, to_page_shift, in_place;
  hyp_attn_totals_t totals;
  int keep, sink, recent;
  const int *now;
  int *kept, *list;           // list: [n_requests * n_kv_heads][2 * keep]
  int vec;                    // rows move in pieces of 16 bytes
};

// wide: 16-byte pieces of keys, values and rows are aligned and whole
template <typename T> hipError_t span_prompt(const SpanCall &p, bool wide, hipStream_t s);
template <typename T> hipError_t span_token(const SpanCall &p, bool wide, hipStream_t s);
template <typename T> hipError_t span_received(const SpanCall &p, bool wide, hipStream_t s);
template <typename T> hipError_t span_join(const SpanCall &p, hipStream_t s);
hipError_t span_evict(const EvictCall &p, hipStream_t s);

// Shape of the kernels for a head size, by its padded number of 16-feature steps (4, 6, 8, 16).
__host__ __device__ constexpr int span_steps(int d, bool wide) { return !wide ? (d <= 128 ? 8 : 16) : d <= 64 ? 4 : d <= 96 ? 6 : d <= 128 ? 8 : 16; }
__host__ __device__ constexpr int span_chunks(int nt, int es) { return (nt == 6 ? 8 : nt) * es; }                 // 16-byte pieces of an LDS row
__host__ __device__ constexpr int span_stage_keys(int nt, int es) { return es == 2 && nt <= 8 ? 64 : 32; }        // a wave's keys of a stage, waves by rows
__host__ __device__ constexpr int span_token_waves(int nt, int es) { return span_chunks(nt, es) <= 32 ? 4 : 2; }
__host__ __device__ constexpr int span_steps_waves(int nt) { return nt <= 8 ? 2 : 1; }  // waves a SIMD that the registers are shared out for
constexpr int kSpanWaves = 4;          // attn_prompt: waves of 32 rows
constexpr int kSpanTile = 32 * kSpanWaves;


// Workgroups of a launch over `items` of each of the KV heads, which go to the eight XCDs in turn (head_item).
constexpr int64_t span_head_items(int64_t heads, int64_t items) { return 8 * ((heads >> 3) * items + ((heads & 7) * items + 7) / 8); }

// attn_received: rows of a stage that fit LDS twice, keys of a block (64, or 128 where two fit the registers), waves.
struct SpanReceived { int rows, keys, waves; };
constexpr SpanReceived span_received_form(int nt, int es, bool pairs_of_blocks) {
  const int rows = span_chunks(nt, es) <= 32 ? 128 : 64;
  return {rows, pairs_of_blocks && span_chunks(nt, es) <= 16 ? 128 : 64, pairs_of_blocks ? rows / 16 : 4};
}
inline int64_t span_received_items(const SpanCall &p, int keys) {  // of a KV head
  const int64_t blocks = (p.c.most + keys - 1) / keys;
  return (p.pairs_of_blocks ? (blocks + 1) / 2 : blocks) * p.c.n_requests;
}

// attn_evict: in one launch up to so many keys, else by so many threads, and moved so many slots at a time.
constexpr int kEvictSmall = 256, kEvictThreads = 1024, kEvictRows = 32;
// In place the new lengths may be written only after all heads' workgroups have read the old ones: two launches.
inline bool span_evict_once(const EvictCall &p) { return !p.in_place && p.c.most <= kEvictSmall; }

}  // namespace hyp
