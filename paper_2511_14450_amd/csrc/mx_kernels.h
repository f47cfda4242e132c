// Caches in 8 and 4 bits: what the host side and the kernels agree on.
#pragma once

#include "common.h"
#include "hyp_mx.h"

namespace hyp {

// A cache as the kernels see it; shift: log2(page_keys) where there are pages
struct MxCache {
  hyp_mx_cache_t c;
  int shift, groups, block_shift;
};

struct MxWriteCall {
  MxCache m;
  hyp_mx_rows_t r;
  int block_shift;            // of the tiles: of the cache's blocks, or of kMxPlainBlock
  int tiles;
  int wide;                   // eight features of a row are whole 16-byte pieces, of all tensors
};

struct MxReadCall {
  MxCache m;
  hyp_mx_out_t o;
  const int *first;
  int tiles;                  // of 64 keys, of a request
  int wide;
};

struct MxSelectCall {
  MxCache m;
  hyp_mx_q_t q;
  int keep, sink, recent;
  int *blocks;
  int most_blocks;
  unsigned long long *order;  // [n_requests][n_kv_heads][most_blocks]
  int wide;                   // eight features of a row and of a bound are whole 16-byte pieces
};

struct MxTokenCall {
  MxCache m;
  hyp_mx_q_t q;
  float scale2, to_cap, cap2, cap_c[4], cap_most;  // attn_score.h
  const float *slopes;
  const int *blocks;
  int listed;
  void *out;
  int64_t out_rs, out_hs;
  float *lse;
  int G, tiles, head_tiles;   // query heads of a KV head, tiles of 16 of them of a wave, workgroups that share them
  int unit, units, parts;     // log2(keys of a unit), units of a part
  float *part_o, *part_ml;    // [part][row][d] sums, and (maximum, sum)
  int wide_q;                 // eight features of a row at once
};

template <typename T> hipError_t mx_write(const MxWriteCall &p, hipStream_t s);
template <typename T> hipError_t mx_read(const MxReadCall &p, hipStream_t s);
template <typename T> hipError_t mx_select(const MxSelectCall &p, hipStream_t s);
template <typename T, int KF, int VF> hipError_t mx_token(const MxTokenCall &p, hipStream_t s);
template <typename T> hipError_t mx_join(const MxTokenCall &p, hipStream_t s);

}  // namespace hyp
