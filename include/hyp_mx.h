/*
 * hyp_mx.h - C ABI of caches of keys and values in 8 or 4 bits, and of single tokens that read them
 * whole or in selected blocks, for AMD MI355X (gfx950).  It stands beside hyp_attn.h, whose caches
 * hold 16 or 32 bits a number: what bounds a token over a long context is the bytes of the cache, and
 * here a key takes a half or a quarter of them, and a token may read the blocks of keys alone whose
 * scores can be large.  The caller owns all memory, in plain [head][key][...] order or in pages.
 *
 *   mx_write   new rows of every request are quantised into its cache
 *   mx_read    what requests hold, as rows of 16 or 32 bits (for attn_prompt over a prompt's next
 *              chunk, or to move a request)
 *   mx_select  the blocks of keys whose scores with a token's row can be the largest
 *   mx_token   attention of one row a request over all its keys, or over listed blocks of them
 *
 * Numbers.  Features 32 g .. 32 g + 31 of a key are its group g and share a power of two 2^s, kept as
 * the byte s + 127; a feature is kept as a code, which stands for the number code * 2^s:
 *   HYP_E4M3  8 bits: sign, 4 bits of exponent (bias 7), 3 of fraction; largest 448; 0x7f and 0xff: NaN
 *   HYP_E2M1  4 bits: sign, 2 bits of exponent (bias 1), 1 of fraction: 0, 0.5, 1, 1.5, 2, 3, 4, 6; of a
 *             byte the low half is the even feature
 * Scale byte 255: all of the group are NaN.  mx_write takes the least s under which no feature passes
 * the largest number, within -117..119 (HYP_E4M3) or -125..125 (HYP_E2M1), so that every number is a
 * normal float and a bf16 as it stands, and rounds feature / 2^s to the nearest number, ties to the even
 * code; what is still larger (above 1.75 * 2^127 or 1.5 * 2^127) becomes the largest.  A group with an
 * infinity or a NaN gets byte 255 and reads as NaN.  The last group is filled up with zeros: a key of
 * head_dim d takes ceil(d / 32) groups of 32 or 16 bytes.  Keys under scale bytes that mx_write does not
 * write are read as well, but what they give is not defined.
 *
 * A row is the newest key of its request (hyp_attn.h): rows are cached and counted in lens before the
 * calls that use them; of mx_write, row i of the n_b rows of request b goes to key lens[b] - n_b + i.
 * Every result has the same bits from run to run; sums are grouped by the size of the call.
 *
 * All pointers are device memory of the current device unless "host" is said, owned by the caller.  No
 * call allocates or frees device memory or waits for the stream; each may be recorded into a HIP graph.
 * No call throws, aborts or prints; every failure is a status code (hyp_stage.h) with a text from
 * mx_last_error().  Values on the device are not trusted: lengths are cut to 0..most, row ranges to the
 * rows there are, page numbers to the pool, and blocks that a request does not hold are not read, so that
 * wrong ones give wrong numbers but no access outside the tensors.  The calls keep no state; any number
 * of threads and streams may make them, each with a workspace of its own.  Calls that write a request's
 * cache and calls that read it are the caller's to order, as are two requests whose tables name the same
 * page.
 */
#ifndef HYP_MX_H
#define HYP_MX_H

#include "hyp_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { HYP_E4M3 = 0, HYP_E2M1 = 1 } hyp_mx_format_t;

/* Keys and values of n_requests requests.  Strides of codes and scales count bytes.
 * Slab (page_table null): codes of key j of request b and head c are at
 *   k + b * k_page_stride + c * k_head_stride + j * k_key_stride, the byte of its group g at
 *   k_scale + b * k_scale_page_stride + c * k_scale_head_stride + g * k_scale_group_stride + j,
 *   j < page_keys, which is the room of a request (a multiple of 16).
 * Pages: page = page_table[b * pages_per_request + j / page_keys] instead of b and j % page_keys
 *   instead of j; page_keys is a power of two, 16 at least; pages_per_request * page_keys >= most.
 * k, v, and their strides are multiples of 16; k_scale, v_scale and their strides multiples of 4; key
 * strides lie in 0..2^24 - 1, group strides in 0..2^28 - 1.
 * Bounds: lo and hi (bf16) hold the least and the largest number of each feature over the keys of a
 *   block, blocks being block_keys keys from key 0 on: those of block i at
 *   lo + page * bound_page_stride + c * bound_head_stride + (i % blocks of a page) * bound_block_stride
 *   (elements).  mx_write begins a block's bounds with the block's first key and widens them from there
 *   on, so that keys that are written again leave bounds that are too wide, never too narrow.
 *   block_keys is 0 (no blocks) or a power of two from 16 to 4096 that divides page_keys. */
typedef struct {
  uint8_t *k, *v;                    /* written by mx_write only, as are scales and bounds     */
  uint8_t *k_scale, *v_scale;
  int64_t k_page_stride, k_head_stride, k_key_stride;
  int64_t v_page_stride, v_head_stride, v_key_stride;
  int64_t k_scale_page_stride, k_scale_head_stride, k_scale_group_stride;
  int64_t v_scale_page_stride, v_scale_head_stride, v_scale_group_stride;
  const int32_t *page_table;         /* [n_requests][pages_per_request] or null                */
  int32_t pages_per_request, page_keys, n_pages;
  const int32_t *lens;               /* [n_requests] keys held                                 */
  int32_t most;                      /* no length is above it; launches are sized by it        */
  int32_t n_requests, n_kv_heads, head_dim; /* head_dim 1..256                                 */
  int32_t k_format, v_format;        /* hyp_mx_format_t                                        */
  void *lo, *hi;                     /* both or neither                                        */
  int64_t bound_page_stride, bound_head_stride, bound_block_stride;
  int32_t block_keys;
} hyp_mx_cache_t;

/* Rows to be cached, features contiguous: row i, head c at k + i * k_row_stride + c * k_head_stride. */
typedef struct {
  const void *k, *v;
  int64_t k_row_stride, k_head_stride, v_row_stride, v_head_stride;
  void *k_out, *v_out;               /* the numbers that were stored, same type; both or neither; may be k and v
                                        themselves (then with the same strides)                */
  int64_t k_out_row_stride, k_out_head_stride, v_out_row_stride, v_out_head_stride;
  int64_t n_rows;
  const int32_t *q_start;            /* [n_requests + 1]: request b has rows q_start[b] .. q_start[b + 1] - 1;
                                        null: row b is request b's, n_rows == n_requests       */
  int32_t dtype;                     /* hyp_dtype_t of rows and k_out / v_out                  */
} hyp_mx_rows_t;

/* Where mx_read puts keys: key j of request b, head c, to k + b * k_request_stride + c * k_head_stride + (j - first[b]) * k_key_stride
 * for first[b] <= j < lens[b], j - first[b] < keys. */
typedef struct {
  void *k, *v;
  int64_t k_request_stride, k_head_stride, k_key_stride, v_request_stride, v_head_stride, v_key_stride;
  int32_t keys;
  int32_t dtype;                     /* hyp_dtype_t                                            */
} hyp_mx_out_t;

/* One row a request: row b, head h at q + b * q_row_stride + h * q_head_stride, features contiguous. */
typedef struct {
  const void *q;
  int64_t q_row_stride, q_head_stride;
  int32_t n_q_heads;                 /* a multiple of n_kv_heads, at most 256 times that       */
  int32_t dtype;                     /* hyp_dtype_t of rows and outputs                        */
} hyp_mx_q_t;

/* Quantise rows into the cache, and move bounds along where the cache has them.  Rows for keys below 0
 * are left out (a request with more rows than keys; a length above `most` counts as `most`), rows and
 * slots that no request names stay as they are.
 * Errors of all calls: HYP_EINVAL (null pointer, bad enum or value, misaligned, results that share memory
 * by a stride of 0), HYP_ESHAPE (sizes that do not go together), HYP_ENOMEM (workspace too small),
 * HYP_EDEVICE. */
HYP_API hyp_status_t mx_write(const hyp_mx_cache_t *cache, const hyp_mx_rows_t *rows, void *hip_stream);

/* Numbers of the keys that requests hold, rounded to dtype (a rounding that changes nothing of what
 * mx_write stores); first: [n_requests], or null: 0.  What lies behind them in the result stays as it is. */
HYP_API hyp_status_t mx_read(const hyp_mx_cache_t *cache, const int32_t *first, const hyp_mx_out_t *to, void *hip_stream);

/* For every request and KV head the blocks that a row should read: of at most `keep` blocks the first `sink`
 * and the newest `recent` always, then those of the largest score, of equal scores the first; all where a
 * request holds no more than keep.  For query head h of the group and block i
 *   score(h, i) = sum over features f of max(q_f, 0) * hi_f + min(q_f, 0) * lo_f,
 * which no <q, k> of the block passes; a KV head's is the largest of its query heads.  Scores are formed in
 * 64 bits; one that is NaN counts as larger than any number.  Distances (slopes) are not looked at, and a
 * cap, which keeps the order, has no part in it.
 *   blocks  [n_requests][n_kv_heads][keep], ascending, -1 behind the last
 *   workspace  >= mx_select_workspace_bytes(), 16-byte aligned; may be null where that is 0
 * HYP_EINVAL also: a cache without bounds, keep < 1, sink or recent < 0, sink + recent > keep. */
HYP_API size_t mx_select_workspace_bytes(const hyp_mx_cache_t *cache, const hyp_mx_q_t *q, int32_t keep);
HYP_API hyp_status_t mx_select(const hyp_mx_cache_t *cache, const hyp_mx_q_t *q, int32_t keep, int32_t sink, int32_t recent,
                               int32_t *blocks, void *workspace, size_t workspace_bytes, void *hip_stream);

/* out and lse as attn_token gives them (hyp_attn.h: the rule, rows that see no key), of keys and values
 * that are the cache's numbers; positions count from key 0, the row's is lens[b] - 1.
 *   blocks  [n_requests][n_kv_heads][listed]: only the keys of these blocks are seen; what is no block of
 *           the request (-1) is left out, one that stands there twice counts twice.  null with listed 0: all keys.
 *   workspace  >= mx_token_workspace_bytes(), 16-byte aligned; may be null where that is 0
 * Sums and the softmax are held in 32-bit floats.  Products are exact but for the probabilities that multiply
 * values: next to bf16 rows these are taken as two bf16 (off by at most 2^-16 of themselves; their sum is not
 * rounded), next to float rows they and the rows are taken in three parts of 8 bits, which hold them whole. */
HYP_API size_t mx_token_workspace_bytes(const hyp_mx_cache_t *cache, const hyp_mx_q_t *q, int32_t listed);
HYP_API hyp_status_t mx_token(const hyp_mx_cache_t *cache, const hyp_attn_rule_t *rule, const hyp_mx_q_t *q, const int32_t *blocks, int32_t listed,
                              const hyp_attn_out_t *out, void *workspace, size_t workspace_bytes, void *hip_stream);

/* Text of the last failing call of this header on this thread; owned by the library, never null. */
HYP_API const char *mx_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* HYP_MX_H */
