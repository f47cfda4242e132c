/*
 * hyp_attn.h - C ABI of attention over caches that requests share and that stay within a
 * budget, for AMD MI355X (gfx950).  It stands beside hyp_stage.h: a stage keeps its caches in a
 * layout of its own and gives each request one that only grows; here the caller owns keys and
 * values, in plain [head][key][feature] order or in pages, and several requests may start with
 * the same keys (a system prompt), which are stored and, for single tokens, read once.
 *
 *   attn_prompt    rows of prompts, or of a prompt's next chunk, over the shared prefix and the
 *                  request's own keys
 *   attn_token     the same for one row a request; adds the weight each own key gets to a total
 *   attn_received  the weight that own keys got from a prompt's rows, added to a total
 *   attn_evict     keeps the keys with the largest totals
 *
 * Row i of the n_b rows of request b has the own index o = lens[b] - n_b + i: the rows are the
 * newest keys of their request, which are cached before the call.  For query head h, key head
 * c = h / (n_q_heads / n_kv_heads):
 *   s(i, j) = scale * <q_i, k_j>;  with cap > 0: cap * tanh(s / cap);
 *             with slopes: s - slopes[h] * |position(i) - position(j)|
 *   seen(i, j): every shared key; own key j if (j <= o or j < see_all[b]) and, with ids, if
 *             either id is negative or both are the same
 *   lse_i = log(sum over seen j of exp s(i, j));  p(i, j) = exp(s(i, j) - lse_i);  out_i = sum p v_j
 * A row that sees no key gives zeros and an lse of -infinity.  Keys and values that a row does
 * not see have no influence on it, whatever they hold (infinities and NaN too; rows that meet such
 * values, or share a tile's keys with rows that do, are summed again one key at a time: a prompt
 * whose rows all do takes 60 to 120 times as long, and a value that is hidden from a row costs it
 * as much as one that it sees).  Positions:
 * shared key j has j, own key j has prefix_len + j unless key_pos is given, row i prefix_len + o
 * unless q_pos is given; distances count in 32 bits.
 *
 * Sums and the softmax are held in 32-bit floats.  Products of bf16 tensors are exact; the
 * probabilities that multiply bf16 values are rounded to bf16 once (which moves a result by about
 * as much as rounding it to bf16 does), their sum is not.  Every result has the same bits from run
 * to run; sums are grouped by the size of the call.
 *
 * All pointers are device memory of the current device unless "host" is said, owned by the
 * caller; strides count elements, features are contiguous.  No call allocates or frees device
 * memory or waits for the stream; each may be recorded into a HIP graph.  No call throws, aborts
 * or prints; every failure is a status code (hyp_stage.h) with a text from attn_last_error().
 * Values on the device are not trusted: lengths are cut to 0..most, row ranges to the rows there
 * are, page numbers to the pool, so that wrong ones give wrong numbers but no access outside the
 * tensors.  The calls keep no state; any number of threads and streams may make them.
 */
#ifndef HYP_ATTN_H
#define HYP_ATTN_H

#include "hyp_stage.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Keys and values of n_requests requests, and those that all of them share.
 * Slab (page_table null): own key j of request b and head c is at
 *   k + b * k_page_stride + c * k_head_stride + j * k_key_stride, j < most.
 * Pages: at k + page * k_page_stride + c * k_head_stride + (j % page_keys) * k_key_stride with
 *   page = page_table[b * pages_per_request + j / page_keys]; page_keys is a power of two and
 *   pages_per_request * page_keys >= most. */
typedef struct {
  void *k, *v;                       /* read; written by attn_evict only                      */
  int64_t k_page_stride, k_head_stride, k_key_stride;
  int64_t v_page_stride, v_head_stride, v_key_stride;
  const int32_t *page_table;         /* [n_requests][pages_per_request] or null               */
  int32_t pages_per_request, page_keys, n_pages;
  int32_t *lens;                     /* [n_requests] own keys held; written by attn_evict only */
  int32_t most;                      /* no length is above it; launches are sized by it        */
  int32_t n_requests, n_kv_heads, head_dim; /* head_dim 1..256                                 */
  int32_t dtype;                     /* hyp_dtype_t of keys, values, rows and outputs          */
  const void *prefix_k, *prefix_v;   /* shared keys, [head][key][feature], or null             */
  int64_t prefix_k_head_stride, prefix_k_key_stride;
  int64_t prefix_v_head_stride, prefix_v_key_stride;
  int32_t prefix_len;
  int32_t *key_pos, *key_doc;        /* positions / ids of own keys, key stride 1, or null     */
  int64_t key_pos_request_stride, key_pos_head_stride; /* head stride 0: the same for all heads */
  int64_t key_doc_request_stride, key_doc_head_stride;
} hyp_attn_cache_t;

typedef struct {
  float scale;           /* > 0; below 2.3e38 if scores are not capped                */
  float cap;             /* 0: scores are not capped                                  */
  const float *slopes;   /* [n_q_heads] or null                                       */
} hyp_attn_rule_t;

typedef struct {
  const void *q;                     /* row i, head h at q + i * q_row_stride + h * q_head_stride */
  int64_t q_row_stride, q_head_stride;
  int64_t n_rows;
  int32_t n_q_heads;                 /* a multiple of n_kv_heads                               */
  const int32_t *q_start;            /* [n_requests + 1]: request b has rows q_start[b] .. q_start[b + 1] - 1;
                                        attn_token: null, row b is request b's                 */
  const int32_t *see_all;            /* [n_requests] or null                                   */
  const int32_t *q_pos, *q_doc;      /* [n_rows] or null; q_doc is read if the cache has key_doc (null: all -1) */
} hyp_attn_rows_t;

typedef struct {
  void *out;                         /* row i, head h at out + i * out_row_stride + h * out_head_stride */
  int64_t out_row_stride, out_head_stride;
  float *lse;                        /* [n_rows][n_q_heads] or null                            */
} hyp_attn_out_t;

/* Running totals of the weight that own keys got: key j of request b, head c at
 * in + b * in_request_stride + c * in_head_stride + j, the sum to the same place of `out`; for all
 * j < most (those a request does not hold are copied).  in == out with equal strides adds in place. */
typedef struct {
  const float *in;
  float *out;
  int64_t in_request_stride, in_head_stride, out_request_stride, out_head_stride;
} hyp_attn_totals_t;

/* Bytes of workspace that attn_prompt (q_start given) or attn_token (null) needs for these
 * arguments, 0 if none or if the arguments are refused; totals: as for attn_token, or null. */
HYP_API size_t attn_workspace_bytes(const hyp_attn_cache_t *cache, const hyp_attn_rows_t *rows,
                                    const hyp_attn_totals_t *totals);

/* out and lse of all rows.  workspace: >= attn_workspace_bytes(cache, rows, null), 16-byte aligned;
 * one call at a time may use it.
 * Errors of all calls: HYP_EINVAL (null pointer, bad enum or value, workspace misaligned, results
 * that share memory by a stride of 0),
 * HYP_ESHAPE (sizes that do not go together), HYP_ENOMEM (workspace too small), HYP_EDEVICE. */
HYP_API hyp_status_t attn_prompt(const hyp_attn_cache_t *cache, const hyp_attn_rule_t *rule, const hyp_attn_rows_t *rows,
                                 const hyp_attn_out_t *out, void *workspace, size_t workspace_bytes, void *hip_stream);

/* One row a request (q_start null, n_rows == n_requests), the newest of its keys; see_all has no
 * meaning here.  totals: where given, total[j] += sum over the heads of c of p(j), own keys only. */
HYP_API hyp_status_t attn_token(const hyp_attn_cache_t *cache, const hyp_attn_rule_t *rule, const hyp_attn_rows_t *rows,
                                const hyp_attn_out_t *out, const hyp_attn_totals_t *totals, void *workspace,
                                size_t workspace_bytes, void *hip_stream);

/* total[j] += sum over the heads of c and the last `last` rows of request b (0: all its rows) of
 * p(i, j), own keys only; lse: [n_rows][n_q_heads] as attn_prompt gives it (-infinity: a row that
 * sees nothing, which gives no weight).  Needs no workspace. */
HYP_API hyp_status_t attn_received(const hyp_attn_cache_t *cache, const hyp_attn_rule_t *rule, const hyp_attn_rows_t *rows,
                                   const float *lse, int32_t last, const hyp_attn_totals_t *totals, void *hip_stream);

/* Keep at most `keep` keys of every request and KV head.  A request that holds more keeps its keys
 * in the order (always kept first, larger total first, lower slot first), where a key is always
 * kept if its position is below prefix_len + sink or at least now[b] - recent (now null:
 * prefix_len + lens[b]); a NaN total counts as the lowest.  Kept keys of slots below `keep` stay
 * in their slots; the slots freed there take the kept keys of higher slots, both in ascending
 * order.  So the order of the keys changes: rows that come later are scored right by key_pos, and
 * causality, which goes by slots, holds because later rows' own keys lie behind.
 *   into   null: in place - totals, key_pos and key_doc move along, lens becomes min(lens, keep).
 *          Else another cache of the same types and heads with most >= keep, sharing no memory with
 *          `cache`: it gets the keys that stay, their key_pos / key_doc where it has such (a
 *          source without key_pos gives prefix_len + slot), and lens; its slots from there on are
 *          left as they are.  Its prefix is not looked at.
 *   totals in: of `cache`; out: of the result (in place: out == in, equal strides).
 *   now    [n_requests] or null
 *   kept   [n_requests][n_kv_heads][keep]: the slot each key came from, -1 behind the last one
 *   workspace  >= attn_evict_workspace_bytes(), 16-byte aligned
 * HYP_EINVAL also: keep < 1, sink or recent < 0, sink + recent > keep, a result whose requests or
 * heads share keys, values, key_pos, key_doc or totals (a stride of 0).  Pages that several
 * requests' tables name are the caller's to keep out of an eviction in place, and of `into`. */
HYP_API size_t attn_evict_workspace_bytes(const hyp_attn_cache_t *cache, int32_t keep);
HYP_API hyp_status_t attn_evict(const hyp_attn_cache_t *cache, const hyp_attn_cache_t *into, const hyp_attn_totals_t *totals,
                                int32_t keep, int32_t sink, int32_t recent, const int32_t *now, int32_t *kept,
                                void *workspace, size_t workspace_bytes, void *hip_stream);

/* Text of the last failing call of this header on this thread; owned by the library, never null. */
HYP_API const char *attn_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* HYP_ATTN_H */
