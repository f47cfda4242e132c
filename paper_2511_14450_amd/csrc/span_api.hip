// C entry points of hyp_attn.h: checks of the arguments and the cut of a call into launches.
#include "attn_rule.h"
#include "span_kernels.h"
#include "span_rules.h"

namespace hyp {
namespace {

int es_of(const hyp_attn_cache_t &c) { return c.dtype == HYP_BF16 ? 2 : 4; }

int shift_of(const hyp_attn_cache_t &c) {
  int s = 0;
  if (c.page_table)
    while ((1 << s) < c.page_keys) ++s;
  return s;
}

void check_cache(const hyp_attn_cache_t *c) {
  need(c, HYP_EINVAL, "cache is null");
  need(c->k && c->v && c->lens, HYP_EINVAL, "cache: k, v or lens is null");
  need(c->dtype == HYP_F32 || c->dtype == HYP_BF16, HYP_EINVAL, "cache: dtype is neither HYP_F32 nor HYP_BF16");
  need(c->n_requests >= 1 && c->n_kv_heads >= 1, HYP_ESHAPE, "cache: n_requests and n_kv_heads must be positive");
  need((int64_t)c->n_requests * c->n_kv_heads < (1 << 24), HYP_ESHAPE, "cache: n_requests * n_kv_heads must be below 2^24");
  need(c->head_dim >= 1 && c->head_dim <= 256, HYP_ESHAPE, "cache: head_dim must be 1..256");
  need(c->most >= 1 && c->most < (1 << 30), HYP_ESHAPE, "cache: most must be 1..2^30 - 1");
  need(c->prefix_len >= 0 && c->prefix_len < (1 << 30), HYP_ESHAPE, "cache: prefix_len must be 0..2^30 - 1");
  need(c->prefix_len == 0 || (c->prefix_k && c->prefix_v), HYP_EINVAL, "cache: prefix_len without prefix_k and prefix_v");
  need(aligned(c->k, es_of(*c)) && aligned(c->v, es_of(*c)) && aligned(c->prefix_k, es_of(*c)) && aligned(c->prefix_v, es_of(*c)), HYP_EINVAL,
       "cache: a tensor is not aligned to its elements");
  if (c->page_table) {
    need(c->page_keys >= 1 && (c->page_keys & (c->page_keys - 1)) == 0, HYP_EINVAL, "cache: page_keys is not a power of two");
    need(c->n_pages >= 1 && c->pages_per_request >= 1, HYP_ESHAPE, "cache: pages_per_request and n_pages must be positive");
    need((int64_t)c->pages_per_request * c->page_keys >= c->most, HYP_ESHAPE, "cache: pages_per_request * page_keys is below most");
  }
}

void check_rows(const hyp_attn_cache_t &c, const hyp_attn_rows_t *r, bool token) {
  need(r, HYP_EINVAL, "rows is null");
  need(r->n_q_heads >= 1 && r->n_q_heads % c.n_kv_heads == 0, HYP_ESHAPE, "rows: n_q_heads must be a multiple of n_kv_heads");
  need(r->n_q_heads / c.n_kv_heads <= 256, HYP_ESHAPE, "rows: more than 256 query heads for a KV head");
  need(r->n_rows >= 0 && r->n_rows <= ((1 << 30) - 1) / (r->n_q_heads / c.n_kv_heads), HYP_ESHAPE, "rows: n_rows times the group's heads must be 0..2^30 - 1");
  need(r->q || r->n_rows == 0, HYP_EINVAL, "rows: q is null");
  need(aligned(r->q, es_of(c)), HYP_EINVAL, "rows: q is not aligned to its elements");
  if (token) need(!r->q_start && r->n_rows == c.n_requests, HYP_ESHAPE, "rows: one row for each request, without q_start");
  else need(r->q_start, HYP_EINVAL, "rows: q_start is null");
}

void check_totals(const hyp_attn_totals_t *t) {
  need(t && t->in && t->out, HYP_EINVAL, "totals: null");
  need(t->in != t->out || (t->in_request_stride == t->out_request_stride && t->in_head_stride == t->out_head_stride), HYP_EINVAL,
       "totals: in place with unequal strides");
}
void check_apart(const hyp_attn_cache_t &c, const hyp_attn_totals_t &t) {
  need(apart(t.out_request_stride, c.n_requests) && apart(t.out_head_stride, c.n_kv_heads), HYP_EINVAL, "totals: requests or heads share those that are written");
}

// Rows of keys and queries can be fetched in aligned 16-byte pieces, and a stage's rows lie within 31 bits of its first
bool is_wide(const hyp_attn_cache_t &c, const hyp_attn_rows_t &r) {
  const int per = 16 / es_of(c);
  auto tensor = [&](const void *p, int64_t a, int64_t b, int64_t key) {
    return aligned(p, 16) && a % per == 0 && b % per == 0 && key % per == 0 && key >= 0 && key < (1 << 20);
  };
  return c.head_dim % per == 0 && tensor(c.k, c.k_page_stride, c.k_head_stride, c.k_key_stride) &&
         tensor(c.v, c.v_page_stride, c.v_head_stride, c.v_key_stride) &&
         (!c.prefix_len || (tensor(c.prefix_k, 0, c.prefix_k_head_stride, c.prefix_k_key_stride) &&
                            tensor(c.prefix_v, 0, c.prefix_v_head_stride, c.prefix_v_key_stride))) &&
         aligned(r.q, 16) && r.q_row_stride % per == 0 && r.q_head_stride % per == 0;
}

SpanCall begin(const hyp_attn_cache_t &c, const hyp_attn_rows_t &r) {
  SpanCall p = {};
  p.c = c;
  p.page_shift = shift_of(c);
  p.nq = r.n_q_heads;
  p.G = r.n_q_heads / c.n_kv_heads;
  p.g_shift = -1;
  for (int s = 0; s < 9; ++s)
    if (p.G == 1 << s) p.g_shift = s;
  p.q = r.q;
  p.q_rs = r.q_row_stride;
  p.q_hs = r.q_head_stride;
  p.n_rows = r.n_rows;
  p.q_start = r.q_start;
  p.see_all = r.see_all;
  p.q_pos = r.q_pos;
  p.q_doc = r.q_doc;
  if (!r.q_doc) p.c.key_doc = nullptr;  // rows without ids see every id
  return p;
}

void add_out(SpanCall &p, const hyp_attn_out_t *o) {
  need(o && (o->out || p.n_rows == 0), HYP_EINVAL, "out is null");
  const int es = es_of(p.c);
  need(aligned(o->out, es), HYP_EINVAL, "out is not aligned to its elements");
  need(p.n_rows == 0 || (apart(o->out_row_stride, p.n_rows) && apart(o->out_head_stride, p.nq)), HYP_EINVAL, "out: rows or heads share their results");
  p.out = o->out;
  p.out_rs = o->out_row_stride;
  p.out_hs = o->out_head_stride;
  p.lse = o->lse;
  p.out_vec = aligned(o->out, 4 * es) && o->out_row_stride % 4 == 0 && o->out_head_stride % 4 == 0 && p.c.head_dim % 4 == 0;
}

// The cut of a call, and its workspace: floats of partial sums, of (maximum, sum) pairs, of scores.
struct Plan {
  int64_t part_o = 0, part_ml = 0, scores = 0;
  size_t bytes() const { return (size_t)(part_o + part_ml + scores) * 4; }
};

Plan plan_prompt(SpanCall &p, bool wide) {
  const int es = es_of(p.c), nt = span_steps(p.c.head_dim, wide);
  const int64_t pairs = p.n_rows * p.G;
  const int64_t stage = span_stage_keys(nt, es);
  const int64_t tiles = pairs / kSpanTile + p.c.n_requests;
  const int64_t stages = (p.c.prefix_len + stage - 1) / stage + (p.c.most + stage - 1) / stage;
  p.tiles = (int)tiles;
  p.splits = span_prompt_splits(tiles * p.c.n_kv_heads, stages, es == 2 ? 4 : 2);
  check_launch(span_head_items(p.c.n_kv_heads, tiles * p.splits), 64 * kSpanWaves);
  Plan w;
  if (p.splits > 1) {
    check_launch((p.n_rows * p.nq + 3) / 4, 256);
    w.part_o = (p.splits * p.n_rows * p.nq * p.c.head_dim + 3) / 4 * 4;  // pairs of floats follow
    w.part_ml = (int64_t)p.splits * p.n_rows * p.nq * 2;
  }
  return w;
}

Plan plan_token(SpanCall &p, bool wide, bool totals) {
  const int es = es_of(p.c), nt = span_steps(p.c.head_dim, wide);
  const SpanTokenPlan t = span_token_plan(p.c.n_requests, p.c.n_kv_heads, p.G, p.c.most, p.c.prefix_len, span_token_waves(nt, es), span_stage_keys(nt, es));
  p.tiles = t.tiles;
  p.splits = t.splits;
  p.pre_wide = t.pre_wide;
  p.pre_tiles = t.pre_tiles;
  p.pre_splits = t.pre_splits;
  const int64_t pre = (int64_t)t.pre_tiles * t.pre_splits * p.c.n_kv_heads, own = (int64_t)p.c.n_requests * t.tiles * t.splits * p.c.n_kv_heads;
  check_launch(pre + own, 64 * span_token_waves(nt, es));
  p.pre_items = (int)pre;
  Plan w;
  const int64_t slots = t.splits + t.pre_splits;
  if (slots > 1 || totals) {
    check_launch((p.n_rows * p.nq + 3) / 4 + (totals ? (int64_t)((p.c.most + 1023) / 1024) * p.c.n_kv_heads * p.c.n_requests : 0), 256);
    w.part_o = slots * p.n_rows * p.nq * p.c.head_dim;
    w.part_ml = slots * p.n_rows * p.nq * 2;
  }
  if (totals) {
    p.score_pitch = (p.c.most + 127) / 128 * 128;
    w.scores = (int64_t)p.c.n_requests * p.nq * p.score_pitch;
  }
  w.part_o = (w.part_o + 3) / 4 * 4;
  w.part_ml = (w.part_ml + 3) / 4 * 4;
  return w;
}

void add_workspace(SpanCall &p, const Plan &w, void *workspace, size_t bytes) {
  if (w.bytes() == 0) return;
  need(workspace && aligned(workspace, 16), HYP_EINVAL, "workspace is null or not aligned to 16 bytes");
  need(bytes >= w.bytes(), HYP_ENOMEM, "workspace is smaller than attn_workspace_bytes()");
  float *f = (float *)workspace;
  p.scores = w.scores ? f : nullptr;
  p.part_o = f + w.scores;
  p.part_ml = p.part_o + w.part_o;
}

void join(SpanCall &p, hipStream_t s) {
  if (!p.part_o) return;
  p.join_items = (int)((p.n_rows * p.nq + 3) / 4);
  run(p.c.dtype == HYP_BF16 ? span_join<bf16_t>(p, s) : span_join<float>(p, s));
}

}  // namespace
}  // namespace hyp

using namespace hyp;

extern "C" {

size_t attn_workspace_bytes(const hyp_attn_cache_t *cache, const hyp_attn_rows_t *rows, const hyp_attn_totals_t *totals) {
  size_t bytes = 0;
  guarded([&] {
    check_cache(cache);
    need(rows, HYP_EINVAL, "rows is null");
    check_rows(*cache, rows, !rows->q_start);
    SpanCall p = begin(*cache, *rows);
    const bool wide = is_wide(*cache, *rows);
    if (p.n_rows) bytes = (rows->q_start ? plan_prompt(p, wide) : plan_token(p, wide, totals != nullptr)).bytes();
  });
  return bytes;
}

hyp_status_t attn_prompt(const hyp_attn_cache_t *cache, const hyp_attn_rule_t *rule, const hyp_attn_rows_t *rows, const hyp_attn_out_t *out,
                         void *workspace, size_t workspace_bytes, void *hip_stream) {
  return guarded([&] {
    check_cache(cache);
    check_rule(rule);
    check_rows(*cache, rows, false);
    SpanCall p = begin(*cache, *rows);
    add_rule(p, *rule);
    add_out(p, out);
    if (p.n_rows == 0) return;
    const bool wide = is_wide(*cache, *rows);
    add_workspace(p, plan_prompt(p, wide), workspace, workspace_bytes);
    const hipStream_t s = (hipStream_t)hip_stream;
    run(p.c.dtype == HYP_BF16 ? span_prompt<bf16_t>(p, wide, s) : span_prompt<float>(p, wide, s));
    join(p, s);
  });
}

hyp_status_t attn_token(const hyp_attn_cache_t *cache, const hyp_attn_rule_t *rule, const hyp_attn_rows_t *rows, const hyp_attn_out_t *out,
                        const hyp_attn_totals_t *totals, void *workspace, size_t workspace_bytes, void *hip_stream) {
  return guarded([&] {
    check_cache(cache);
    check_rule(rule);
    check_rows(*cache, rows, true);
    if (totals) {
      check_totals(totals);
      check_apart(*cache, *totals);
    }
    SpanCall p = begin(*cache, *rows);
    add_rule(p, *rule);
    add_out(p, out);
    if (totals) p.totals = *totals;
    const bool wide = is_wide(*cache, *rows);
    add_workspace(p, plan_token(p, wide, totals != nullptr), workspace, workspace_bytes);
    const hipStream_t s = (hipStream_t)hip_stream;
    run(p.c.dtype == HYP_BF16 ? span_token<bf16_t>(p, wide, s) : span_token<float>(p, wide, s));
    join(p, s);
  });
}

hyp_status_t attn_received(const hyp_attn_cache_t *cache, const hyp_attn_rule_t *rule, const hyp_attn_rows_t *rows, const float *lse, int32_t last,
                           const hyp_attn_totals_t *totals, void *hip_stream) {
  return guarded([&] {
    check_cache(cache);
    check_rule(rule);
    check_rows(*cache, rows, false);
    check_totals(totals);
    check_apart(*cache, *totals);
    need(lse || rows->n_rows == 0, HYP_EINVAL, "lse is null");
    need(last >= 0, HYP_EINVAL, "last is negative");
    SpanCall p = begin(*cache, *rows);
    add_rule(p, *rule);
    p.totals = *totals;
    p.lse_in = lse;
    p.last = last;
    const bool wide = is_wide(*cache, *rows);
    p.pairs_of_blocks = span_received_pairs(p.c.most, last, p.c.n_requests, p.c.n_kv_heads, p.G);
    const SpanReceived form = span_received_form(span_steps(p.c.head_dim, wide), es_of(p.c), p.pairs_of_blocks);
    check_launch(span_head_items(p.c.n_kv_heads, span_received_items(p, form.keys)), 64 * form.waves);
    const hipStream_t s = (hipStream_t)hip_stream;
    run(p.c.dtype == HYP_BF16 ? span_received<bf16_t>(p, wide, s) : span_received<float>(p, wide, s));
  });
}

size_t attn_evict_workspace_bytes(const hyp_attn_cache_t *cache, int32_t keep) {
  size_t bytes = 0;
  guarded([&] {
    check_cache(cache);
    need(keep >= 1 && keep < (1 << 30), HYP_EINVAL, "keep must be 1..2^30 - 1");
    bytes = (size_t)cache->n_requests * cache->n_kv_heads * 2 * keep * 4;
  });
  return bytes;
}

hyp_status_t attn_evict(const hyp_attn_cache_t *cache, const hyp_attn_cache_t *into, const hyp_attn_totals_t *totals, int32_t keep, int32_t sink,
                        int32_t recent, const int32_t *now, int32_t *kept, void *workspace, size_t workspace_bytes, void *hip_stream) {
  return guarded([&] {
    check_cache(cache);
    if (into) check_cache(into);
    check_totals(totals);
    need(kept, HYP_EINVAL, "kept is null");
    need(keep >= 1 && keep < (1 << 30), HYP_EINVAL, "keep must be 1..2^30 - 1");
    need(sink >= 0 && recent >= 0 && (int64_t)sink + recent <= keep, HYP_EINVAL, "sink and recent must not be negative, nor pass keep together");
    EvictCall p = {};
    p.c = *cache;
    p.to = into ? *into : *cache;
    p.in_place = into == nullptr;
    if (into) {
      need(into->n_requests == cache->n_requests && into->n_kv_heads == cache->n_kv_heads && into->head_dim == cache->head_dim &&
               into->dtype == cache->dtype, HYP_ESHAPE, "into: other requests, heads, head_dim or dtype than the cache's");
      need(into->most >= keep, HYP_ESHAPE, "into: most is below keep");
      need(into->k != cache->k && into->v != cache->v && into->lens != cache->lens && totals->in != totals->out, HYP_EINVAL,
           "into: shares memory with the cache");
    } else {
      need(totals->in == totals->out, HYP_EINVAL, "totals: in place means out == in");
    }
    need(!into || ((!into->key_pos || into->key_pos != cache->key_pos) && (!into->key_doc || into->key_doc != cache->key_doc)), HYP_EINVAL,
         "into: shares key_pos or key_doc with the cache");
    // requests and heads keep different keys: what the result shares would be written by several workgroups, in place while others read it
    const hyp_attn_cache_t &to = p.to;
    const int64_t n = to.n_requests, heads = to.n_kv_heads, slabs = to.page_table ? to.n_pages : n, keys = to.page_table ? to.page_keys : to.most;
    need(apart(to.k_page_stride, slabs) && apart(to.k_head_stride, heads) && apart(to.k_key_stride, keys) && apart(to.v_page_stride, slabs) &&
             apart(to.v_head_stride, heads) && apart(to.v_key_stride, keys), HYP_EINVAL, "k or v of the result are shared by its requests, heads or keys");
    need((!to.key_pos || (apart(to.key_pos_request_stride, n) && apart(to.key_pos_head_stride, heads))) &&
             (!to.key_doc || (apart(to.key_doc_request_stride, n) && apart(to.key_doc_head_stride, heads))), HYP_EINVAL,
         "key_pos or key_doc of the result are shared by its requests or heads");
    check_apart(*cache, *totals);
    const size_t bytes = (size_t)cache->n_requests * cache->n_kv_heads * 2 * keep * 4;
    need(workspace && aligned(workspace, 16), HYP_EINVAL, "workspace is null or not aligned to 16 bytes");
    need(workspace_bytes >= bytes, HYP_ENOMEM, "workspace is smaller than attn_evict_workspace_bytes()");
    p.page_shift = shift_of(p.c);
    p.to_page_shift = shift_of(p.to);
    p.totals = *totals;
    p.keep = keep;
    p.sink = sink;
    p.recent = recent;
    p.now = now;
    p.kept = kept;
    p.list = (int *)workspace;
    const int per = 16 / es_of(p.c);
    auto wide = [&](const hyp_attn_cache_t &c) {
      return c.head_dim % per == 0 && aligned(c.k, 16) && aligned(c.v, 16) && c.k_page_stride % per == 0 && c.k_head_stride % per == 0 &&
             c.k_key_stride % per == 0 && c.v_page_stride % per == 0 && c.v_head_stride % per == 0 && c.v_key_stride % per == 0;
    };
    p.vec = wide(p.c) && wide(p.to);
    const int64_t pairs = (int64_t)p.c.n_requests * p.c.n_kv_heads;
    if (span_evict_once(p)) {
      check_launch(pairs, kEvictSmall);
    } else {
      check_launch(pairs, kEvictThreads);
      check_launch(pairs * ((keep + kEvictRows - 1) / kEvictRows), 256);
    }
    run(span_evict(p, (hipStream_t)hip_stream));
  });
}

const char *attn_last_error(void) { return t_error.c_str(); }

}  // extern "C"
