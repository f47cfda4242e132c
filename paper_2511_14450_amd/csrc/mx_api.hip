// C entry points of hyp_mx.h: checks of the arguments and the cut of a call into launches.
#include "attn_rule.h"
#include "mx_kernels.h"
#include "mx_rules.h"

namespace hyp {
namespace {

int log2_of(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}
bool power_of_two(int v) { return v > 0 && (v & (v - 1)) == 0; }

int64_t slabs_of(const hyp_mx_cache_t &c) { return c.page_table ? c.n_pages : c.n_requests; }

MxCache check_cache(const hyp_mx_cache_t *c) {
  need(c, HYP_EINVAL, "cache is null");
  need(c->k && c->v && c->k_scale && c->v_scale && c->lens, HYP_EINVAL, "cache: k, v, k_scale, v_scale or lens is null");
  need((c->k_format == HYP_E4M3 || c->k_format == HYP_E2M1) && (c->v_format == HYP_E4M3 || c->v_format == HYP_E2M1), HYP_EINVAL,
       "cache: a format is neither HYP_E4M3 nor HYP_E2M1");
  need(c->n_requests >= 1 && c->n_kv_heads >= 1, HYP_ESHAPE, "cache: n_requests and n_kv_heads must be positive");
  need((int64_t)c->n_requests * c->n_kv_heads < (1 << 24), HYP_ESHAPE, "cache: n_requests * n_kv_heads must be below 2^24");
  need(c->head_dim >= 1 && c->head_dim <= 256, HYP_ESHAPE, "cache: head_dim must be 1..256");
  need(c->most >= 1 && c->most < (1 << 30), HYP_ESHAPE, "cache: most must be 1..2^30 - 1");
  if (c->page_table) {
    need(power_of_two(c->page_keys) && c->page_keys >= 16, HYP_EINVAL, "cache: page_keys is not a power of two from 16 on");
    need(c->n_pages >= 1 && c->pages_per_request >= 1, HYP_ESHAPE, "cache: pages_per_request and n_pages must be positive");
    need((int64_t)c->pages_per_request * c->page_keys >= c->most, HYP_ESHAPE, "cache: pages_per_request * page_keys is below most");
  } else {
    need(c->page_keys >= 16 && c->page_keys % 16 == 0, HYP_EINVAL, "cache: the room of a request (page_keys) is not a multiple of 16");
    need(c->page_keys >= c->most, HYP_ESHAPE, "cache: the room of a request (page_keys) is below most");
  }
  need(aligned(c->k, 16) && aligned(c->v, 16) && c->k_page_stride % 16 == 0 && c->k_head_stride % 16 == 0 && c->k_key_stride % 16 == 0 &&
           c->v_page_stride % 16 == 0 && c->v_head_stride % 16 == 0 && c->v_key_stride % 16 == 0,
       HYP_EINVAL, "cache: k, v or a stride of theirs is no multiple of 16 bytes");
  need(c->k_key_stride >= 0 && c->k_key_stride < (1 << 24) && c->v_key_stride >= 0 && c->v_key_stride < (1 << 24), HYP_ESHAPE,
       "cache: key strides must be 0..2^24 - 1");
  need(aligned(c->k_scale, 4) && aligned(c->v_scale, 4) && c->k_scale_page_stride % 4 == 0 && c->k_scale_head_stride % 4 == 0 &&
           c->k_scale_group_stride % 4 == 0 && c->v_scale_page_stride % 4 == 0 && c->v_scale_head_stride % 4 == 0 && c->v_scale_group_stride % 4 == 0,
       HYP_EINVAL, "cache: k_scale, v_scale or a stride of theirs is no multiple of 4 bytes");
  need(c->k_scale_group_stride >= 0 && c->k_scale_group_stride < (1 << 28) && c->v_scale_group_stride >= 0 && c->v_scale_group_stride < (1 << 28), HYP_ESHAPE,
       "cache: group strides of scales must be 0..2^28 - 1");
  need((c->lo == nullptr) == (c->hi == nullptr), HYP_EINVAL, "cache: lo and hi go together");
  need(aligned(c->lo, 2) && aligned(c->hi, 2), HYP_EINVAL, "cache: lo or hi is not aligned to its elements");
  need(!c->lo || c->block_keys, HYP_EINVAL, "cache: bounds without block_keys");
  need(c->block_keys == 0 || (power_of_two(c->block_keys) && c->block_keys >= 16 && c->block_keys <= 4096), HYP_EINVAL,
       "cache: block_keys is neither 0 nor a power of two from 16 to 4096");
  need(c->block_keys == 0 || c->page_keys % c->block_keys == 0, HYP_ESHAPE, "cache: block_keys does not divide page_keys");
  return {*c, c->page_table ? log2_of(c->page_keys) : 0, (c->head_dim + 31) / 32, c->block_keys ? log2_of(c->block_keys) : 0};
}

int es_of(int dtype) { return dtype == HYP_BF16 ? 2 : 4; }
void check_dtype(int dtype) { need(dtype == HYP_F32 || dtype == HYP_BF16, HYP_EINVAL, "dtype is neither HYP_F32 nor HYP_BF16"); }

// eight features of a row are whole, aligned pieces of 16 bytes
bool pieces(const void *p, int es, int d, int64_t a, int64_t b, int64_t c = 0) {
  const int per = 16 / es;
  return d % 8 == 0 && aligned(p, 16) && a % per == 0 && b % per == 0 && c % per == 0;
}

void check_q(const hyp_mx_cache_t &c, const hyp_mx_q_t *q) {
  need(q && q->q, HYP_EINVAL, "q is null");
  check_dtype(q->dtype);
  need(q->n_q_heads >= 1 && q->n_q_heads % c.n_kv_heads == 0, HYP_ESHAPE, "q: n_q_heads must be a multiple of n_kv_heads");
  need(q->n_q_heads / c.n_kv_heads <= 256, HYP_ESHAPE, "q: more than 256 query heads for a KV head");
  need(aligned(q->q, es_of(q->dtype)), HYP_EINVAL, "q is not aligned to its elements");
}

int blocks_of(const hyp_mx_cache_t &c) { return (int)(((int64_t)c.most + c.block_keys - 1) / c.block_keys); }

void check_select(const hyp_mx_cache_t &c, int32_t keep) {
  need(c.lo, HYP_EINVAL, "cache: no bounds to select by");
  need(keep >= 1 && keep < (1 << 30), HYP_EINVAL, "keep must be 1..2^30 - 1");
}
size_t select_bytes(const hyp_mx_cache_t &c, int32_t keep) {
  const int blocks = blocks_of(c);
  return mx_select_once(blocks, keep) ? 0 : (size_t)c.n_requests * c.n_kv_heads * blocks * 8;
}

void check_listed(const hyp_mx_cache_t &c, int32_t listed) {
  need(listed >= 0, HYP_EINVAL, "listed is negative");
  need(listed == 0 || c.block_keys, HYP_EINVAL, "cache: blocks are listed, but it has none");
  need(listed == 0 || (int64_t)listed * (c.block_keys / 16) < (1 << 30), HYP_ESHAPE, "listed blocks hold 2^34 keys or more");
}

// The cut of a call, and its workspace: floats of partial sums, of (maximum, sum) pairs.
struct Plan {
  MxTokenPlan cut;
  int group;
  int64_t items, part_o = 0, part_ml = 0;
  size_t bytes() const { return (size_t)(part_o + part_ml) * 4; }
};
Plan plan_token(const MxCache &m, const hyp_mx_q_t &q, int32_t listed) {
  const hyp_mx_cache_t &c = m.c;
  Plan p = {};
  p.group = q.n_q_heads / c.n_kv_heads;
  p.cut = mx_token_plan((int64_t)c.n_requests * c.n_kv_heads, p.group, listed ? (int64_t)listed << m.block_shift : c.most, c.page_keys, listed ? c.block_keys : 0,
                        m.groups * ((c.k_format == HYP_E4M3 ? 32 : 16) + (c.v_format == HYP_E4M3 ? 32 : 16) + 2), m.groups, q.dtype == HYP_F32);
  p.items = (int64_t)c.n_requests * c.n_kv_heads * p.cut.head_tiles;
  check_launch(p.items * p.cut.parts, 256);
  if (p.cut.parts > 1) {
    const int64_t rows = (int64_t)c.n_requests * q.n_q_heads;
    check_launch(rows, 256);
    p.part_o = (p.cut.parts * rows * c.head_dim + 3) / 4 * 4;
    p.part_ml = 2 * p.cut.parts * rows;
  }
  return p;
}

}  // namespace
}  // namespace hyp

using namespace hyp;

extern "C" {

hyp_status_t mx_write(const hyp_mx_cache_t *cache, const hyp_mx_rows_t *rows, void *hip_stream) {
  return guarded([&] {
    MxWriteCall p = {};
    p.m = check_cache(cache);
    const hyp_mx_cache_t &c = *cache;
    need(rows, HYP_EINVAL, "rows is null");
    const hyp_mx_rows_t &r = *rows;
    check_dtype(r.dtype);
    const int es = es_of(r.dtype);
    need(r.n_rows >= 0 && r.n_rows < (1 << 30), HYP_ESHAPE, "rows: n_rows must be 0..2^30 - 1");
    need(r.q_start || r.n_rows == c.n_requests, HYP_ESHAPE, "rows: without q_start one row for each request");
    need((r.k && r.v) || r.n_rows == 0, HYP_EINVAL, "rows: k or v is null");
    need(aligned(r.k, es) && aligned(r.v, es) && aligned(r.k_out, es) && aligned(r.v_out, es), HYP_EINVAL, "rows: a tensor is not aligned to its elements");
    need((r.k_out == nullptr) == (r.v_out == nullptr), HYP_EINVAL, "rows: k_out and v_out go together");
    // requests and heads write different keys: what they share would be written by several workgroups
    const int64_t n = slabs_of(c), heads = c.n_kv_heads, groups = p.m.groups;
    need(apart(c.k_page_stride, n) && apart(c.k_head_stride, heads) && apart(c.k_key_stride, c.page_keys) && apart(c.v_page_stride, n) &&
             apart(c.v_head_stride, heads) && apart(c.v_key_stride, c.page_keys), HYP_EINVAL, "cache: k or v are shared by its requests, heads or keys");
    need(apart(c.k_scale_page_stride, n) && apart(c.k_scale_head_stride, heads) && apart(c.k_scale_group_stride, groups) && apart(c.v_scale_page_stride, n) &&
             apart(c.v_scale_head_stride, heads) && apart(c.v_scale_group_stride, groups), HYP_EINVAL, "cache: scales are shared by its requests, heads or groups");
    if (c.lo)
      need(c.lo != c.hi && apart(c.bound_page_stride, n) && apart(c.bound_head_stride, heads) && apart(c.bound_block_stride, c.page_keys / c.block_keys), HYP_EINVAL,
           "cache: bounds are shared by its requests, heads or blocks");
    if (r.k_out) {
      need(r.n_rows == 0 || (apart(r.k_out_row_stride, r.n_rows) && apart(r.k_out_head_stride, heads) && apart(r.v_out_row_stride, r.n_rows) &&
                             apart(r.v_out_head_stride, heads)), HYP_EINVAL, "rows: k_out or v_out are shared by rows or heads");
      need(r.n_rows == 0 || (r.k_out != r.v_out && r.k_out != r.v && r.v_out != r.k), HYP_EINVAL, "rows: k_out and v_out are one, or the other's rows");
      need((r.k_out != r.k || (r.k_out_row_stride == r.k_row_stride && r.k_out_head_stride == r.k_head_stride)) &&
               (r.v_out != r.v || (r.v_out_row_stride == r.v_row_stride && r.v_out_head_stride == r.v_head_stride)), HYP_EINVAL, "rows: in place with unequal strides");
    }
    if (r.n_rows == 0) return;
    p.r = r;
    const int block = c.lo ? c.block_keys : c.page_table ? std::min(c.page_keys, kMxPlainBlock) : kMxPlainBlock;  // a tile lies in one page
    p.block_shift = log2_of(block);
    const int64_t tiles = mx_write_tiles(r.n_rows, c.n_requests, block, !r.q_start);
    check_launch(tiles * heads, 512);
    p.tiles = (int)tiles;
    const int d = c.head_dim;
    p.wide = pieces(r.k, es, d, r.k_row_stride, r.k_head_stride) && pieces(r.v, es, d, r.v_row_stride, r.v_head_stride) &&
             pieces(r.k_out, es, d, r.k_out_row_stride, r.k_out_head_stride) && pieces(r.v_out, es, d, r.v_out_row_stride, r.v_out_head_stride);
    const hipStream_t s = (hipStream_t)hip_stream;
    run(r.dtype == HYP_BF16 ? mx_write<bf16_t>(p, s) : mx_write<float>(p, s));
  });
}

hyp_status_t mx_read(const hyp_mx_cache_t *cache, const int32_t *first, const hyp_mx_out_t *to, void *hip_stream) {
  return guarded([&] {
    MxReadCall p = {};
    p.m = check_cache(cache);
    const hyp_mx_cache_t &c = *cache;
    need(to, HYP_EINVAL, "to is null");
    check_dtype(to->dtype);
    const int es = es_of(to->dtype);
    need(to->keys >= 0 && to->keys < (1 << 30), HYP_ESHAPE, "to: keys must be 0..2^30 - 1");
    need((to->k && to->v) || to->keys == 0, HYP_EINVAL, "to: k or v is null");
    need(aligned(to->k, es) && aligned(to->v, es), HYP_EINVAL, "to: k or v is not aligned to its elements");
    need(to->keys == 0 || (to->k != to->v && apart(to->k_request_stride, c.n_requests) && apart(to->k_head_stride, c.n_kv_heads) && apart(to->k_key_stride, to->keys) &&
                           apart(to->v_request_stride, c.n_requests) && apart(to->v_head_stride, c.n_kv_heads) && apart(to->v_key_stride, to->keys)), HYP_EINVAL,
         "to: k or v are shared by requests, heads or keys");
    if (to->keys == 0) return;
    p.o = *to;
    p.first = first;
    p.tiles = (std::min(to->keys, c.most) + 63) / 64;
    check_launch((int64_t)p.tiles * c.n_kv_heads * c.n_requests, 256);
    p.wide = pieces(to->k, es, c.head_dim, to->k_request_stride, to->k_head_stride, to->k_key_stride) &&
             pieces(to->v, es, c.head_dim, to->v_request_stride, to->v_head_stride, to->v_key_stride);
    const hipStream_t s = (hipStream_t)hip_stream;
    run(to->dtype == HYP_BF16 ? mx_read<bf16_t>(p, s) : mx_read<float>(p, s));
  });
}

size_t mx_select_workspace_bytes(const hyp_mx_cache_t *cache, const hyp_mx_q_t *q, int32_t keep) {
  size_t bytes = 0;
  guarded([&] {
    check_cache(cache);
    check_q(*cache, q);
    check_select(*cache, keep);
    bytes = select_bytes(*cache, keep);
  });
  return bytes;
}

hyp_status_t mx_select(const hyp_mx_cache_t *cache, const hyp_mx_q_t *q, int32_t keep, int32_t sink, int32_t recent, int32_t *blocks, void *workspace,
                       size_t workspace_bytes, void *hip_stream) {
  return guarded([&] {
    MxSelectCall p = {};
    p.m = check_cache(cache);
    const hyp_mx_cache_t &c = *cache;
    check_q(c, q);
    check_select(c, keep);
    need(sink >= 0 && recent >= 0 && (int64_t)sink + recent <= keep, HYP_EINVAL, "sink and recent must not be negative, nor pass keep together");
    need(blocks, HYP_EINVAL, "blocks is null");
    const size_t bytes = select_bytes(c, keep);
    need(bytes == 0 || (workspace && aligned(workspace, 16)), HYP_EINVAL, "workspace is null or not aligned to 16 bytes");
    need(workspace_bytes >= bytes, HYP_ENOMEM, "workspace is smaller than mx_select_workspace_bytes()");
    p.q = *q;
    p.keep = keep;
    p.sink = sink;
    p.recent = recent;
    p.blocks = blocks;
    p.most_blocks = blocks_of(c);
    p.order = (unsigned long long *)workspace;
    const int64_t pairs = (int64_t)c.n_requests * c.n_kv_heads;
    if (bytes) {
      check_launch(pairs, 1024);
      check_launch(pairs * mx_score_tiles(p.most_blocks, mx_score_turns(pairs, p.most_blocks)), 256);
    } else {
      check_launch(pairs, 256);
    }
    p.wide = pieces(q->q, es_of(q->dtype), c.head_dim, q->q_row_stride, q->q_head_stride) && pieces(c.lo, 2, c.head_dim, c.bound_page_stride, c.bound_head_stride, c.bound_block_stride) && aligned(c.hi, 16);
    const hipStream_t s = (hipStream_t)hip_stream;
    run(q->dtype == HYP_BF16 ? mx_select<bf16_t>(p, s) : mx_select<float>(p, s));
  });
}

size_t mx_token_workspace_bytes(const hyp_mx_cache_t *cache, const hyp_mx_q_t *q, int32_t listed) {
  size_t bytes = 0;
  guarded([&] {
    const MxCache m = check_cache(cache);
    check_q(*cache, q);
    check_listed(*cache, listed);
    bytes = plan_token(m, *q, listed).bytes();
  });
  return bytes;
}

hyp_status_t mx_token(const hyp_mx_cache_t *cache, const hyp_attn_rule_t *rule, const hyp_mx_q_t *q, const int32_t *blocks, int32_t listed,
                      const hyp_attn_out_t *out, void *workspace, size_t workspace_bytes, void *hip_stream) {
  return guarded([&] {
    MxTokenCall p = {};
    p.m = check_cache(cache);
    const hyp_mx_cache_t &c = *cache;
    check_rule(rule);
    check_q(c, q);
    check_listed(c, listed);
    need((blocks != nullptr) == (listed > 0), HYP_EINVAL, "blocks without listed, or listed without blocks");
    const int es = es_of(q->dtype);
    need(out && out->out, HYP_EINVAL, "out is null");
    need(aligned(out->out, es), HYP_EINVAL, "out is not aligned to its elements");
    need(apart(out->out_row_stride, c.n_requests) && apart(out->out_head_stride, q->n_q_heads), HYP_EINVAL, "out: rows or heads share their results");
    const Plan w = plan_token(p.m, *q, listed);
    need(w.bytes() == 0 || (workspace && aligned(workspace, 16)), HYP_EINVAL, "workspace is null or not aligned to 16 bytes");
    need(workspace_bytes >= w.bytes(), HYP_ENOMEM, "workspace is smaller than mx_token_workspace_bytes()");
    p.q = *q;
    add_rule(p, *rule);
    p.blocks = blocks;
    p.listed = listed;
    p.out = out->out;
    p.out_rs = out->out_row_stride;
    p.out_hs = out->out_head_stride;
    p.lse = out->lse;
    p.G = w.group;
    p.tiles = w.cut.tiles;
    p.head_tiles = w.cut.head_tiles;
    p.unit = w.cut.unit;
    p.units = w.cut.units;
    p.parts = w.cut.parts;
    if (w.bytes()) {
      p.part_o = (float *)workspace;
      p.part_ml = p.part_o + w.part_o;
    }
    p.wide_q = pieces(q->q, es, c.head_dim, q->q_row_stride, q->q_head_stride);
    const hipStream_t s = (hipStream_t)hip_stream;
    const bool b = q->dtype == HYP_BF16, k8 = c.k_format == HYP_E4M3, v8 = c.v_format == HYP_E4M3;
    if (b) run(k8 ? (v8 ? mx_token<bf16_t, HYP_E4M3, HYP_E4M3>(p, s) : mx_token<bf16_t, HYP_E4M3, HYP_E2M1>(p, s))
                  : (v8 ? mx_token<bf16_t, HYP_E2M1, HYP_E4M3>(p, s) : mx_token<bf16_t, HYP_E2M1, HYP_E2M1>(p, s)));
    else run(k8 ? (v8 ? mx_token<float, HYP_E4M3, HYP_E4M3>(p, s) : mx_token<float, HYP_E4M3, HYP_E2M1>(p, s))
                : (v8 ? mx_token<float, HYP_E2M1, HYP_E4M3>(p, s) : mx_token<float, HYP_E2M1, HYP_E2M1>(p, s)));
    if (p.parts > 1) run(b ? mx_join<bf16_t>(p, s) : mx_join<float>(p, s));
  });
}

const char *mx_last_error(void) { return t_error.c_str(); }

}  // extern "C"
