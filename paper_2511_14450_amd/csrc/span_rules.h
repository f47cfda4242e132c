// How a call of hyp_attn.h is cut into workgroups.  Plain C++, so that it can be checked on the host.
#pragma once

#include <algorithm>
#include <cstdint>

namespace hyp {

// attn_prompt: parts that the keys of a row tile are cut into.  Without a cut a tile's workgroup meets all its keys; that fills the
// chip from one workgroup a CU on.  fewest: stages of a part, below which joining costs more than it gains
// (18 tiles of 4 f32 heads over up to 16 stages: 256, 512 and 1024 workgroups take 50, 42 and 43 us).
inline int span_prompt_splits(int64_t workgroups, int64_t stages, int64_t fewest) {
  if (workgroups >= 256 || stages < 2 * fewest) return 1;
  return (int)std::max<int64_t>(1, std::min<int64_t>({512 / std::max<int64_t>(workgroups, 1), stages / fewest, 64}));
}

struct SpanTokenPlan { int pre_wide, pre_tiles, pre_splits, tiles, splits; };

// attn_token: parts of an even share of all keys for 512 workgroups.  32 requests of 100 to 608 keys behind 8192 take 37 us so; with half,
// 0.75, 1.5 and twice as many parts of the shared keys 45, 38, 40 and 43 us, with 0.75 and 1.5 times those of the own ones 44 and 37 us
// (8 requests of 9216 keys: 68 and 73 instead of 60 us).  Of up to 16 rows the waves share the shared keys (2 requests of 4 heads a group:
// 25 us, a wave for each 32 rows 28), more have a wave for each 32 (4 requests 28 either way, 8: 33 and 28).
// waves: of a workgroup; pre_stage: keys of a stage of items over the shared keys where each wave has rows of its own
inline SpanTokenPlan span_token_plan(int64_t requests, int64_t kv_heads, int64_t group, int64_t most, int64_t prefix, int waves, int pre_stage) {
  SpanTokenPlan t = {};
  const int64_t rows = requests * group;
  t.tiles = (int)((group + 31) / 32);
  t.pre_wide = rows > 16;
  const int64_t tile = t.pre_wide ? 32 * waves : 32;
  t.pre_tiles = prefix ? (int)((rows + tile - 1) / tile) : 0;
  const int64_t own_items = requests * kv_heads * t.tiles, pre_items = (int64_t)t.pre_tiles * kv_heads;
  const int64_t keys = own_items * most + pre_items * prefix;
  const int64_t part = std::max<int64_t>((keys + 511) / 512, 256);
  auto cut = [&](int64_t n, int64_t stage) { return (int)std::max<int64_t>(1, std::min<int64_t>((n + part - 1) / part, (n + stage - 1) / stage)); };
  t.splits = cut(most, 32 * waves);
  t.pre_splits = prefix ? cut(prefix, t.pre_wide ? pre_stage : 32 * waves) : 0;
  return t;
}

// attn_received: whether a workgroup has a block of keys from the front and one from the back.  Causality gives the first keys the most rows, and
// pairs of blocks even that out, of 128 keys, which fetch the rows half as often: 8 prompts of 2048 rows of 32 heads 300 instead of 370 us, one
// of 4500 of 40 heads 327 instead of 397, of 6007 430 instead of 675.  Not where all blocks meet as many rows (the last 512 of 8 prompts of 512 to
// 2048: 155 instead of 128), nor where the pairs do not fill the chip (one prompt of 3500 rows, 140 of them: 268 instead of 254; 2048, 80:
// 178, 158).  All rows of prompts of unequal length lose by it, which the host does not know (those of 512 to 2048: 274 instead of 248).
inline bool span_received_pairs(int64_t most, int64_t last, int64_t requests, int64_t kv_heads, int64_t group) {
  const int64_t counts = last ? std::min(last, most) : most, pairs = (most + 255) / 256 * requests * kv_heads;
  return 2 * counts > most && counts * group > 512 && pairs >= 160;
}

}  // namespace hyp
