// How calls of hyp_mx.h are cut into workgroups.  Plain C++, so that it can be checked on the host.
#pragma once

#include <algorithm>
#include <cstdint>

namespace hyp {

constexpr int kMxPlainBlock = 64;    // mx_write: keys of a tile where the cache has no blocks

// mx_write: tiles of the rows.  Those of request b begin at q_start[b] / block + 2 b, which leaves it one for each block that its keys can
// touch: n rows touch at most n / block + 2, rounded down, and the difference of two such quotients is no less than the quotient of the
// difference.  With a row each there is a tile each.
inline int64_t mx_write_tiles(int64_t rows, int64_t requests, int64_t block, bool one_each) { return one_each ? requests : rows / block + 2 * requests; }

// mx_select: in one launch up to so many blocks of a request, or where all are kept.
constexpr int kMxSmallBlocks = 256;
inline bool mx_select_once(int blocks, int keep) { return blocks <= kMxSmallBlocks || blocks <= keep; }
// Up to so many blocks are chosen among by 512 threads, which hold them in registers, more by 1024 (64 caches of up to 2048: 23.5 us, 25.3 with 1024;
// 16 of 7813: 35, 38 with 512).
constexpr int kMxChooseBlocks = 2048;
// Scores are formed by workgroups of 64 blocks once to four times: a row is converted once for all of them, but there have to be two workgroups
// a CU.
inline int mx_score_turns(int64_t pairs, int64_t blocks) {
  int turns = 4;
  while (turns > 1 && pairs * ((blocks + 64 * turns - 1) / (64 * turns)) < 512) turns /= 2;
  return turns;
}
inline int mx_score_tiles(int64_t blocks, int turns) { return (int)((blocks + 64 * turns - 1) / (64 * turns)); }

// mx_token: whether there is a kernel whose waves take two tiles of 16 query heads, which share the keys' conversions.
constexpr bool mx_token_two_tiles(int groups_of_features, bool f32) { return groups_of_features <= 4 && !f32; }

// mx_token: units of 32 keys, or of 16 where pages or listed blocks are so short, of a part, and parts of a request.
constexpr int kMxMostUnits = 256;    // of a part: their places lie in LDS
struct MxTokenPlan { int tiles, head_tiles, unit, units, parts; };  // tiles: of a wave; head_tiles: workgroups that share the heads; unit: log2 of its keys
// Of one part a request, as many parts as give one workgroup a CU, and as many as give two, the one that a call is estimated to take the least time
// with, by what was measured: a workgroup alone on a CU goes through 125 keys a us (f32 rows: 65) and two through 170 (85) together, as far
// as a CU's 24 KB a us last; joining parts takes 6 us.  Eight heads of 8 x 32768 keys of 128 features: e4m3 in 256 / 512 workgroups 92 / 96 us,
// e2m1 66 / 54, of 64 features 74 / 56; eight of 8 x 512 keys in one part 13, in two 18; ten heads of 24 x 2048 keys (e4m3, e2m1) in one part
// 23, in two 29.  No part has fewer than 256 keys, and more workgroups than have room at once (2 a CU) wait for others to end.
//
// Groups of more than 16 query heads go by two tiles of heads a wave where that still gives two workgroups a CU (one KV head of 8 x 131072 keys with 24
// query heads: 75 us, by one tile 92; of 8 x 2000: 21.5 and 17).  pairs: of requests and KV heads
inline MxTokenPlan mx_token_plan(int64_t pairs, int group, int64_t keys, int64_t page_keys, int64_t block_keys, int64_t key_bytes, int groups_of_features, bool f32) {
  MxTokenPlan t = {};
  const bool two_tiles = group > 16 && mx_token_two_tiles(groups_of_features, f32) && pairs * ((group + 31) / 32) * (keys / 256) >= 512;
  t.tiles = two_tiles ? 2 : 1;
  t.head_tiles = (group + 16 * t.tiles - 1) / (16 * t.tiles);
  const int64_t items = pairs * t.head_tiles;
  t.unit = page_keys % 32 == 16 || block_keys == 16 ? 4 : 5;  // page_keys: also the room of a slab; block_keys: 0 where none are listed
  const int64_t units = (keys + (1 << t.unit) - 1) >> t.unit;
  const int64_t cu = 24000 / key_bytes, alone = std::min<int64_t>(cu, two_tiles ? 45 : f32 ? 65 : 125), two = std::min<int64_t>(cu, two_tiles ? 80 : f32 ? 85 : 170);  // keys a us
  int64_t parts = 1, least = 0;
  for (int64_t places : {int64_t(0), int64_t(256), int64_t(512)}) {
    const int64_t n = std::max<int64_t>(1, std::min<int64_t>(places / items, keys / 256));
    const int64_t time = (n * items <= 256 ? keys * 1000 / (n * alone) : keys * 2000 / (n * two)) + (n > 1 ? 6000 : 0);
    if (places == 0 || time < least) {
      parts = n;
      least = time;
    }
  }
  int64_t each = (units + parts - 1) / parts;
  each = std::min<int64_t>((each + 7) / 8 * 8, kMxMostUnits);
  t.units = (int)each;
  t.parts = (int)((units + each - 1) / each);
  return t;
}

}  // namespace hyp
