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
// Up to so many blocks are chosen among by 512 threads, which hold them in registers, more by 1024 (64 caches of up to 2048: 22.7 us, 24.5 with 1024;
// 16 of 7813: 33, 37 with 512).
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

// Whether two workgroups have room on a CU; the kernels of float rows of more than 192 features take the registers of one.
constexpr bool mx_token_two_workgroups(int groups_of_features, bool f32) { return !(f32 && groups_of_features > 6); }

// Keys a us that go through a CU with one workgroup and with two, as far as a CU's 24 KB a us last.  Measured over 8 x 32768 keys of 8 KV heads (float
// rows and 256 features: 4), less the 5 us of the join:
//   bf16 rows     128 features, e2m1: 121, 147 (e4m3: bytes); 256 features, e2m1: 67, 70
//   float rows    e4m3: 64 features 100, 138; 128 features 51, 76; 192 features 33, 47; 256 features 28
//   two tiles     24 heads over one KV head of 8 x 131072 keys, 128 features: e4m3 58, 69; e2m1 58, 79
struct MxTokenRates { int64_t alone, two; };
inline MxTokenRates mx_token_rates(int64_t key_bytes, int groups_of_features, bool f32, bool two_tiles) {
  const int64_t cu = 24000 / key_bytes, g = groups_of_features;
  const MxTokenRates bf16 = {480 / std::max<int64_t>(g, 4), 590 / std::max<int64_t>(g, 4)};
  const MxTokenRates r = two_tiles ? MxTokenRates{58, 74} : f32 ? MxTokenRates{std::min(204 / g, bf16.alone), std::min(300 / g, bf16.two)} : bf16;
  return {std::min(cu, r.alone), std::min(cu, r.two)};
}

// Of one part a request, as many parts as give one workgroup a CU, and as many as give two, the one that a call is estimated to take the least time
// with, by these rates and the longest part; joining parts takes 6 us.  Eight heads of 8 x 32768 keys of 128 features in 256 / 512 workgroups: e4m3
// 90.7 / 95.1 us, e2m1 72.8 / 61, float rows over four heads 86 / 59, over four of 192 features 129 / 92; of 256 features and e2m1, which have no room
// for two a CU, 105 / 112.  Eight heads of 8 x 512 keys in one part 10, in two 14; ten heads of 24 x 2048 keys (e4m3, e2m1) in one part 23.6, in two 29.5.
// Parts are cut in whole multiples of eight units, and of 256 keys at least; the last one of a request has what is left.  More workgroups than have
// room at once wait for others to end.
//
// Groups of more than 16 query heads go by two tiles of heads a wave, by which keys are read and converted half as often and by half as many
// workgroups, where pairs and two tiles of their heads are eight at least and have 2048 times 256 keys together: of fewer, each has more parts, and the join
// has one workgroup for a query
// head.  24 heads over one KV head of 128 features, e4m3 / e2m1, by one tile and by two: 8 x 131072 keys 82 / 60 and 65 / 58 us, 64 x 8192
// 57 / 43 and 44 / 39, 8 x 65536 47 / 38 and 43 / 38, 8 x 16384 20 / 19 and 24 / 22, 524288 of one request 50 / 47 and 62 / 59, 131072 25 / 28 and 45 / 44.
// pairs: of requests and KV heads
inline MxTokenPlan mx_token_plan(int64_t pairs, int group, int64_t keys, int64_t page_keys, int64_t block_keys, int64_t key_bytes, int groups_of_features, bool f32) {
  MxTokenPlan t = {};
  const int64_t by_two = pairs * ((group + 31) / 32);
  const bool two_tiles = group > 16 && mx_token_two_tiles(groups_of_features, f32) && by_two >= 8 && by_two * (keys / 256) >= 2048;
  t.tiles = two_tiles ? 2 : 1;
  t.head_tiles = (group + 16 * t.tiles - 1) / (16 * t.tiles);
  const int64_t items = pairs * t.head_tiles;
  t.unit = page_keys % 32 == 16 || block_keys == 16 ? 4 : 5;  // page_keys: also the room of a slab; block_keys: 0 where none are listed
  const int64_t units = (keys + (1 << t.unit) - 1) >> t.unit;
  const MxTokenRates rate = mx_token_rates(key_bytes, groups_of_features, f32, two_tiles);
  const int64_t room = mx_token_two_workgroups(groups_of_features, f32) ? 512 : 256;
  int64_t least = 0;
  for (int64_t places : {int64_t(0), int64_t(256), int64_t(512)}) {
    if (places > room) continue;
    const int64_t n = std::max<int64_t>(1, std::min<int64_t>(places / items, keys / 256));
    const int64_t each = std::min<int64_t>(((units + n - 1) / n + 7) / 8 * 8, kMxMostUnits), parts = (units + each - 1) / each;
    const int64_t workgroups = items * parts, rounds = (workgroups + room - 1) / room, of_two = workgroups > 256 && room == 512;
    const int64_t longest = std::min(keys, each << t.unit), time = longest * 1000 * rounds * (of_two ? 2 : 1) / (of_two ? rate.two : rate.alone) + (parts > 1 ? 6000 : 0);
    if (places == 0 || time < least) {
      t.units = (int)each;
      t.parts = (int)parts;
      least = time;
    }
  }
  return t;
}

}  // namespace hyp
