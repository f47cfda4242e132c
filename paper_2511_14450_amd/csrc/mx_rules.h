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
constexpr int kMxSmallBlocks = 256, kMxScoreBlocks = 64;  // else blocks of a workgroup that forms scores
inline bool mx_select_once(int blocks, int keep) { return blocks <= kMxSmallBlocks || blocks <= keep; }

// mx_token: runs of 16 keys (of one page, or of one listed block) of a part, and parts of a request.
constexpr int kMxMostRuns = 512;     // of a part: their places lie in LDS
struct MxTokenPlan { int runs, parts; };
inline MxTokenPlan mx_token_plan(int64_t items, int64_t runs) {
  // 512 workgroups, but no part of less than 256 keys, which is 8 runs for two waves of four
  int64_t parts = std::max<int64_t>(1, std::min<int64_t>((512 + items - 1) / items, (runs + 15) / 16));
  int64_t each = (runs + parts - 1) / parts;
  each = std::min<int64_t>((each + 7) / 8 * 8, kMxMostRuns);
  return {(int)each, (int)((runs + each - 1) / each)};
}

}  // namespace hyp
