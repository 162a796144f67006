// Work items of generation over a forest of cached segments: the layout that
// the host tables (gen_plan.cpp) and the kernels (gen.hip) share.
#pragma once

#include <cstdint>

namespace harts {

constexpr int GEN_PAGE = 64;  // rows of a cache page

// One work item: a tile of stacked rows of one segment against one split of its
// keys (int32 words).
enum GenItem : int {
  GI_SEG = 0,     // segment
  GI_FIRST = 1,   // place in `order` of the first row below the segment
  GI_ROW = 2,     // first stacked row of the tile (query row x query heads of a key head)
  GI_N = 3,       // stacked rows
  GI_SPLIT = 4,   // split, of
  GI_SPLITS = 5,  // splits
  GI_NEW = 6,     // the segment's own new rows (the first of its rows in `order`)
  GI_PART = 7,    // a row's first part in the segment
  GI_TILES = 8,   // 16-row tiles of a wave: 1 or 2
  GI_WAVES = 9,   // waves along the rows: 1, 2 or 4; where fewer than 4, the others share the keys
  GI_MUL = 10,    // multiplier and
  GI_SHIFT = 11,  // shift that divide by GI_SPLITS (fast_div.hpp)
  GI_WORDS = 12
};

// How long segments are split.  The chip holds GEN_SLOTS workgroups at once
// (three on each of 256 CUs).  While a fair share of a call's keys per slot is
// below GEN_ROUND, a split is that share, lengthened by up to 2 until all
// workgroups run in one round (a second one, of few, would double the time:
// 1,000 new rows of 1,000, 4 key heads 47 us in 1,024 workgroups, 35 in 672), but
// no shorter than GEN_MIN_SPLIT keys nor, up to GEN_ALONE keys, so short that a
// segment has more than GEN_FEW_PARTS parts, whose join would cost more than
// the shorter splits save (one row of 3,000 keys, 16 heads: 13.5 us in 24
// parts, 11.4 in 12).  Past that, splits are such shares where the workgroups
// then fit one round (256 rows of 65k keys, 8 heads: 113 us, 125 in one and a
// half), else shares of one and a half rounds, which balances items of unequal
// weight (with 64 tails of 2,000 keys: 165 us at one round, 148 so).  A call whose rows each see one segment of at most
// GEN_ALONE keys is not split at all and needs no join (333 keys, 16 heads: 9.1 us
// in one launch, 9.6 in two, and the second launch is the host's time too).
constexpr int64_t GEN_SLOTS = 768;
constexpr int64_t GEN_ROUND = 1024;
constexpr int64_t GEN_MIN_SPLIT = 128;
constexpr int64_t GEN_FEW_PARTS = 16;
constexpr int64_t GEN_ALONE = 512;
constexpr int64_t GEN_MAX_SPLITS = 4096;

}  // namespace harts
