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
  GI_WORDS = 12
};

// A split is as long as leaves GEN_FILL workgroups, and at least GEN_MIN_SPLIT
// keys.
constexpr int64_t GEN_FILL = 768;
constexpr int64_t GEN_MIN_SPLIT = 512;
constexpr int64_t GEN_MAX_SPLITS = 4096;

}  // namespace harts
