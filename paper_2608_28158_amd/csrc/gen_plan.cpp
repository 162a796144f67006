// Host tables of generation over a forest of cached segments (gen.hip): the
// new rows in depth-first order, in which the rows below any segment are
// contiguous (a segment's own new rows first); work items that each take a
// stack of those rows, one split of the segment's keys and, at launch, one key
// head; and where every row's partial results lie.  A row has one part per
// split of every segment on its chain, root first.
//
// Linear in segments, rows and items.
#include <algorithm>
#include <cstdint>
#include <new>
#include <numeric>
#include <string>
#include <vector>

#include "fast_div.hpp"
#include "gen.hpp"
#include "harts_rollout.h"
#include "plan.hpp"

using harts::set_error;

namespace {

using namespace harts;

struct GenPlan {
  std::vector<int64_t> row0;               // first query row of a segment
  std::vector<int32_t> order;
  std::vector<int64_t> start, below;       // a segment's rows in order: own, then its descendants'
  std::vector<int32_t> base, splits;       // first part of a row in the segment, splits
  std::vector<int64_t> part_off;           // [n_rows + 1]
  std::vector<int32_t> preorder;
  harts_gen_sizes sz{};
};

// How an item takes a stack of m rows of a segment of `cap` keys: up to 32 with
// 16 rows a wave, one or two waves along the rows, the others sharing the keys;
// past that in tiles of 128 rows whose four waves step through the keys
// together.  33 to 64 rows of a short segment, where latency counts, have four
// waves along the rows (31 samples of 2 rows after a 282-row prompt: 14.2 us in
// half-empty tiles, 11.8 so), but those of a long one do not, as each wave reads
// all keys (64 rows of 65k keys, 8 heads: 115 us against 80).
struct Shape { int32_t tiles, waves; };
Shape shape_of(int64_t m, int64_t cap) {
  if (m <= 16) return {1, 1};
  if (m <= 32) return {1, 2};
  if (m <= 64 && cap <= GEN_ALONE) return {1, 4};
  return {2, 4};
}

int64_t ceil_div(int64_t a, int64_t b) { return a / b + (a % b != 0); }   // (a up to 2^63 - 1)

int make(const char* where, int32_t n_seg, const int32_t* parent, const int32_t* n_new, const int64_t* cap, int32_t Hq,
         int32_t Hkv, GenPlan& P) {
  const auto bad = [&](const std::string& what) {
    set_error(std::string(where) + ": " + what);
    return HARTS_EINVAL;
  };
  if (!parent || !n_new || !cap) return bad("NULL argument");
  if (n_seg < 1 || Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 || Hq > 65535)
    return bad("need n_seg >= 1 and 1 <= Hkv <= Hq <= 65535 with Hq a multiple of Hkv");
  const int64_t group = Hq / Hkv;
  std::vector<std::vector<int32_t>> child(n_seg);
  P.row0.assign(n_seg + 1, 0);
  for (int32_t s = 0; s < n_seg; ++s) {
    if (parent[s] < -1 || parent[s] >= n_seg || parent[s] == s)
      return bad("parent of segment " + std::to_string(s) + " is invalid");
    if (n_new[s] < 0 || cap[s] < 0) return bad("segment " + std::to_string(s) + " has a negative count");
    if (parent[s] >= 0) child[parent[s]].push_back(s);
    P.row0[s + 1] = P.row0[s] + n_new[s];
  }
  const int64_t n_rows = P.row0[n_seg];
  if (n_rows > INT32_MAX / Hq) {
    set_error(std::string(where) + ": more than 2^31 - 1 (row, head) pairs");
    return HARTS_EUNSUPPORTED;
  }
  P.start.assign(n_seg, 0);
  P.below.assign(n_seg, 0);
  P.order.reserve(n_rows);
  std::vector<int32_t> stack;
  for (int32_t r = n_seg; r-- > 0;)
    if (parent[r] < 0) stack.push_back(r);
  while (!stack.empty()) {
    const int32_t s = stack.back();
    stack.pop_back();
    P.preorder.push_back(s);
    P.start[s] = static_cast<int64_t>(P.order.size());
    for (int64_t i = 0; i < n_new[s]; ++i) P.order.push_back(static_cast<int32_t>(P.row0[s] + i));
    for (size_t c = child[s].size(); c-- > 0;) stack.push_back(child[s][c]);
  }
  if (static_cast<int64_t>(P.preorder.size()) != n_seg) return bad("the parent array has a cycle");
  for (size_t i = P.preorder.size(); i-- > 0;) {
    const int32_t s = P.preorder[i];
    P.below[s] += n_new[s];
    if (parent[s] >= 0) P.below[parent[s]] += P.below[s];
  }
  const auto tiles_of = [&](int32_t s) {
    const int64_t m = P.below[s] * group;
    const Shape f = shape_of(m, cap[s]);
    return ceil_div(m, int64_t{16} * f.tiles * f.waves);
  };
  // keys of a split (gen.hpp says why)
  const auto splits_of = [&](int32_t s, int64_t len) {
    return std::max<int64_t>(1, std::min<int64_t>(ceil_div(cap[s], len), GEN_MAX_SPLITS));
  };
  const auto workgroups = [&](int64_t len) {         // (without the very short ones)
    int64_t n = 0;
    for (int32_t s = 0; s < n_seg; ++s)
      if (P.below[s] > 0 && cap[s] >= len / 8) n += tiles_of(s) * splits_of(s, len) * Hkv;
    return n;
  };
  double total = 0;
  int64_t longest = 0;
  bool alone = true;                                // no row has keys but in a short segment of its own
  for (int32_t s = 0; s < n_seg; ++s) {
    if (P.below[s] == 0) continue;
    total += static_cast<double>(tiles_of(s)) * static_cast<double>(cap[s]) * Hkv;
    longest = std::max(longest, cap[s]);
    alone = alone && parent[s] < 0 && cap[s] <= GEN_ALONE;
  }
  const auto share = [&](int64_t n) { return static_cast<int64_t>(std::min(total / n, 1e9)); };
  int64_t L = share(GEN_SLOTS);
  if (alone) {
    L = GEN_ALONE;
  } else if (L >= GEN_ROUND) {
    int64_t i = 0;
    while (i <= 2 && workgroups(L * (16 + i) / 16) > GEN_SLOTS) ++i;
    L = i <= 2 ? L * (16 + i) / 16 : std::max(GEN_ROUND, share(GEN_SLOTS * 3 / 2));
  } else {
    L = std::max({L, GEN_MIN_SPLIT, std::min(GEN_ALONE, longest / GEN_FEW_PARTS)});
    const int64_t least = L;
    for (int64_t i = 0; i <= 8; ++i)
      if (workgroups(least * (8 + i) / 8) <= GEN_SLOTS) {
        L = least * (8 + i) / 8;
        break;
      }
  }
  P.base.assign(n_seg, 0);
  P.splits.assign(n_seg, 0);
  int64_t n_items = 0;
  for (const int32_t s : P.preorder) {
    if (P.below[s] == 0) continue;
    P.splits[s] = static_cast<int32_t>(splits_of(s, L));
    if (parent[s] >= 0) P.base[s] = P.base[parent[s]] + P.splits[parent[s]];
    n_items += tiles_of(s) * P.splits[s];
    if (P.base[s] > INT32_MAX / 2) return bad("more than 2^30 parts of a row");
  }
  P.part_off.assign(n_rows + 1, 0);
  int64_t n_join = 0;
  for (int32_t s = 0; s < n_seg; ++s)
    for (int64_t i = 0; i < n_new[s]; ++i) {
      const int64_t r = P.row0[s] + i, n = int64_t{P.base[s]} + P.splits[s];
      P.part_off[r + 1] = P.part_off[r] + n;
      n_join += n > 1;
    }
  P.sz = {n_rows, n_items, P.part_off[n_rows], n_join};
  if (n_items * Hkv > INT32_MAX || P.sz.n_parts > INT32_MAX) {
    set_error(std::string(where) + ": more than 2^31 - 1 work items or parts");
    return HARTS_EUNSUPPORTED;
  }
  return HARTS_OK;
}

}  // namespace

extern "C" int harts_gen_layout(int32_t n_seg, const int32_t* parent, const int32_t* n_new, const int64_t* cap,
                                int32_t Hq, int32_t Hkv, harts_gen_sizes* out) {
  if (!out) {
    set_error("harts_gen_layout: NULL argument");
    return HARTS_EINVAL;
  }
  try {
    GenPlan P;
    if (int rc = make("harts_gen_layout", n_seg, parent, n_new, cap, Hq, Hkv, P)) return rc;
    *out = P.sz;
  } catch (const std::bad_alloc&) {
    set_error("harts_gen_layout: out of host memory");
    return HARTS_ENOMEM;
  }
  return HARTS_OK;
}

extern "C" int harts_gen_tables(int32_t n_seg, const int32_t* parent, const int32_t* n_new, const int64_t* cap,
                                int32_t Hq, int32_t Hkv, int32_t* rows, int32_t* order, int32_t* items,
                                int32_t* part_off) {
  try {
    GenPlan P;
    if (int rc = make("harts_gen_tables", n_seg, parent, n_new, cap, Hq, Hkv, P)) return rc;
    if (!part_off || (P.sz.n_rows > 0 && (!rows || !order || !items))) {
      set_error("harts_gen_tables: NULL argument");
      return HARTS_EINVAL;
    }
    for (int32_t s = 0; s < n_seg; ++s)
      for (int32_t i = 0; i < n_new[s]; ++i) {
        const int64_t r = P.row0[s] + i;
        rows[2 * r] = s;
        rows[2 * r + 1] = i - n_new[s];
      }
    std::copy(P.order.begin(), P.order.end(), order);
    for (int64_t r = 0; r <= P.sz.n_rows; ++r) part_off[r] = static_cast<int32_t>(P.part_off[r]);
    struct Item { int32_t seg, split; int64_t row, n, work; };
    std::vector<Item> list;
    list.reserve(P.sz.n_items);
    const int64_t group = Hq / Hkv;
    for (const int32_t s : P.preorder) {
      const int64_t m = P.below[s] * group;
      if (m == 0) continue;
      const Shape f = shape_of(m, cap[s]);
      const int64_t tile = int64_t{16} * f.tiles * f.waves, keys = ceil_div(cap[s], P.splits[s]);
      for (int32_t c = 0; c < P.splits[s]; ++c)
        for (int64_t r = 0; r < m; r += tile)
          list.push_back({s, c, r, std::min(tile, m - r), keys * f.tiles * f.waves});
    }
    // longest first (fewer stragglers at the end of the launch); ties keep the order
    std::stable_sort(list.begin(), list.end(), [](const Item& a, const Item& b) { return a.work > b.work; });
    int32_t* w = items;
    for (const Item& it : list) {
      const Shape f = shape_of(P.below[it.seg] * group, cap[it.seg]);
      w[GI_SEG] = it.seg;
      w[GI_FIRST] = static_cast<int32_t>(P.start[it.seg]);
      w[GI_ROW] = static_cast<int32_t>(it.row);
      w[GI_N] = static_cast<int32_t>(it.n);
      w[GI_SPLIT] = it.split;
      w[GI_SPLITS] = P.splits[it.seg];
      w[GI_NEW] = n_new[it.seg];
      w[GI_PART] = P.base[it.seg];
      w[GI_TILES] = f.tiles;
      w[GI_WAVES] = f.waves;
      const FastDiv by(static_cast<uint32_t>(P.splits[it.seg]));
      w[GI_MUL] = static_cast<int32_t>(by.m);
      w[GI_SHIFT] = static_cast<int32_t>(by.s);
      w += GI_WORDS;
    }
  } catch (const std::bad_alloc&) {
    set_error("harts_gen_tables: out of host memory");
    return HARTS_ENOMEM;
  }
  return HARTS_OK;
}

extern "C" int harts_gen_workspace_size(const harts_gen_sizes* sizes, int32_t Hq, int32_t d, size_t* bytes) {
  if (!sizes || !bytes || Hq < 1 || Hq > 65535 || sizes->n_parts < 0 || sizes->n_parts > INT32_MAX ||
      (d != 64 && d != 128)) {
    set_error("harts_gen_workspace_size: NULL argument or bad sizes");
    return HARTS_EINVAL;
  }
  // per (part, head): d accumulators, then maximum and sum; nothing where every row has one part
  *bytes = sizes->n_join == 0 ? 0 : static_cast<size_t>(sizes->n_parts) * Hq * (d + 2) * sizeof(float);
  return HARTS_OK;
}
