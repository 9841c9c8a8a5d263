// How a batch of drafted rows is cut into workgroups (host side, no HIP).
#pragma once

#include <vector>

#include "tree.hpp"

namespace cptree {

// Rows of the products: a (node, q head) pair of one kv head's group.  Up to
// kNarrowRows of them, one workgroup takes all of a kv head's and its four
// waves share the keys.
constexpr int kNarrowRows = 64;
// Keys that a narrow workgroup's four waves take in one turn.
constexpr int kNarrowKeys = 128;

struct TreePlan {
  std::vector<TreeRow> narrow;
  int narrow_rows = 0;             // the most rows of the products among them
  std::vector<TreeRow> merge;      // the rows that are split
  int64_t partial_rows = 0;
  size_t off_lse = 0, ws_bytes = 256;  // partial rows of D fp32, then their log sums
};

// rows: valid for desc, at most kMaxNodes nodes each.
void plan_tree(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, TreePlan& out);

// Tiles of a row of m rows of the products, in a launch of at most `most`.
constexpr int narrow_tiles(int m, int most) {
  const int tile = most <= 16 ? 16 : most <= 32 ? 32 : kNarrowRows;
  return (m + tile - 1) / tile;
}

// Output rows (node, q head) per workgroup of the merge: its 256 threads hold
// 1024 / d of them at a time, and several share a row with many splits.
constexpr int merge_rows(int d, int n_split) {
  int rows = 1024 / d;
  for (int s = 8; s < n_split && rows > 1; s *= 2) rows /= 2;
  return rows;
}

}  // namespace cptree
