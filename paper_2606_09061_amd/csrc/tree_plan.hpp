// How a batch of drafted rows is cut into workgroups (host side, no HIP).
#pragma once

#include <vector>

#include "tree.hpp"

namespace cptree {

// Rows of the products: a (node, q head) pair of one kv head's group.  Rows
// with up to kNarrowRows of them go to the narrow kernel, whose four waves
// share the keys, the others to the wide one, whose waves share the rows.
constexpr int kNarrowRows = 64;

// Rows of the products per workgroup in a narrow launch of at most `most`.
constexpr int narrow_tile(int most) { return most <= 16 ? 16 : most <= 32 ? 32 : kNarrowRows; }
// Waves of a wide launch of at most `most`, 32 rows of the products each.
constexpr int wide_waves(int most) { return most <= 128 ? 4 : 8; }

// Output rows (node, q head) per workgroup of the merge: its 256 threads hold
// 1024 / d of them at a time, and several share a row with many splits.
constexpr int merge_rows(int d, int n_split) {
  int rows = 1024 / d;
  for (int s = 8; s < n_split && rows > 1; s *= 2) rows /= 2;
  return rows;
}

struct TreeLaunch {
  std::vector<TreeRow> rows;  // longest pieces first
  int most = 0;               // rows of the products of the largest tree
};

struct TreePlan {
  TreeLaunch narrow, wide;
  std::vector<TreeRow> merge;  // the rows that are split
  int64_t partial_rows = 0;
  size_t off_lse = 0, ws_bytes = 256;  // partial rows of D fp32, then their log sums
};

// rows: valid for desc, at most kMaxNodes nodes each.
void plan_tree(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, TreePlan& out);

}  // namespace cptree
