// How a batch of drafted rows is cut into workgroups (host side, no HIP).
#pragma once

#include <vector>

#include "tree.hpp"

namespace cptree {

// Rows of the products: a (node, q head) pair of one kv head's group.  A batch
// whose largest tree has up to kNarrowRows of them runs on the narrow kernel,
// whose waves share the keys, any other on the wide one, whose waves share the
// rows, kWideRows a workgroup.
constexpr int kNarrowRows = 32;
constexpr int kWideRows = 128;

// Output rows (node, q head) per workgroup of the merge: its 256 threads hold
// 1024 / d of them at a time, and several share a row with many splits.
constexpr int merge_rows(int d, int n_split) {
  int rows = 1024 / d;
  for (int s = 8; s < n_split && rows > 1; s *= 2) rows /= 2;
  return rows;
}

struct TreePlan {
  int most = 0;                // rows of the products of the largest tree
  std::vector<TreeRow> rows;   // longest pieces first
  std::vector<TreeRow> merge;  // those that are split
  int64_t partial_rows = 0;
  size_t off_lse = 0, ws_bytes = 256;  // partial rows of D fp32, then their log sums

  bool wide() const { return most > kNarrowRows; }
  // workgroups per piece of keys and kv head
  int tiles(const TreeRow& t, int group) const {
    return wide() ? (t.n * group + kWideRows - 1) / kWideRows : 1;
  }
};

// rows: valid for desc, at most kMaxNodes nodes each.
void plan_tree(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, TreePlan& out);

}  // namespace cptree
