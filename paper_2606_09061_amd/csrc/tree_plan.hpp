// How a batch of drafted rows is cut into workgroups (host side, no HIP).
#pragma once

#include <vector>

#include "tree.hpp"

namespace cptree {

// Rows of the products: a (node, q head) pair of one kv head's group.  The
// narrow kernel takes kNarrowRows of them a workgroup, whose waves share the
// keys, and trees of one word of mask; the wide one kWideRows, whose waves share
// the rows.
constexpr int kNarrowRows = 32, kNarrowNodes = 64;
constexpr int kWideRows = 128;
// Workgroups per piece of keys and kv head of a tree of m rows.
constexpr int tree_tiles(int m, bool wide) {
  return wide ? (m + kWideRows - 1) / kWideRows : (m + kNarrowRows - 1) / kNarrowRows;
}

// Output rows (node, q head) per workgroup of the merge: its 256 threads hold
// 1024 / d of them at a time, and several share a row with many splits (one
// request of 33,000 keys on 32/8 heads 4.3 us, without sharing 15.8; on 8/1
// heads 6.2 / 42).
constexpr int merge_rows(int d, int n_split) {
  int rows = 1024 / d;
  for (int s = 8; s < n_split && rows > 1; s *= 2) rows /= 2;
  return rows;
}

// Bounds that need no check.  Rows that are split make at most kMaxSplitItems
// workgroups: cutting brings their number to the next rounds of the GPU's 512
// slots, 2,048 more than the rows uncut, or to 8 times at most 512, and a row
// that is cut at least doubles its own.  An uncut row makes 16 per kv head at
// most.  So the partial rows, 128 a workgroup, keep to 32-bit indexes, and the
// kTreeRows rows of a launch to the 2^24 workgroups of 256 threads that it takes.
constexpr int64_t kMaxSplitItems = 4096, kMaxPartialRows = kMaxSplitItems * kWideRows;
constexpr int kMaxRowItems = 16 << 10;  // of 1,024 kv heads
static_assert((int64_t)kTreeRows * kMaxRowItems + kMaxSplitItems < 1 << 24, "a launch's grid");

struct TreePlan {
  bool wide = false;           // the kernel
  int most = 0;                // rows of the products of the largest tree
  std::vector<TreeRow> rows;   // longest pieces first
  std::vector<TreeRow> merge;  // those that are split
  int64_t partial_rows = 0;
  size_t off_lse = 0, ws_bytes = 256;  // partial rows of D fp32, then their log sums

};

// rows: valid for desc, at most kMaxNodes nodes and CP_TREE_MAX_KEYS keys each (key
// indexes stay in 32 bits, rounded up to pieces and a piece further).
void plan_tree(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, TreePlan& out);

}  // namespace cptree
