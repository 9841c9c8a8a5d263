// Structures and launches of libcptree (include/cp_tree.h).
//
// The rows, forks and layer pointers of a call travel inside the kernel
// arguments (at most 4 KB), a batch of them per launch: no call uploads
// anything, so every one can be captured in a graph as it is.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "cp_tree.h"

namespace cptree {

constexpr int kMaxNodes = CP_TREE_MAX_NODES;
constexpr int kMaxWords = kMaxNodes / 64;

// Rows of a launch, N at most; few of them travel in a block of kFewRows.
template <class T, int N>
struct RowsOf {
  T r[N];
};
constexpr int kFewRows = 8;

struct NodeRow {   // 12 bytes: a row of cp_tree_layout or cp_tree_verify
  int32_t tok0, n, start;
};
constexpr int kNodeRows = 256;
using NodeRows = RowsOf<NodeRow, kNodeRows>;

struct MoveRow {   // 16 bytes: a row of cp_kv_compact
  int32_t row, n, start, req;
};
constexpr int kMoveRows = 128;
using MoveRows = RowsOf<MoveRow, kMoveRows>;

constexpr int kForks = 128;
using Forks = RowsOf<cp_fork, kForks>;

constexpr int kLayers = 64;
struct Layers {
  uint16_t* k[kLayers];
  uint16_t* v[kLayers];
};

struct TreeRow {   // 32 bytes: a row of cp_tree_attn
  int32_t tok0, n, start, req;
  int32_t item0;      // first workgroup of the row in its launch
  int32_t n_split;    // pieces of its key range
  int32_t split_keys; // keys of a piece (the last has the rest)
  int32_t part0;      // its first partial row; unused when n_split is 1
};
constexpr int kTreeRows = 112;
using TreeRows = RowsOf<TreeRow, kTreeRows>;

}  // namespace cptree
