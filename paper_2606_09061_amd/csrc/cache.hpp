// Structures of libcpcache (include/cp_cache.h).
//
// The rows of a call travel inside the kernel arguments (at most 4 KB), a batch
// of them per launch: no call uploads anything, so every one can be captured
// in a graph as it is.
#pragma once

#include <limits.h>
#include <stddef.h>
#include <stdint.h>

#include "cp_cache.h"

namespace cpcache {

// Rows of a launch, N at most; few of them travel in a block of kFewRows.  The
// places behind them begin at an item that no workgroup reaches.
template <class T, int N>
struct RowsOf {
  T r[N];
};
constexpr int kFewRows = 8;

struct AppendRow {   // 24 bytes: a piece of a row of cp_qkv_append
  int32_t tok0;      // its first token
  int32_t item0;     // the first of the launch's (page, some kv heads) items of V
  int32_t n, req, start, first;  // `first`: tokens of the launch before it
};
constexpr int kAppendRows = 144;
using AppendRows = RowsOf<AppendRow, kAppendRows>;

struct BoundsRow {   // 16 bytes: a piece of a row of cp_page_bounds
  int32_t item0;     // the launch's pages before it
  int32_t req, page0, ctx;
};
constexpr int kBoundsRows = 224;
using BoundsRows = RowsOf<BoundsRow, kBoundsRows>;

struct SelectRow {   // 32 bytes: a piece of a row of cp_page_select
  int32_t item0;     // the launch's workgroups before it
  int32_t tok0, n, start, req;
  int32_t stride;    // scores per (token, kv head); 0: every page is selected
  int64_t score0;    // its first score in the workspace
};
constexpr int kSelectRows = 112;
using SelectRows = RowsOf<SelectRow, kSelectRows>;

// A piece of a row of cp_page_attn or cp_prefix_attn.  A launch's rows follow each
// other: the next one's first token ends a row, and the place behind the last row
// holds the launch's end.  With `own` keys (or entries of a list) of its last
// token, a row has ceil(own / piece) pieces, and the partial rows of its item x,
// (piece, up to T tokens, kv head), are (item0 + x) T G and on, behind those of the
// launches before.
struct AttnRow {     // 16 bytes
  int32_t item0;     // the launch's items of rows before it
  int32_t tok0, start, req;
};

struct PrefixRow {   // 44 bytes: a group's common keys
  int32_t item0;     // the launch's workgroups of groups before it
  int32_t tok0, n, req;      // its first token, its tokens, a table row that has the keys
  int32_t keys;              // whole pages, read once for the group
  int32_t n_split, split_keys, part0;  // partial rows: [kv head][split][n G]
  int32_t wide;              // its kernel
  int32_t row0, row1;        // the launch's rows that are its
};

constexpr int kAttnRows = 150, kGroups = 24;
template <int NG, int NR>
struct AttnBatchOf {
  PrefixRow g[NG];
  AttnRow r[NR + 1];
};
using AttnBatch = AttnBatchOf<kGroups, kAttnRows>;
using FewAttnBatch = AttnBatchOf<4, kFewRows>;

}  // namespace cpcache
