// How the attention calls of libcpcache are cut into workgroups (host side, no HIP).
#pragma once

#include <vector>

#include "cache.hpp"

namespace cpcache {

// Bounds of include/cp_cache.h: they keep launches' grids and index types in range.
constexpr int kMaxKvHeads = 1024;
constexpr int64_t kMaxTokens = 1 << 23, kMaxPairs = 1 << 27;
// Workgroups of a launch: 2^24 of 256 threads are what a grid takes.
constexpr int64_t kMaxItems = (1 << 24) - 1;
// Tokens and pages of a piece of a row: longer rows come as several.
constexpr int kPieceTokens = 512, kPiecePages = 2048;

// Keys that the four waves of a narrow attention workgroup take in turn, and those
// of a wide one's step.
constexpr int kTurn = 128, kWideTurn = 64;
// Waves of a workgroup where all take the same item (others have four).
constexpr int kAllWaves = 8;
// Most pages of a piece of a page list (its workgroup holds them in LDS).
constexpr int kListPages = 256;
// Most pieces of a group's keys (the factors of their merge are in LDS).
constexpr int kMaxGroupSplits = 128;

// A group's (token, q head) rows per kv head that a workgroup takes: the narrow
// kernel's waves share the keys, the wide one's the rows.
constexpr int kNarrowTile = 32, kWideTile = 128;
// PrefixRow::wide: a group's kernel, and how a wide one reads its keys.
constexpr int32_t kNarrow = 0, kCached = 1, kStreamed = 2;

struct TokenRow {    // a piece of a row's tokens
  int32_t tok0, n, start, req;
  int32_t group;     // AttnPlan::prefix's, or -1
  int32_t n_split;   // pieces of its key range
};

struct AttnPlan {
  std::vector<TokenRow> rows;       // in the order of their tokens
  std::vector<PrefixRow> prefix;    // of the groups that share something
  int unit_waves = 4;               // waves of a (tokens, kv head, piece) item: 1, 2, 4 or 8
  int log2_tokens = 0;              // most tokens of an item: neighbours share their keys
  int piece = 0;                    // keys, or entries of a list, of a piece of the rows' ranges
  bool parts = false;               // some row has several, and all have partial rows
  int32_t row_part0 = 0;            // the first of them; the groups' come before
  int64_t partial_rows = 0;
  size_t off_lse = 0, ws_bytes = 256;  // partial rows of D fp32, then their log sums

  // items of n tokens, per kv head and piece
  int items_of(int n) const { return ((n - 1) >> log2_tokens) + 1; }
};

// How one launch of cp_page_select scores and chooses for tokens of up to so many pages,
// by four waves each or by as many as their registers allow, if it does.
enum class One { kNo, kFour256, kFour1024, kAll1024 };

// Threads that choose from up to so many pages: they hold 4, 4 or 16 keys each, or, of
// more, read them again in each pass.
constexpr int kFewPages = 1024, kSomePages = 4096, kManyPages = 16384;
constexpr int choose_threads(int most) { return most > kFewPages && most <= kManyPages ? 1024 : 256; }

struct SelectPlan {
  std::vector<SelectRow> rows;  // pieces of the rows, in the order of their tokens
  int64_t scores = 0;           // that tokens which may have to choose keep
  int most = 0;                 // the largest number of pages of a token
  int chunk = 0;                // pages that a workgroup scores
  One one = One::kNo;

  int threads() const {  // of a workgroup that chooses, at most
    return one == One::kNo ? choose_threads(most) : one == One::kAll1024 ? 1024 : 256;
  }
};

void plan_select(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, int32_t n_pages,
                 SelectPlan& out);

// rows: valid for desc, within the limits of cp_cache.h.  Both return whether the
// partial rows fit their index type.
bool plan_pages(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows, int32_t n_pages,
                AttnPlan& out);
bool plan_prefix(const cp_attn_desc& desc, const cp_row_meta* rows, int32_t n_rows,
                 const cp_prefix_group* groups, int32_t n_groups, AttnPlan& out);

// Workgroups of a group's common keys.
inline int64_t prefix_items(const PrefixRow& p, int group, int hkv) {
  const int tile = p.wide != kNarrow ? kWideTile : kNarrowTile;
  return ((int64_t)p.n * group + tile - 1) / tile * hkv * p.n_split;
}

// The merge's threads hold this many rows (token, q head) at a time, and `share` sets
// of D / 4 of them take the pieces of one; a workgroup's rows are one token's.
constexpr int merge_slots(int d) { return 1024 / d; }
inline int64_t merge_items(const cp_attn_desc& d, int64_t n_tokens, int share) {
  const int per = merge_slots(d.head_dim) / share;
  return n_tokens * ((d.num_q_heads + per - 1) / per);
}
// For rows of up to so many pieces, of which a thread loads eight at once.
inline int merge_share(const cp_attn_desc& d, int64_t n_tokens, int most) {
  int share = 1;
  while (share < merge_slots(d.head_dim) && share * 8 < most &&
         merge_items(d, n_tokens, 2 * share) < kMaxItems / 2)
    share *= 2;
  return share;
}

}  // namespace cpcache
