// Launches of libcpcache's kernels.
#pragma once

#include <hip/hip_runtime.h>

#include "cache_plan.hpp"

namespace cpcache {

struct AppendArgs {
  const uint16_t* qkv;
  const uint16_t* qw;
  const uint16_t* kw;
  const int32_t* positions;  // or null: the tokens' own
  uint16_t* q;
  uint16_t* k_cache;
  uint16_t* v_cache;
  const int32_t* bt;
  double step, step8;        // theta^(-2/D) and its eighth power
  float eps;
  int hq, hkv, mbr, num_blocks;
};

struct BoundsArgs {
  const uint16_t* k_cache;
  const int32_t* bt;
  uint16_t* bounds;
  int hkv, mbr, num_blocks;
};

struct SelectArgs {
  const uint16_t* q;
  const uint16_t* bounds;
  const int32_t* bt;
  int32_t* pages;
  uint64_t* scores;
  int hq, hkv, mbr, num_blocks, block, n_pages, n_first, n_last;
  int chunk;  // pages that a workgroup scores
};

struct AttnArgs {
  const uint16_t* q;
  const uint16_t* k_cache;
  const uint16_t* v_cache;
  const int32_t* bt;
  const int32_t* pages;  // page lists, or null
  uint16_t* out;
  float* part_o;         // [partial rows][D], normalised
  float* part_lse;       // [partial rows], log2 of the weights' sum
  int hq, hkv, mbr, log2_group, n_pages, piece;
  int part0;             // the partial rows of the launch's first item of rows
  int items, log2_waves; // the launch's (tokens, kv head, piece) items, and waves of each
  int log2_tokens;       // most tokens of an item
  int n_groups;          // of the launch
  int group_items;       // its first workgroups, which are the groups'
  float scale_log2;      // sm_scale * log2(e)
};

// (page, some kv heads) items of V per page of a launch
int append_v_items(int d, int block, int hkv);
hipError_t launch_append(int d, int block, const AppendArgs& a, const AppendRows& rows, int n_rows,
                         int tokens, int v_items, hipStream_t s);
hipError_t launch_bounds(int d, int block, const BoundsArgs& a, const BoundsRows& rows, int n_rows,
                         int pages, hipStream_t s);
hipError_t launch_score(int d, const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                        hipStream_t s);
// scores and choice in one
hipError_t launch_select(int d, const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                         One one, hipStream_t s);
// most: the largest number of pages of a token
hipError_t launch_choose(const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                         int most, hipStream_t s);
// tokens over their page lists
hipError_t launch_pages(int d, int block, const AttnArgs& a, const AttnBatch& b, int n_rows,
                        int items, hipStream_t s);
// groups over their common keys, and tokens over their own
hipError_t launch_shared(int d, int block, const AttnArgs& a, const AttnBatch& b, int n_rows,
                         int items, hipStream_t s);
// the same where some group is wide
hipError_t launch_shared_wide64(int block, const AttnArgs& a, const AttnBatch& b, int items,
                                hipStream_t s);
hipError_t launch_shared_wide128(int block, const AttnArgs& a, const AttnBatch& b, int items,
                                 hipStream_t s);
// the merge of the same batch's rows that have several pieces, `most` at most, of
// n_tokens tokens
hipError_t launch_cache_merge(const cp_attn_desc& d, const AttnArgs& a, const AttnBatch& b,
                              int n_rows, int n_tokens, int most, hipStream_t s);

}  // namespace cpcache
