// Launches of libcpcache's kernels.
#pragma once

#include <hip/hip_runtime.h>

#include "cache.hpp"

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
};
// Pages that a workgroup scores.
constexpr int kScorePages = 256;

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
  int part0;             // the partial rows of the launch's first workgroup
  int n_groups;          // of the launch
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
hipError_t launch_choose(const SelectArgs& a, const SelectRows& rows, int n_rows, int items,
                         hipStream_t s);
// groups' rows over their common keys: partial rows
hipError_t launch_prefix_narrow(int d, int block, const AttnArgs& a, const PrefixRows& rows,
                                int n_rows, int items, hipStream_t s);
hipError_t launch_prefix_wide64(int block, const AttnArgs& a, const PrefixRows& rows, int items,
                                hipStream_t s);
hipError_t launch_prefix_wide128(int block, const AttnArgs& a, const PrefixRows& rows, int items,
                                 hipStream_t s);
// tokens over their own keys or their page lists
hipError_t launch_tokens(int d, int block, const AttnArgs& a, const AttnRows& rows, int n_rows,
                         const GroupRefs& groups, int items, hipStream_t s);
// the merge of the same launch's rows that are split, of n_tokens tokens
hipError_t launch_cache_merge(int d, int block, const AttnArgs& a, const AttnRows& rows, int n_rows,
                              const GroupRefs& groups, int n_tokens, hipStream_t s);

}  // namespace cpcache
