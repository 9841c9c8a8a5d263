// Launches of the tree attention (tree_attn.hip).
#pragma once

#include <hip/hip_runtime.h>

#include "tree.hpp"

namespace cptree {

struct AttnArgs {
  const uint16_t* q;
  const uint16_t* k_cache;
  const uint16_t* v_cache;
  const int32_t* bt;
  const uint64_t* mask;
  uint16_t* out;
  float* part_o;    // [partial rows][D], normalised
  float* part_lse;  // [partial rows], log2 of the weights' sum
  int words, hq, hkv, mbr, log2_group;
  float scale_log2;  // sm_scale * log2(e)
};

// The rows of a launch; the places behind them hold an item0 that no workgroup
// reaches.
hipError_t launch_narrow(int d, int block, int most, const AttnArgs& a, const TreeRows& rows,
                         int n_rows, int items, hipStream_t s);
hipError_t launch_wide64(int block, const AttnArgs& a, const TreeRows& rows, int items,
                         hipStream_t s);
hipError_t launch_wide128(int block, const AttnArgs& a, const TreeRows& rows, int items,
                          hipStream_t s);
hipError_t launch_tree_merge(int d, const AttnArgs& a, const TreeRows& rows, int n_rows, int items,
                             hipStream_t s);

}  // namespace cptree
