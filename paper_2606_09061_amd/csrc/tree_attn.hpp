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
  int words, hq, hkv, mbr;
  float scale_log2;  // sm_scale * log2(e)
};

hipError_t launch_attn(int d, int block, const AttnArgs& a, const TreeRows& rows, int n_rows,
                       int items, hipStream_t s);

}  // namespace cptree
