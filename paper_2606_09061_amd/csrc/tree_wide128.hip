// The wide tree attention for head_dim 128.
#include "tree_wide.hpp"

namespace cptree {

hipError_t launch_wide128(int block, const AttnArgs& a, const TreeRows& rows, int items,
                          hipStream_t s) {
  return block == 16 ? launch_wide_g<128, 16>(a, rows, items, s)
                     : launch_wide_g<128, 32>(a, rows, items, s);
}

}  // namespace cptree
