// The wide tree attention for head_dim 64.
#include "tree_wide.hpp"

namespace cptree {

hipError_t launch_wide64(int block, const AttnArgs& a, const TreeRows& rows, int items,
                         hipStream_t s) {
  return block == 16 ? launch_wide_g<64, 16>(a, rows, items, s)
                     : launch_wide_g<64, 32>(a, rows, items, s);
}

}  // namespace cptree
