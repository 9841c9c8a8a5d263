// The wide tree attention for head_dim 128.
#include "tree_wide.hpp"

namespace cptree {

hipError_t launch_wide128(int block, int waves, const AttnArgs& a, const TreeRows& rows, int items,
                         hipStream_t s) {
  return block == 16 ? launch_wide_g<128, 16>(waves, a, rows, items, s)
                     : launch_wide_g<128, 32>(waves, a, rows, items, s);
}

}  // namespace cptree
