// The shared-prefix attention of wide groups for head_dim 64.
#include "cache_wide.hpp"

namespace cpcache {

hipError_t launch_shared_wide64(int block, const AttnArgs& a, const AttnBatch& b, int items,
                               hipStream_t s) {
  return block == 16 ? launch_shared_wide_g<64, 16>(a, b, items, s)
                     : launch_shared_wide_g<64, 32>(a, b, items, s);
}

}  // namespace cpcache
