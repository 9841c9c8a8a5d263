#include "cache_wide.hpp"

namespace cpcache {

hipError_t launch_prefix_wide128(int block, const AttnArgs& a, const PrefixRows& rows, int items,
                                hipStream_t s) {
  return block == 16 ? launch_prefix_wide_g<128, 16>(a, rows, items, s)
                     : launch_prefix_wide_g<128, 32>(a, rows, items, s);
}

}  // namespace cpcache
