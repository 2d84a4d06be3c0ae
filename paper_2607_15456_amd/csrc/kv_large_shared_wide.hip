// Large tiles over a shared prompt: the queries of many entries, heads above 128.

#include "kv_tile_large.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_large_prefix_wide(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  return a.out_dtype == LLA_BF16 ? launch_large_wide<2, kPrefix>(a, grid, stream)
                                 : launch_large_wide<3, kPrefix>(a, grid, stream);
}

}  // namespace lla
