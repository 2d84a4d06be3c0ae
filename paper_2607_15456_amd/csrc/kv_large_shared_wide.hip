// Large tiles over a shared prompt: the queries of many entries, heads above 128.

#include "kv_tile_large.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_large_prefix_wide(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  return launch_large_wide<kPrefix>(a, grid, stream);
}

}  // namespace lla
