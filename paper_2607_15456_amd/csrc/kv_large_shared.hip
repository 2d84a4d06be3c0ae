// Large tiles over a shared prompt: the queries of many entries, heads of up to 128.

#include "kv_tile_large.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_large_prefix(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  if (a.p.d > 128) return launch_large_prefix_wide(a, grid, stream);
  return launch_large_narrow<kPrefix>(a, grid, stream);
}

}  // namespace lla
