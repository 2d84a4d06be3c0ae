// Large tiles of packed tokens: prompts and pieces of prompts, heads of up to 128.

#include "kv_tile_large.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_large_packed(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  if (a.p.d > 128) return launch_large_packed_wide(a, grid, stream);
  return launch_large_narrow<kPacked>(a, grid, stream);
}

}  // namespace lla
