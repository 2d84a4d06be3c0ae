// Large tiles of packed tokens: prompts and pieces of prompts, heads above 128.

#include "kv_tile_large.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_large_packed_wide(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  return launch_large_wide<kPacked>(a, grid, stream);
}

}  // namespace lla
