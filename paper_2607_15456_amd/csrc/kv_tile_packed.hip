// Small tiles of packed tokens: the entries of few new tokens.

#include "kv_tile_small.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_small_packed(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  return launch_small_type<2, kPacked>(a, grid, stream);
}

}  // namespace lla
