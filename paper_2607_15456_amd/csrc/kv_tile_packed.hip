// Small tiles of packed tokens: the entries of few new tokens.

#include "kv_tile_small.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_small_packed(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  return a.small_cols == 16 ? launch_small_type<1, true>(a, grid, stream) : launch_small_type<2, true>(a, grid, stream);
}

}  // namespace lla
