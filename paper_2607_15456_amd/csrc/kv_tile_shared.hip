// Small tiles of entries that share a prompt: the prompt's pages for all queries that
// read it, and an entry's own pages behind them.

#include "kv_tile_small.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_small_prefix(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  return launch_small_type<2, kPrefix>(a, grid, stream);
}

hipError_t launch_small_own(const KvTileArgs& a, int tiles, unsigned grid, hipStream_t stream) {
  return tiles == 2 ? launch_small_type<2, kOwn>(a, grid, stream) : launch_small_type<1, kOwn>(a, grid, stream);
}

}  // namespace lla
