// Small tiles of entries that share a prompt: every entry's own pages behind it, and the
// prompt's pages for the few queries that read it.

#include "kv_tile_small.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_small_shared(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  return a.small_cols == 16 ? launch_small_type<1, false>(a, grid, stream) : launch_small_type<2, false>(a, grid, stream);
}

}  // namespace lla
