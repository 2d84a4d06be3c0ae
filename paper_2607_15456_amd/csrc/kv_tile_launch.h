// Launches of the tile kernels (host).
#pragma once

#include "kv_internal.h"

namespace lla {

constexpr int kSmallCols = 32;  // rows of a small tile

hipError_t launch_small_packed(const KvTileArgs& a, unsigned grid, hipStream_t stream);
hipError_t launch_small_prefix(const KvTileArgs& a, unsigned grid, hipStream_t stream);
// tiles: of 16 query heads, 1 or 2 a workgroup
hipError_t launch_small_own(const KvTileArgs& a, int tiles, unsigned grid, hipStream_t stream);

}  // namespace lla
