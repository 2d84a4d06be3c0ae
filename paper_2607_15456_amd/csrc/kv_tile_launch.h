// Launches of the tile kernels (host).
#pragma once

#include "kv_internal.h"

namespace lla {

// small_cols: 16 or 32
hipError_t launch_small_packed(const KvTileArgs& a, unsigned grid, hipStream_t stream);
hipError_t launch_small_shared(const KvTileArgs& a, unsigned grid, hipStream_t stream);

constexpr int large_cols(int d) { return d <= 128 ? 256 : 128; }  // rows of a large tile (bf16)
hipError_t launch_large_packed(const KvTileArgs& a, unsigned grid, hipStream_t stream);
hipError_t launch_large_packed_wide(const KvTileArgs& a, unsigned grid, hipStream_t stream);
hipError_t launch_large_prefix(const KvTileArgs& a, unsigned grid, hipStream_t stream);
hipError_t launch_large_prefix_wide(const KvTileArgs& a, unsigned grid, hipStream_t stream);

}  // namespace lla
