// Large tiles of packed tokens: prompts and pieces of prompts, heads above 128.

#include "kv_tile_large.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_large_packed_wide(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  return a.out_dtype == LLA_BF16 ? launch_large_wide<1, kPacked>(a, grid, stream)
                                 : launch_large_wide<3, kPacked>(a, grid, stream);
}

}  // namespace lla
