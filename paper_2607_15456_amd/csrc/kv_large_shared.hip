// Large tiles over a shared prompt: the queries of many entries, heads of up to 128.

#include "kv_tile_large.h"
#include "kv_tile_launch.h"

namespace lla {

hipError_t launch_large_prefix(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  if (a.p.d > 128) return launch_large_prefix_wide(a, grid, stream);
  // results in bf16 take weights of 16 bits
  return a.out_dtype == LLA_BF16 ? launch_large_narrow<2, kPrefix>(a, grid, stream)
                                 : launch_large_narrow<3, kPrefix>(a, grid, stream);
}

}  // namespace lla
