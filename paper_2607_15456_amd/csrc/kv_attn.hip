// Attention of packed tokens and of shared prompts over the paged K/V cache: how the
// work is cut, and the join of the slices.

#include <algorithm>

#include "kv_tile.h"
#include "kv_tile_launch.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr float kLn2 = 0.69314718055994531f;

// Partial rows of one result: `count` of them from `at`, `stride` floats apart.
struct Slices {
  const float* at;
  int64_t stride;
  int count;
};

// Joins the partial rows of one result in a wavefront: the maximum first, then the
// weights 2^(m_s - m), a slice a lane, then four features a lane over all slices.
template <int N>
__device__ __forceinline__ void join_row(const KvTileArgs& a, const Slices (&in)[N], int64_t row) {
  const int lane = threadIdx.x % kWave, d = a.p.d;
  float m = neg_inf();
#pragma unroll
  for (int n = 0; n < N; ++n)
    for (int s = lane; s < in[n].count; s += kWave) m = fmaxf(m, in[n].at[s * in[n].stride + d]);
#pragma unroll
  for (int x = kWave / 2; x; x >>= 1) m = fmaxf(m, xor_shfl(m, x));
  const float base = m == neg_inf() ? 0.f : m;
  float l = 0.f;
  f32x4 o = f32x4{0.f};
  const int f = 4 * min(lane, d / 4 - 1);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    for (int s0 = 0; s0 < in[n].count; s0 += kWave) {
      const int many = min(kWave, in[n].count - s0);
      const float* part = in[n].at + s0 * in[n].stride;
      float w = 0.f;
      if (lane < many) {
        w = __builtin_amdgcn_exp2f(part[lane * in[n].stride + d] - base);
        l += part[lane * in[n].stride + d + 1] * w;
      }
#pragma unroll 4
      for (int s = 0; s < many; ++s) o += *reinterpret_cast<const f32x4*>(part + s * in[n].stride + f) * __shfl(w, s, kWave);
    }
  }
#pragma unroll
  for (int x = kWave / 2; x; x >>= 1) l += xor_shfl(l, x);
  if (4 * lane < d) store_row4(a, row, f, o / l);
  if (a.lse && lane == 0) a.lse[row] = (base + __builtin_amdgcn_logf(l)) * kLn2;
}

__device__ __forceinline__ void none_row(const KvTileArgs& a, int64_t row, bool nan) {
  const int lane = threadIdx.x % kWave;
  const float none = nan ? __builtin_nanf("") : 0.f;
  if (4 * lane < a.p.d) store_row4(a, row, 4 * lane, f32x4{none, none, none, none});
  if (a.lse && lane == 0) a.lse[row] = nan ? none : neg_inf();
}

// Slices of a tile, from row x of its first.
__device__ __forceinline__ Slices slices_of(const KvTileArgs& a, const Tile& t, int tiles, int tile, int slices,
                                            const float* part, int cols, int kvh, int x) {
  const int per = slice_pages(a, t.keys.pages, slices), row = a.p.d + 4;
  return {part + (item_of(a, tiles, 0, tile, kvh) * cols + x) * row, (int64_t)tiles * a.p.Hkv * cols * row,
          (t.keys.pages + per - 1) / per};
}

__global__ __launch_bounds__(kThreads) void join_packed_kernel(KvTileArgs a) {
  __shared__ int s_small[kMostEntries + 1], s_off[kMostEntries + 1], s_wave[kWaves];
  count_tiles<kPacked, kThreads>(a, kSmallCols, 0, a.small_rows, s_small, s_wave);
  const int small = s_small[a.B], small_slices = tile_slices(a, small, a.small_wgs);
  if (small_slices == 1) return;
  for (int b = threadIdx.x; b <= a.B; b += kThreads) s_off[b] = offset_of(a, b);
  __syncthreads();
  const int group = a.H / a.p.Hkv;
  const int64_t rows = (int64_t)a.total * a.H;
  for (int64_t i = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; i < rows; i += (int64_t)gridDim.x * kWaves) {
    const int token = (int)(i / a.H), h = (int)(i - (int64_t)token * a.H), kvh = h / group;
    if (token < s_off[0]) continue;
    Tile t;
    t.entry = last_at_most(s_off, a.B, token);
    if (token >= s_off[t.entry + 1]) continue;
    const int col = (token - s_off[t.entry]) * group + h - kvh * group, nth = col / kSmallCols;
    t.at<kPacked>(a, s_small, kSmallCols, nth);
    const Slices in[1] = {slices_of(a, t, small, s_small[t.entry] + nth, small_slices, a.small_part, kSmallCols, kvh,
                                    col - nth * kSmallCols)};
    if (t.state == kFine && in[0].count > 1) join_row(a, in, i);
  }
}

__global__ __launch_bounds__(kThreads) void join_shared_kernel(KvTileArgs a, int own_cols) {
  __shared__ int s_first[kMostEntries + 1], s_wave[kWaves];
  count_tiles<kPrefix, kThreads>(a, kSmallCols, 0, 0, s_first, s_wave);
  const int tiles = s_first[a.B], slices = tile_slices(a, tiles, a.small_wgs);
  const int group = a.H / a.p.Hkv, own_blocks = (group + own_cols - 1) / own_cols;
  const int64_t rows = (int64_t)a.B * a.H;
  for (int64_t i = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave; i < rows; i += (int64_t)gridDim.x * kWaves) {
    const int b = (int)(i / a.H), h = (int)(i - (int64_t)b * a.H), kvh = h / group, r = h - kvh * group;
    Tile own;
    own.entry = b;
    own.at<kOwn>(a, s_first, own_cols, r / own_cols);
    if (own.state != kFine) {
      none_row(a, i, own.state == kNone);
      continue;
    }
    Slices in[2] = {{nullptr, 0, 0},
                    slices_of(a, own, a.B * own_blocks, b * own_blocks + r / own_cols, a.own_slices, a.own_part, own_cols,
                              kvh, r % own_cols)};
    if (a.shared[b] > 0) {
      // the tile that b's queries are of: the last that begins at or before b
      const int each = tile_entries(group, kSmallCols), nth = each == 1 ? r / kSmallCols : 0;
      Tile t;
      const int tile = s_first[b + 1] - 1;  // the last of the entry's, or of the run's
      t.entry = last_at_most(s_first, a.B, tile);
      t.at<kPrefix>(a, s_first, kSmallCols, nth);
      if (t.state != kFine) {
        none_row(a, i, true);
        continue;
      }
      in[0] = slices_of(a, t, tiles, s_first[t.entry] + nth, slices, a.small_part, kSmallCols, kvh,
                        (b - t.entry) * group + r - nth * kSmallCols);
    }
    join_row(a, in, i);
  }
}

int cols_of(int group) { return group > 16 ? 32 : 16; }
int64_t blocks_of(int64_t rows, int cols) { return (rows + cols - 1) / cols; }
int bound_pages(const KvTileArgs& a) { return (a.n_ctx + kPage - 1) / kPage; }
// Most pages that a tile reads.
int most_pages(const KvTileArgs& a) {
  if (!a.window) return bound_pages(a);
  const int64_t budget = blocks_of(a.sink, kPage) + blocks_of((int64_t)a.window + 32, kPage) + 1;
  return (int)std::min<int64_t>(bound_pages(a), budget);
}
size_t row_bytes(const KvTileArgs& a) { return (size_t)(a.p.d + 4) * sizeof(float); }

constexpr int kLeast = 4;

}  // namespace

namespace {
// Tiles that a packed batch may have, at most: every entry may end inside one.
int64_t most_tiles(const KvTileArgs& a, int cols) { return (int64_t)a.total * (a.H / a.p.Hkv) / cols + a.B; }
int64_t split_items(const KvTileArgs& a, int64_t tiles, int wgs) {
  const int64_t each = std::min<int64_t>(a.most, blocks_of(most_pages(a), a.least));
  return each <= 1 ? 0 : std::min<int64_t>(wgs, tiles * a.p.Hkv * each);
}
}  // namespace

size_t kv_prefill_shape(KvTileArgs& a) {
  a.least = kLeast;
  a.most = most_pages(a) <= a.least ? 1 : 512;
  a.small_wgs = 2 * device_cu_count();
  a.small_rows = 0x7fffffff;
  return (size_t)split_items(a, most_tiles(a, kSmallCols), a.small_wgs) * kSmallCols * row_bytes(a);
}
size_t kv_prefill_workspace(const KvTileArgs& a) {
  KvTileArgs x = a;
  return kv_prefill_shape(x);
}

hipError_t launch_kv_prefill(const KvTileArgs& a, hipStream_t stream) {
  const int64_t tiles = most_tiles(a, kSmallCols), items = split_items(a, tiles, a.small_wgs);
  const unsigned grid = (unsigned)std::min<int64_t>(std::max(items, tiles * a.p.Hkv), 1 << 20);
  const hipError_t e = launch_small_packed(a, grid, stream);
  if (e != hipSuccess || items == 0) return e;
  const unsigned joins = (unsigned)std::min<int64_t>(blocks_of((int64_t)a.total * a.H, kWaves), 2048);
  hipLaunchKernelGGL(join_packed_kernel, dim3(joins), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

size_t kv_shared_shape(KvTileArgs& a) {
  const int group = a.H / a.p.Hkv, cols = cols_of(group), cus = device_cu_count(), pages = bound_pages(a);
  const int64_t units = (int64_t)a.B * a.p.Hkv * blocks_of(group, cols);
  a.least = kLeast;
  a.most = pages <= a.least ? 1 : 512;
  a.small_wgs = 2 * cus;
  a.own_slices = (int)std::max<int64_t>(1, std::min<int64_t>(2 * cus / units, blocks_of(pages, a.least)));
  // prefix tiles without a split: of a run for every two entries, or a run for all
  const int64_t tiles = (int64_t)a.B * blocks_of(group, kSmallCols);
  const int64_t prefix = std::max(split_items(a, tiles, a.small_wgs), tiles * a.p.Hkv);
  return ((size_t)prefix * kSmallCols + (size_t)units * a.own_slices * cols) * row_bytes(a);
}
size_t kv_shared_workspace(const KvTileArgs& a) {
  size_t most = 0;
  for (int B = 1; B <= a.B; ++B) {
    KvTileArgs x = a;
    x.B = B;
    most = std::max(most, kv_shared_shape(x));
  }
  return most;
}

hipError_t launch_kv_shared(const KvTileArgs& args, hipStream_t stream) {
  KvTileArgs a = args;
  const int group = a.H / a.p.Hkv, cols = cols_of(group);
  const int64_t tiles = (int64_t)a.B * blocks_of(group, kSmallCols);
  const int64_t prefix = std::max(split_items(a, tiles, a.small_wgs), tiles * a.p.Hkv);
  a.own_part = a.small_part + prefix * kSmallCols * (a.p.d + 4);
  const int64_t own = (int64_t)a.B * a.p.Hkv * blocks_of(group, cols) * a.own_slices;
  hipError_t e = launch_small_prefix(a, (unsigned)std::min<int64_t>(prefix, 1 << 20), stream);
  if (e != hipSuccess) return e;
  e = launch_small_own(a, cols / 16, (unsigned)std::min<int64_t>(own, 1 << 20), stream);
  if (e != hipSuccess) return e;
  const unsigned joins = (unsigned)std::min<int64_t>(blocks_of((int64_t)a.B * a.H, kWaves), 2048);
  hipLaunchKernelGGL(join_shared_kernel, dim3(joins), dim3(kThreads), 0, stream, a, cols);
  return hipGetLastError();
}

}  // namespace lla
