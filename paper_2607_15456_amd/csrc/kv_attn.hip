// Attention of packed tokens and of shared prompts over the paged K/V cache: how the
// work is cut, and the join of the slices.

#include <algorithm>

#include "kv_tile.h"
#include "kv_tile_launch.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr int kThreads = 256;
constexpr float kLn2 = 0.69314718055994531f;

// A result from its partial rows: d / 4 neighbouring threads hold four features each, and
// all of them the maximum and the sum.  `count` partial rows from `at`, `stride` floats apart, join it.
__device__ __forceinline__ void join_slices(float& m, float& l, f32x4& o, const float* at, int64_t stride, int count, int d, int f) {
#pragma unroll 4
  for (int s = 0; s < count; ++s) {
    const float* part = at + s * stride;
    const float m2 = part[d], l2 = part[d + 1], to = fmaxf(m, m2), base = to == neg_inf() ? 0.f : to;
    const f32x4 o2 = *reinterpret_cast<const f32x4*>(part + f);
    const float x = __builtin_amdgcn_exp2f(m - base), y = __builtin_amdgcn_exp2f(m2 - base);
    m = to;
    l = l * x + l2 * y;
    o = o * x + o2 * y;
  }
}
__device__ __forceinline__ void store_joined(const KvTileArgs& a, int64_t row, int f, float m, float l, f32x4 o) {
  store_row4(a, row, f, o / l);
  if (a.lse && f == 0) a.lse[row] = ((m == neg_inf() ? 0.f : m) + __builtin_amdgcn_logf(l)) * kLn2;
}

// Partial rows of a tile's row: from slice 0's, how far apart and how many.
struct Slices {
  const float* at;
  int64_t stride;
  int count;
};
// Of row x of a tile of `cols` rows and `pages` pages, number `tile` of `tiles` that are cut into `slices`.
__device__ __forceinline__ Slices slices_of(const KvTileArgs& a, int pages, int least, const float* part, int tiles, int tile,
                                            int slices, int cols, int kvh, int x) {
  const int per = slice_pages(least, pages, slices), row = a.p.d + 4;
  return {part + ((int64_t)item_of(a, tiles, 0, tile, kvh) * cols + x) * row, (int64_t)tiles * a.p.Hkv * cols * row,
          (pages + per - 1) / per};
}

// Rows of a tile that a workgroup joins at a time: one a thread, d / 4 threads for each.
__host__ __device__ __forceinline__ int join_rows(int d) { return kThreads / (d / 4); }
__host__ __device__ __forceinline__ int join_chunks(int d, int cols) { return (cols + join_rows(d) - 1) / join_rows(d); }

// What differs between the kinds of tiles is chosen value by value, and a result's sums are
// values of their own: a choice between structures, or a structure read in part,
// is kept in memory, for which a workgroup reads its dispatch packet from the host's memory (11 us
// of the join's 22 after a piece of 512 tokens over 15,001).

// Packed tokens: the tiles that were cut, a workgroup some rows of one.
__global__ __launch_bounds__(kThreads) void join_packed_kernel(KvTileArgs a, int large_cols) {
  __shared__ int s_small[kMostEntries + 1], s_large[kMostEntries + 1];
  __shared__ int s_wave[kThreads / kWave];
  count_packed<kThreads>(a, a.small_cols, 0, a.small_rows, s_small, s_wave);
  count_packed<kThreads>(a, large_cols, a.small_rows, kAllRows, s_large, s_wave);
  const int small = tiles_of(a.small, s_small[a.B]), small_slices = tile_slices(a.small, small * a.p.Hkv);
  const int large = tiles_of(a.large, s_large[a.B]), large_slices = tile_slices(a.large, large * a.p.Hkv);
  const int of_small = small_slices > 1 ? small * a.p.Hkv * join_chunks(a.p.d, a.small_cols) : 0;
  const int of_large = large_slices > 1 ? large * a.p.Hkv * join_chunks(a.p.d, large_cols) : 0;
  const int lanes = a.p.d / 4, r = threadIdx.x / lanes, f = 4 * (threadIdx.x % lanes);
  if (r >= join_rows(a.p.d)) return;
#pragma unroll 1
  for (int i = blockIdx.x; i < of_small + of_large; i += gridDim.x) {
    const bool is_small = i < of_small;
    const int cols = is_small ? a.small_cols : large_cols, chunks = join_chunks(a.p.d, cols), j = is_small ? i : i - of_small;
    const int unit = j / chunks, tile = unit / a.p.Hkv, kvh = unit - tile * a.p.Hkv;
    const int x = (j - unit * chunks) * join_rows(a.p.d) + r;
    const int b = is_small ? last_at_most(s_small, a.B, tile) : last_at_most(s_large, a.B, tile);
    Tile t;
    t.at<kPacked>(a, b, cols, tile - (is_small ? s_small[b] : s_large[b]));
    if (t.state != kFine || x >= t.rows) continue;
    const Slices in = slices_of(a, t.keys.pages, is_small ? a.small.least : a.large.least, is_small ? a.small.part : a.large.part,
                                is_small ? small : large, tile, is_small ? small_slices : large_slices, cols, kvh, x);
    if (in.count <= 1) continue;  // (written by the tile itself)
    float m = neg_inf(), l = 0.f;
    f32x4 o = f32x4{0.f};
    join_slices(m, l, o, in.at, in.stride, in.count, a.p.d, f);
    int64_t q_at, out_at;
    t.row_keys<kPacked>(a, kvh, x, q_at, out_at);
    store_joined(a, out_at, f, m, l, o);
  }
}

// Shared prompts: every (entry, query head), of its prompt's slices and its own.
__global__ __launch_bounds__(kThreads) void join_shared_kernel(KvTileArgs a) {
  __shared__ int s_runs[kMostEntries + 1], s_small[kMostEntries + 1], s_large[kMostEntries + 1];
  __shared__ int s_wave[kThreads / kWave];
  count_shared<kThreads>(a, s_runs, s_small, s_large, s_wave);
  const int small = tiles_of(a.small, s_small[a.B]), small_slices = tile_slices(a.small, small * a.p.Hkv);
  const int large = tiles_of(a.large, s_large[a.B]), large_slices = tile_slices(a.large, large * a.p.Hkv);
  const int group = a.H / a.p.Hkv, cols = a.small_cols, blocks = (group + cols - 1) / cols;
  const int lanes = a.p.d / 4, f = 4 * (threadIdx.x % lanes), step = join_rows(a.p.d);
  const int rows = a.B * a.H;  // (below 2^31, as every number of tiles and their slices)
  if ((int)threadIdx.x / lanes >= step) return;
#pragma unroll 1
  for (int64_t at = (int64_t)blockIdx.x * step + threadIdx.x / lanes; at < rows; at += (int64_t)gridDim.x * step) {
    const int i = (int)at, b = i / a.H, h = i - b * a.H, kvh = h / group, r = h - kvh * group;
    const int own_block = r / cols;
    Tile t;
    t.at<kOwn>(a, b, cols, own_block);
    TileState state = t.state;
    const int own_pages = t.keys.pages;
    float m = neg_inf(), l = 0.f;
    f32x4 o = f32x4{0.f};
    // the prompt's slices, then its own
#pragma unroll 1
    for (int mine = a.shared[b] <= 0; mine < 2 && state == kFine; ++mine) {
      int least = a.small.least, tiles = a.B * blocks, tile = b * blocks + own_block, slices = a.own_slices, of = cols,
          x = r - own_block * cols, pages = own_pages;
      const float* part = a.own_part;
      if (!mine) {
        // the tile that b's queries are of begins at the last entry up to b that goes on with none
        const int e = last_at_most(s_runs, a.B, s_runs[b + 1] - 1);
        const bool is_small = s_small[e + 1] > s_small[e];
        of = is_small ? cols : a.prefix_cols;
        const int col = (b - e) * group + r, nth = col / of;
        x = col - nth * of;
        t.at<kPrefix>(a, e, of, nth, b - e + 1);  // (its rows up to b's)
        state = t.state;
        if (state != kFine) break;
        pages = t.keys.pages;
        tile = (is_small ? s_small[e] : s_large[e]) + nth;
        tiles = is_small ? small : large;
        slices = is_small ? small_slices : large_slices;
        least = is_small ? a.small.least : a.large.least;
        part = is_small ? a.small.part : a.large.part;
      }
      const Slices in = slices_of(a, pages, least, part, tiles, tile, slices, of, kvh, x);
      join_slices(m, l, o, in.at, in.stride, in.count, a.p.d, f);
    }
    if (state == kFine) {
      store_joined(a, i, f, m, l, o);
      continue;
    }
    const float none = state == kNone ? __builtin_nanf("") : 0.f;
    store_row4(a, i, f, f32x4{none, none, none, none});
    if (a.lse && f == 0) a.lse[i] = state == kNone ? none : neg_inf();
  }
}

constexpr int kMostJoins = 1024;  // workgroups of a join

int64_t blocks_of(int64_t rows, int cols) { return (rows + cols - 1) / cols; }
// Most pages that a tile of `cols` rows reads.
int most_pages(const KvTileArgs& a, int cols) {
  const int all = (int)blocks_of(a.n_ctx, kPage);
  if (!a.window) return all;
  return (int)std::min<int64_t>(all, blocks_of(a.sink, kPage) + blocks_of((int64_t)a.window + cols, kPage) + 1);
}
size_t row_bytes(const KvTileArgs& a) { return (size_t)(a.p.d + 4) * sizeof(float); }
// Partial tiles, at most: `tiles` tiles cut over the workgroups (two rounds of them).
int64_t partial_tiles(const KvTileArgs& a, const KvTileCut& cut, int64_t tiles) {
  return cut.most == 1 ? 0 : std::min<int64_t>(2 * cut.wgs, tiles * a.p.Hkv * cut.most);
}

// A slice keeps a step for each of a small tile's wavefronts (bf16: a page, fp32: half of
// one), and four pages of a large tile; a tile gets no more slices than its longest has such.
constexpr int kMostSlices = 512;
void limits(KvTileArgs& a, int cols) {
  const int cus = device_cu_count(), pages = most_pages(a, cols);
  auto cut = [&](int least, int wgs) {
    return KvTileCut{(int)std::min<int64_t>(kMostSlices, blocks_of(pages, least)), least, wgs, 0, nullptr};
  };
  a.small = cut(a.p.dtype == LLA_F32 ? 2 : 4, 2 * cus);
  a.large = cut(4, cus);
}

// Rows of a small tile: two products' columns where a group of heads is more than one's, and
// for packed tokens of wide heads: two wavefronts a SIMD, which one column leaves room
// for, hold no more registers than the step takes, and its masks need some (32 drafts of 5 tokens
// over 4001, 16 heads of 128: 264 us with one column, 188 with two; at a width of 64 24 heads
// on 8, 32 entries of 4 tokens over 1000, 25 and 30).
int small_cols_of(const KvTileArgs& a, bool packed) { return a.H / a.p.Hkv > 16 || (packed && a.p.d > 96) ? 32 : 16; }

struct PackedShape {
  int64_t small_tiles, large_tiles, small_partial, large_partial;
  explicit PackedShape(const KvTileArgs& a) {
    const int64_t rows = (int64_t)a.total * (a.H / a.p.Hkv);
    const int cols = large_cols(a.p.d);
    // every entry may end inside a tile; large ones have more than small_rows rows
    small_tiles = a.small_rows == 0 ? 0 : std::min(rows / a.small_cols + a.B, rows);
    if (a.small_rows != kAllRows) small_tiles = std::min(small_tiles, a.B * blocks_of(a.small_rows, a.small_cols));
    large_tiles = rows > a.small_rows ? std::min(rows / cols + a.B, blocks_of(rows, a.small_rows + 1)) : 0;
    small_partial = partial_tiles(a, a.small, small_tiles);
    large_partial = partial_tiles(a, a.large, large_tiles);
  }
  size_t bytes(const KvTileArgs& a) const {
    return (size_t)(small_partial * a.small_cols + large_partial * large_cols(a.p.d)) * row_bytes(a);
  }
};

}  // namespace

// Rows up to which an entry is of small tiles, by what the host knows.  fp32 has no large
// ones: small tiles read a page again for every 16 or 32 rows of an entry and keep the matrix units half busy
// (3 entries of 301 .. 101 tokens over 1020 of a window, 24 heads on 8 of 96: 100 us, 57 TFLOP/s, 7.2 TB/s of
// pages from the caches, units 51% busy), but the large fp32 tiles that were tried took 134 us.
// bf16, us with small tiles alone and with both kinds; a batch of few rows is not worth a second launch:
//   16 heads of 128 over 1000 tokens: 32 entries of 8 tokens 72 and 82, of 32 88 and 95, of 64 143 and 114
//   16 heads on 2:                     8 entries of 16 27 and 33, of 32 43 and 41; 32 entries of 16 58 and 45
//   24 heads on 8 of 64:               8 entries of 32 25 and 33; 32 entries of 16 37 and 42, of 32 54 and 44
// An entry of up to 32 rows, two small tiles, leaves most of a large one's 256 empty (200
// entries of 8 .. 1 tokens, 24 heads on 8 of 64: 80 and 133).  A single entry is of one
// kind, so that one launch does: over 4000 tokens 16 heads of 128, 32 tokens 27 and 26, 64 40 and 31;
// 16 heads on 2, 32 tokens 24 and 32, 64 38 and 35; on 4 of 256, 32 tokens 35 and 50, 64 56 and 57.
constexpr int kFewRows = 32, kBatchRows = 1024, kSingleRows = 1024;  // the last: of all heads
static int small_rows_of(const KvTileArgs& a) {
  const int64_t rows = (int64_t)a.total * (a.H / a.p.Hkv);
  if (a.p.dtype == LLA_F32 || rows <= kFewRows) return kAllRows;
  if (a.B == 1) return (int64_t)a.total * a.H < kSingleRows ? kAllRows : 0;
  return rows <= kBatchRows ? kAllRows : kFewRows;
}
static void packed_shape(KvTileArgs& a, int small_rows) {
  limits(a, large_cols(a.p.d));
  a.small_cols = small_cols_of(a, true);
  a.small_rows = small_rows;
}
size_t kv_prefill_shape(KvTileArgs& a) {
  packed_shape(a, small_rows_of(a));
  return PackedShape(a).bytes(a);
}
// Of any smaller batch: of small tiles alone, of both kinds, and of one entry with large ones, where it has such.
size_t kv_prefill_workspace(const KvTileArgs& a) {
  size_t most = 0;
  auto with = [&](int B, int64_t total, int small_rows) {
    KvTileArgs x = a;
    x.B = B;
    x.total = (int)std::min<int64_t>(a.total, total);
    packed_shape(x, small_rows);
    most = std::max(most, PackedShape(x).bytes(x));
  };
  const int group = a.H / a.p.Hkv;
  if (a.p.dtype == LLA_F32) {
    with(a.B, a.total, kAllRows);
    return most;
  }
  with(a.B, std::max(1, kBatchRows / group), kAllRows);
  KvTileArgs one = a;
  one.B = 1;
  if (small_rows_of(one) == 0) with(1, a.total, 0);
  if (small_rows_of(a) == kFewRows) with(a.B, a.total, kFewRows);
  return most;
}

hipError_t launch_kv_prefill(const KvTileArgs& args, hipStream_t stream) {
  KvTileArgs a = args;
  const PackedShape s(a);
  a.small.tiles = (int)s.small_tiles;
  a.large.tiles = (int)s.large_tiles;
  a.large.part = a.small.part + s.small_partial * a.small_cols * (a.p.d + 4);
  hipError_t e = hipSuccess;
  // (a workgroup takes another tile where there are more)
  auto grid = [&](int64_t tiles, int64_t partial) { return (unsigned)std::min<int64_t>(std::max(partial, tiles * a.p.Hkv), 1 << 16); };
  if (s.large_tiles) e = launch_large_packed(a, grid(s.large_tiles, s.large_partial), stream);
  if (e != hipSuccess) return e;
  // (a workgroup has to count the tiles: two rounds of those that run at a time; 200 entries of one
  // token, 16 heads of 128, 348 -> 328 us.  With one round fp32 prompts wait for the last ones, 29 -> 35)
  const unsigned small = grid(s.small_tiles, std::min<int64_t>(s.small_partial, a.small.wgs));
  if (s.small_tiles) e = launch_small_packed(a, std::min(small, 2u * a.small.wgs), stream);
  if (e != hipSuccess || s.small_partial + s.large_partial == 0) return e;
  const int64_t joins = s.small_partial * join_chunks(a.p.d, a.small_cols) + s.large_partial * join_chunks(a.p.d, large_cols(a.p.d));
  hipLaunchKernelGGL(join_packed_kernel, dim3((unsigned)std::min<int64_t>(joins, kMostJoins)), dim3(kThreads), 0, stream, a,
                     large_cols(a.p.d));
  return hipGetLastError();
}

namespace {
struct SharedShape {
  int64_t small_tiles, large_tiles;
  int64_t small, large, own;  // partial tiles: over prompts, small and large, and entries' own
  explicit SharedShape(const KvTileArgs& a) {
    const int group = a.H / a.p.Hkv;
    const int64_t rows = (int64_t)a.B * group, blocks = blocks_of(group, a.prefix_cols);
    auto items = [&](const KvTileCut& cut, int64_t tiles) { return std::max(partial_tiles(a, cut, tiles), tiles * a.p.Hkv); };
    // any entry may begin a run; small tiles are of runs of up to small_rows rows
    const int64_t runs = std::min<int64_t>(a.B, rows / (a.small_rows + (int64_t)1));
    small_tiles = a.small_rows == kAllRows ? a.B * blocks : group <= a.small_rows ? a.B : 0;
    large_tiles = runs * blocks;
    small = items(a.small, small_tiles);
    large = items(a.large, large_tiles);
    own = (int64_t)a.B * a.p.Hkv * blocks_of(group, a.small_cols) * a.own_slices;
  }
  size_t bytes(const KvTileArgs& a) const {
    return (size_t)((small + own) * a.small_cols + large * a.prefix_cols) * row_bytes(a);
  }
};
}  // namespace

// Whether runs of more than a small tile's rows take large tiles: bf16, from 3 * 2^30
// multiply-adds of all queries with the whole context on.  32 heads on 8 of 128, us with small
// tiles alone and with large ones: over a prompt of 4096 tokens 64 answers 56 and 70, 128
// 80 and 91, 256 134 and 122, 1000 439 and 310; of 16,384 tokens 32 81 and 82, 64 116 and
// 103, 128 183 and 132.  2 prompts of 64 answers, 16 heads on 2 of 64: 36 and 51; 8 of 4, 16 heads
// of 128 over 2001: 50 and 57.  In fp32 the matrix instructions take as long from either.
static bool shared_large(const KvTileArgs& a) {
  return a.p.dtype == LLA_BF16 && (int64_t)a.B * a.H * a.p.d * a.n_ctx >= (int64_t)3 << 30;
}
static void shared_shape(KvTileArgs& a, bool large) {
  limits(a, 0);
  a.small_cols = small_cols_of(a, false);
  const int64_t units = (int64_t)a.B * a.p.Hkv * blocks_of(a.H / a.p.Hkv, a.small_cols);
  a.small_rows = large ? a.small_cols : kAllRows;
  a.prefix_cols = large ? large_cols(a.p.d) : a.small_cols;
  a.own_slices =
      (int)std::max<int64_t>(1, std::min<int64_t>(a.small.wgs / units, a.small.most));
}
size_t kv_shared_shape(KvTileArgs& a) {
  shared_shape(a, shared_large(a));
  return SharedShape(a).bytes(a);
}
// Of any smaller batch, which may have small tiles alone: the partial tiles over prompts grow with the entries,
// and of own ones there are no more than workgroups, or than entries have without a cut.
size_t kv_shared_workspace(const KvTileArgs& a) {
  size_t most = 0;
  for (const bool large : {false, true}) {
    if (large && !shared_large(a)) continue;
    KvTileArgs x = a;
    shared_shape(x, large);
    SharedShape s(x);
    const int64_t units = s.own / x.own_slices;
    s.own = std::min(std::max<int64_t>(x.small.wgs, units), units * x.small.most);
    most = std::max(most, s.bytes(x));
  }
  return most;
}

hipError_t launch_kv_shared(const KvTileArgs& args, hipStream_t stream) {
  KvTileArgs a = args;
  const SharedShape s(a);
  a.small.tiles = (int)s.small_tiles;
  a.large.tiles = (int)s.large_tiles;
  a.own_part = a.small.part + s.small * a.small_cols * (a.p.d + 4);
  a.large.part = a.own_part + s.own * a.small_cols * (a.p.d + 4);
  auto grid = [](int64_t items) { return (unsigned)std::min<int64_t>(items, 1 << 16); };
  hipError_t e = hipSuccess;
  if (s.large) e = launch_large_prefix(a, grid(s.large), stream);
  if (e != hipSuccess) return e;
  // (a workgroup has to count the tiles over prompts: no more of them than run at a time, however
  // few of the tiles that there may be there are; 512 answers 178 -> 126 us)
  e = launch_small_shared(a, (unsigned)std::min<int64_t>(s.small + s.own, a.small.wgs), stream);
  if (e != hipSuccess) return e;
  const int64_t joins = blocks_of((int64_t)a.B * a.H, join_rows(a.p.d));
  hipLaunchKernelGGL(join_shared_kernel, dim3((unsigned)std::min<int64_t>(joins, kMostJoins)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace lla
