// Work of the attention of packed tokens and of shared prompts over the paged K/V
// cache: which rows make a tile, which pages it reads, and how tiles are shared out
// (kv_tile_small.h, kv_join.hip).
//
// A tile is up to kCols rows (token or entry, query head of the group) that read the
// same pages for one key head.  How many tiles a call has is known on the device
// alone, by the offsets of a packed batch or the groups of a shared one, so each
// workgroup counts them itself (a prefix sum over at most 1024 entries, 1 us), and with
// fewer tiles than workgroups the pages of each are split.
#pragma once

#include "kv_internal.h"
#include "lla_device.h"

namespace lla {

constexpr int kMostEntries = 1024;

enum TileMode { kPacked, kPrefix, kOwn };

// Keys that a tile attends: row by row, places up to p that lie below `sink` or from
// `low` on; the pages with any of them are 0 .. lead - 1, then lead + skip .. .
struct TileKeys {
  int sink, low_min, low_max, p_min, p_max;
  int lead, skip, pages;
  __device__ __forceinline__ void plan() {
    const int all = p_max < 0 ? 0 : p_max / kPage + 1;
    const bool cut = low_min > sink;
    lead = cut ? min(all, (sink + kPage - 1) / kPage) : all;
    skip = cut ? max(0, min(all, low_min / kPage) - lead) : 0;
    pages = all - skip;
  }
  __device__ __forceinline__ int page(int i) const { return i < lead ? i : i + skip; }
  // whether all rows attend all of t .. t + count - 1
  __device__ __forceinline__ bool whole(int t, int count) const {
    return t + count - 1 <= p_min && (t >= low_max || t + count <= sink);
  }
};

// A row's keys.
struct RowKeys {
  int p, low;
  __device__ __forceinline__ bool seen(int t, int sink) const { return t <= p && (t < sink || t >= low); }
  // any of t .. t + count - 1
  __device__ __forceinline__ bool any(int t, int count, int sink) const {
    const int last = min(t + count - 1, p);
    return last >= t && (t < sink || last >= low);
  }
};

// What stands in the place of a tile's results: zeros for padding, NaN where an index
// is out of its range.
enum TileState { kFine, kZeros, kNone };

// Sum over the workgroup of v's of lower threads.
template <int kThreads, typename V>
__device__ __forceinline__ V prefix_sum(V v, V* s_wave) {
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  V x = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const V y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == kWave - 1) s_wave[w] = x;
  __syncthreads();
  V before = 0;
#pragma unroll
  for (int i = 0; i < kThreads / kWave; ++i) before += i < w ? s_wave[i] : 0;
  return before + x - v;
}

// The largest b in [0, n) with s_at[b] <= x (s_at[0] <= x).
__device__ __forceinline__ int last_at_most(const int* s_at, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (s_at[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// First packed token of entry b, within the tokens that there are.
__device__ __forceinline__ int offset_of(const KvTileArgs& a, int b) { return max(0, min(a.offset[b], a.total)); }

// Entries of a prefix tile: those of one run of equal (lead, shared), cut where the
// entry's number is a multiple of these many.
__host__ __device__ __forceinline__ int tile_entries(int group, int cols) { return group >= cols ? 1 : cols / group; }

// s_first[b] = tiles of the entries before b, s_first[B] = all.
//   kPacked: tiles of entries with more than `over` and at most `upto` rows
//   kPrefix: a run's tile, at its first entry
template <TileMode Mode, int kThreads>
__device__ __forceinline__ void count_tiles(const KvTileArgs& a, int cols, int over, int upto, int* s_first, int* s_wave) {
  constexpr int kEach = (kMostEntries + kThreads - 1) / kThreads;
  const int tid = threadIdx.x, group = a.H / a.p.Hkv;
  int n[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = tid * kEach + i;
    n[i] = 0;
    if (b < a.B) {
      if constexpr (Mode == kPacked) {
        const int64_t rows = (int64_t)max(0, offset_of(a, b + 1) - offset_of(a, b)) * group;
        if (rows > over && rows <= upto) n[i] = (int)((rows + cols - 1) / cols);
      } else {
        const int lead = a.lead[b], shared = a.shared[b];
        if (shared > 0) {
          const bool first = b % tile_entries(group, cols) == 0 || a.lead[b - 1] != lead || a.shared[b - 1] != shared;
          n[i] = first ? (group + cols - 1) / cols : 0;
        }
      }
    }
    sum += n[i];
  }
  int at = prefix_sum<kThreads>(sum, s_wave);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = tid * kEach + i;
    if (b < a.B) s_first[b] = at;
    at += n[i];
    if (b == a.B - 1) s_first[a.B] = at;
  }
  __syncthreads();
}

// Slices that every tile may be cut into: as many as the workgroups there are for.
__device__ __forceinline__ int tile_slices(const KvTileArgs& a, int tiles, int workgroups) {
  const int64_t units = (int64_t)tiles * a.p.Hkv;
  return units == 0 || a.most == 1 ? 1 : (int)max((int64_t)1, min((int64_t)a.most, workgroups / units));
}
__device__ __forceinline__ int slice_pages(const KvTileArgs& a, int pages, int slices) {
  return slices == 1 ? max(pages, 1) : max(a.least, (pages + slices - 1) / slices);
}

// One tile of one key head.
struct Tile {
  int entry, first;  // its first entry; the first of its rows among the entry's
  int rows;          // rows
  int row;           // the sequence whose pages it reads
  TileState state;
  TileKeys keys;

  // Tile t of the call's; s_first as count_tiles left it.
  template <TileMode Mode>
  __device__ __forceinline__ void find(const KvTileArgs& a, const int* s_first, int cols, int t) {
    entry = last_at_most(s_first, a.B, t);
    at<Mode>(a, s_first, cols, t - s_first[entry]);
  }
  // The entry's tile number `nth`.
  template <TileMode Mode>
  __device__ __forceinline__ void at(const KvTileArgs& a, const int* s_first, int cols, int nth) {
    const int group = a.H / a.p.Hkv, b = entry;
    first = nth * cols;
    state = kFine;
    keys.sink = 0;
    keys.low_min = keys.low_max = 0;
    if constexpr (Mode == kPacked) {
      const int n = offset_of(a, b + 1) - offset_of(a, b), start = a.start[b];
      rows = min((int64_t)cols, (int64_t)n * group - first);
      row = a.rows ? a.rows[b] : b;
      if ((a.rows && row == -1) || start < 0) state = kZeros;
      else if (row < 0 || row >= a.p.n_seqs) state = kNone;
      const int64_t p0 = (int64_t)start + first / group, p1 = (int64_t)start + (first + rows - 1) / group;
      keys.p_min = (int)min(p0, (int64_t)a.n_ctx - 1);
      keys.p_max = (int)min(p1, (int64_t)a.n_ctx - 1);
      if (a.window) {
        keys.sink = a.sink;
        keys.low_min = (int)max((int64_t)0, keys.p_min - (int64_t)a.window + 1);
        keys.low_max = (int)max((int64_t)0, keys.p_max - (int64_t)a.window + 1);
      }
    } else if constexpr (Mode == kPrefix) {
      const int lead = a.lead[b];
      int many = 1;
      if (group < cols)
        while (many < tile_entries(group, cols) && b + many < a.B && (b + many) % tile_entries(group, cols) &&
               a.lead[b + many] == lead && a.shared[b + many] == a.shared[b])
          ++many;
      rows = min(cols, many * group - first);
      state = lead < 0 || lead >= a.B ? kNone : kFine;
      row = state == kFine ? (a.rows ? a.rows[lead] : lead) : -1;
      if (row < 0 || row >= a.p.n_seqs) state = kNone;
      else if (a.shared[b] > a.length[row] || a.shared[b] > a.n_ctx) state = kNone;
      keys.p_min = keys.p_max = a.shared[b] - 1;
    } else {
      rows = min(cols, group - first);
      row = a.rows ? a.rows[b] : b;
      int n = 0;
      if (a.rows && row == -1) state = kZeros;
      else if (row < 0 || row >= a.p.n_seqs) state = kNone;
      else {
        n = a.length[row];
        if (n == 0) state = kZeros;
        else if (n < 0 || n > a.n_ctx || a.shared[b] < 0 || a.shared[b] > n) state = kNone;
      }
      keys.p_min = keys.p_max = state == kFine ? n - 1 : -1;
      keys.low_min = keys.low_max = state == kFine ? a.shared[b] : 0;
    }
    if (state != kFine) keys.p_max = -1;
    keys.plan();
    // an entry whose tokens are all shared has none of its own
    if (Mode == kOwn && state == kFine && keys.low_min > keys.p_max) keys.pages = 0;
  }

  // Row x of the tile for key head kvh: where its query starts and its result goes,
  // and its keys.
  template <TileMode Mode>
  __device__ __forceinline__ RowKeys row_keys(const KvTileArgs& a, int kvh, int x, int64_t& q, int64_t& out) const {
    const int group = a.H / a.p.Hkv, i = (first + x) / group, h = kvh * group + (first + x) - i * group;
    const int64_t t = (Mode == kPacked ? offset_of(a, entry) : entry) + i;
    q = t * a.q_t + (int64_t)h * a.p.d;
    out = t * a.H + h;
    RowKeys k;
    if constexpr (Mode == kPacked) {
      k.p = (int)min((int64_t)a.start[entry] + i, (int64_t)a.n_ctx - 1);
      k.low = a.window ? (int)max((int64_t)0, k.p - (int64_t)a.window + 1) : 0;
    } else {
      k.p = keys.p_max;
      k.low = keys.low_min;
    }
    return k;
  }
  // Whether row x lies at or past the bound on the lengths.
  template <TileMode Mode>
  __device__ __forceinline__ bool past_bound(const KvTileArgs& a, int x) const {
    return Mode == kPacked && (int64_t)a.start[entry] + (first + x) / (a.H / a.p.Hkv) >= a.n_ctx;
  }
};

// A partial row: d sums, the maximum (log2 units), the sum of weights, padding.
__device__ __forceinline__ float* partial_row(float* part, int64_t item, int cols, int x, int d) {
  return part + (item * cols + x) * (d + 4);
}
// Number of (slice, tile, key head) among the call's work: heavy tiles of a prompt, its
// last, first, and one key head's work a multiple of the key heads apart, so on one XCD
// where 8 divides them.
__device__ __forceinline__ int64_t item_of(const KvTileArgs& a, int tiles, int slice, int tile, int kvh) {
  return ((int64_t)slice * tiles + (tiles - 1 - tile)) * a.p.Hkv + kvh;
}

// Four features from f on of result row i.
template <typename V>
__device__ __forceinline__ void store_row4(const KvTileArgs& a, int64_t i, int f, V v) {
  const int64_t at = i * a.p.d + f;
  if (a.out_dtype == 1) {
    uint2 w;
    w.x = f32_to_bf16(v[0]) | (uint32_t(f32_to_bf16(v[1])) << 16);
    w.y = f32_to_bf16(v[2]) | (uint32_t(f32_to_bf16(v[3])) << 16);
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.out) + at) = w;
  } else {
    *reinterpret_cast<V*>(static_cast<float*>(a.out) + at) = v;
  }
}

}  // namespace lla
