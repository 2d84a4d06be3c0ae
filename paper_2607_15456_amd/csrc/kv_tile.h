// Work of the attention of packed tokens and of shared prompts over the paged K/V
// cache: which rows make a tile, which pages it reads, and how tiles are shared out
// (kv_tile_small.h, kv_tile_large.h, kv_attn.hip).
//
// A tile is up to kCols rows (token or entry, query head of the group) that read the
// same pages for one key head.  How many tiles a call has is known on the device
// alone, by the offsets of a packed batch or the groups of a shared one, so each
// workgroup counts them itself (a prefix sum over at most 1024 entries), and with fewer
// tiles than workgroups the pages of each are split.
#pragma once

#include "kv_internal.h"
#include "lla_device.h"

namespace lla {

constexpr int kMostEntries = 1024;
constexpr int kAllRows = 0x7fffffff;  // small_rows: all tiles are small ones

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

// Sums stop here: counts of sound arguments stay below, others' do no harm.  Two sums
// that have stopped add up to less than 2^31.
constexpr int kMostSum = (1 << 30) - 1;
__device__ __forceinline__ int add_up(int x, int y) { return min(x + y, kMostSum); }

// Sum over the workgroup of v's of lower threads (0 <= v <= kMostSum).
template <int kThreads>
__device__ __forceinline__ int prefix_sum(int v, int* s_wave) {
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  int x = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(x, o, kWave);
    if (lane >= o) x = add_up(x, y);
  }
  const int lower = __shfl_up(x, 1, kWave);
  __syncthreads();
  if (lane == kWave - 1) s_wave[w] = x;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int i = 0; i < kThreads / kWave; ++i) before = add_up(before, i < w ? s_wave[i] : 0);
  return add_up(before, lane ? lower : 0);
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

// Tiles of entries' counts n[] (entries tid * kEach ..) before each: s_first[b], all in s_first[B].
template <int kThreads>
struct EntryCounts {
  static constexpr int kEach = (kMostEntries + kThreads - 1) / kThreads;
  int n[kEach];
  __device__ __forceinline__ static int entry(int i) { return threadIdx.x * kEach + i; }
  __device__ __forceinline__ void sum(int B, int* s_first, int* s_wave) const {
    int total = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) total = add_up(total, n[i]);
    int at = prefix_sum<kThreads>(total, s_wave);
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int b = entry(i);
      if (b < B) s_first[b] = at;
      at = add_up(at, n[i]);
      if (b == B - 1) s_first[B] = at;
    }
    __syncthreads();
  }
};

// Packed entries with more than `over` and at most `upto` rows.
template <int kThreads>
__device__ __forceinline__ void count_packed(const KvTileArgs& a, int cols, int over, int upto, int* s_first, int* s_wave) {
  const int group = a.H / a.p.Hkv;
  EntryCounts<kThreads> c;
#pragma unroll
  for (int i = 0; i < c.kEach; ++i) {
    const int b = c.entry(i);
    c.n[i] = 0;
    if (b < a.B) {
      const int64_t rows = (int64_t)max(0, offset_of(a, b + 1) - offset_of(a, b)) * group;
      if (rows > over && rows <= upto) c.n[i] = (int)((rows + cols - 1) / cols);
    }
  }
  c.sum(a.B, s_first, s_wave);
}

// Sum over the wavefront.
__device__ __forceinline__ int wave_sum(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);   // of rows of 16 lanes:
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row 0 into 1, 2 into 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // the first two into the others
  return __builtin_amdgcn_readlane(v, kWave - 1);
}

// The x-th tile of a packed batch, those that stand last in their sequences first: what
// a causal tile costs goes by its place, and a heavy one that begins late would run
// alone at the end.  Tiles are numbered by their places' tile in the sequence, v = s_from[b] + nth;
// at_least(v) counts those at v or behind; none is behind `most`.  Every wavefront of the
// workgroup finds it.
struct HeavyFirst {
  const int *s_first, *s_from;
  int B;
  // tiles of entry b at v or behind
  __device__ __forceinline__ int behind(int b, int v) const {
    const int n = s_first[b + 1] - s_first[b];
    return max(0, min(n, s_from[b] + n - v));
  }
  __device__ __forceinline__ int at_least(int v) const {
    int n = 0;
    for (int b = threadIdx.x % kWave; b < B; b += kWave) n += behind(b, v);
    return wave_sum(n);
  }
  __device__ __forceinline__ void find(int x, int most, int& entry, int& nth) const {
    int lo = 0, hi = most;  // the greatest v with at_least(v) > x
    while (lo < hi) {
      const int mid = lo + (hi - lo + 1) / 2;
      if (at_least(mid) > x) lo = mid;
      else hi = mid - 1;
    }
    int skip = max(0, x - at_least(lo + 1));  // of the entries with a tile at lo
    entry = nth = 0;
    for (int b0 = 0; b0 < B; b0 += kWave) {
      const int b = b0 + threadIdx.x % kWave;
      const uint64_t in = __ballot(b < B && behind(min(b, B - 1), lo) > behind(min(b, B - 1), lo + 1));
      const int here = __popcll(in);
      if (skip < here) {
        uint64_t left = in;
        for (; skip; --skip) left &= left - 1;
        entry = b0 + __builtin_ctzll(left);
        nth = lo - s_from[entry];
        return;
      }
      skip -= here;
    }
  }
};

// Entries of a tile over a shared prompt: a run of equal (lead, shared), cut where the
// entry's number is a multiple of these many.
__host__ __device__ __forceinline__ int tile_entries(int group, int cols) { return group >= cols ? 1 : cols / group; }

// Tiles over shared prompts.  s_runs[b]: entries before b that do not go on with the tile
// of the one before them; then the tiles of at most small_rows rows, which are small
// ones, and the others, where an array for them is given.
template <int kThreads>
__device__ __forceinline__ void count_shared(const KvTileArgs& a, int* s_runs, int* s_small, int* s_large,
                                             int* s_wave) {
  const int group = a.H / a.p.Hkv, each = tile_entries(group, a.prefix_cols);
  EntryCounts<kThreads> c, small, large;
  bool begins[c.kEach];
#pragma unroll
  for (int i = 0; i < c.kEach; ++i) {
    const int b = c.entry(i);
    c.n[i] = 0;
    begins[i] = false;
    if (b < a.B) {
      const int lead = a.lead[b], shared = a.shared[b];
      const bool first = shared <= 0 || b % each == 0 || a.lead[b - 1] != lead || a.shared[b - 1] != shared;
      c.n[i] = first;
      begins[i] = first && shared > 0;
    }
  }
  c.sum(a.B, s_runs, s_wave);
#pragma unroll
  for (int i = 0; i < c.kEach; ++i) {
    const int b = c.entry(i);
    small.n[i] = large.n[i] = 0;
    if (!begins[i]) continue;
    // few: all tiles are, or the run has at most `most` entries: one behind it begins
    // another, or there are no more
    const int most = a.small_rows / group, blocks = (group + a.prefix_cols - 1) / a.prefix_cols;
    const bool few = a.small_rows == kAllRows ||
                     (most >= 1 && (b + most >= a.B || s_runs[b + most + 1] > s_runs[b + 1]));
    small.n[i] = few ? blocks : 0;  // (a choice between the two would put both into memory)
    large.n[i] = few ? 0 : blocks;
  }
  if (s_small) small.sum(a.B, s_small, s_wave);
  if (s_large) large.sum(a.B, s_large, s_wave);
}
// Entries of the tile that begins at b.
__device__ __forceinline__ int run_entries(const KvTileArgs& a, const int* s_runs, int b) {
  return last_at_most(s_runs, a.B + 1, s_runs[b + 1]) - b;
}

// The tiles that are worked on, of those that were counted.
__device__ __forceinline__ int tiles_of(const KvTileCut& cut, int counted) { return min(counted, cut.tiles); }
// Slices that every tile may be cut into, where there are fewer tiles than workgroups:
// as many as give each a workgroup, or so many that two rounds of workgroups do better.
__device__ __forceinline__ int tile_slices(const KvTileCut& cut, int units) {
  if (units <= 0 || cut.most == 1 || units >= 2 * cut.wgs) return 1;
  const int one = max(1, cut.wgs / units), two = 2 * cut.wgs / units;
  return min(cut.most, 9 * two > 20 * one ? two : one);
}
__device__ __forceinline__ int slice_pages(int least, int pages, int slices) {
  return slices == 1 ? max(pages, 1) : max(least, (pages + slices - 1) / slices);
}

// One tile of one key head.
struct Tile {
  int entry, first;  // its first entry; the first of its rows among the entry's
  int rows;          // rows
  int row;           // the sequence whose pages it reads
  TileState state;
  TileKeys keys;

  // Entry b's tile number nth, of `cols` rows; many: the entries of a tile over a shared
  // prompt.
  template <TileMode Mode>
  __device__ __forceinline__ void at(const KvTileArgs& a, int b, int cols, int nth, int many = 1) {
    entry = b;
    const int group = a.H / a.p.Hkv;
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
        if (n < 0 || n > a.n_ctx || a.shared[b] < 0 || a.shared[b] > n) state = kNone;
        else if (n == 0) state = kZeros;
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
__device__ __forceinline__ int item_of(const KvTileArgs& a, int tiles, int slice, int tile, int kvh) {
  return (slice * tiles + (tiles - 1 - tile)) * a.p.Hkv + kvh;
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

// The kernel's arguments, read again from memory: a value that is needed before and after
// the steps need not be held meanwhile.
__device__ __forceinline__ const KvTileArgs& args_again() {
  typedef const KvTileArgs __attribute__((address_space(4))) Kernarg;
  Kernarg* p = (Kernarg*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const KvTileArgs*)p;
}

// A pointer that is the same in all lanes, in scalar registers.
template <typename T>
__device__ __forceinline__ const T* scalar(const T* p) {
  const uint64_t x = reinterpret_cast<uintptr_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
  return reinterpret_cast<const T*>(((uint64_t)hi << 32) | lo);
}

// Values that are not finite, of tokens that only some of a tile's rows attend, stay out
// of the matrix product (a weight of zero would make NaN of them).  This adds them to the
// stored results, or partial rows, of the rows that attend them; rare, so nothing of it is
// held in registers meanwhile.  part: the tile's partial rows, or NULL.
template <TileMode Mode, typename T, int D, int kThreads>
__device__ __forceinline__ void add_nonfinite(const KvTileArgs& a, const Tile& t, int kvh, int pb, int pe, float* part) {
  constexpr int N = Elem<T>::kPer16B;
  __syncthreads();  // the results are stored
#pragma unroll 1
  for (int e = threadIdx.x; e < t.rows * D; e += kThreads) {
    const int x = e / D, f = e - x * D;
    int64_t q_at, out_at;
    const RowKeys rk = t.row_keys<Mode>(a, kvh, x, q_at, out_at);
    float sum = 0.f;
    bool any = false;
#pragma unroll 1
    for (int i = pb; i < pe; ++i) {
      const int t0 = t.keys.page(i) * kPage, page = a.p.table[(int64_t)t.row * a.p.max_pages + t.keys.page(i)];
      if (t.keys.whole(t0, kPage) || page < 0 || page >= a.p.n_pages) continue;
      const T* v = static_cast<const T*>(a.p.v) + (((int64_t)page * a.p.Hkv + kvh) * D + f) * kPage;
#pragma unroll 1
      for (int k = 0; k < kPage; k += N) {
        float y[N];
        Elem<T>::unpack(ld16(v + k), y);
#pragma unroll
        for (int n = 0; n < N; ++n)
          if ((__float_as_uint(y[n]) & 0x7f800000u) == 0x7f800000u && rk.seen(t0 + k + n, t.keys.sink)) {
            sum += y[n];
            any = true;
          }
      }
    }
    if (!any) continue;
    const int64_t at = out_at * D + f;
    if (part) part[x * (D + 4) + f] += sum;
    else if (a.out_dtype == 1) static_cast<bf16_t*>(a.out)[at] = f32_to_bf16(bf16_to_f32(static_cast<bf16_t*>(a.out)[at]) + sum);
    else static_cast<float*>(a.out)[at] += sum;
  }
  __syncthreads();
}

}  // namespace lla
