// Bookkeeping of the paged K/V cache on the device: room for new tokens with
// copy on write, sharing, freeing, and the copies of pages and tokens.
//
// The three table calls each run in one workgroup of up to 1024 sequences: the
// rows' needs are a prefix sum, so the outcome is that of one row after another
// in any run, with no lock and no order of atomics that shows.  They move a few
// words a page; a launch and a chain of dependent reads bound them (16 rows of 36
// pages dropped, forked and given room: 16.9 us for the three calls), for thousands of
// pages the scattered words that one compute unit can ask for and the search for rows
// named twice, n^2 / 2 reads of LDS (256 rows of 36 pages 121, 1000 of 30 437).

#include "kv_internal.h"
#include "lla_device.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

constexpr int kRows = LLA_KV_MAX_ROWS, kThreads = 1024;
constexpr int kPadding = -1;  // a row that a call passes over

__device__ __forceinline__ int pages_of(int64_t n) { return (int)((n + kPage - 1) / kPage); }

// Sum over the workgroup of v's of lower threads; total gets the whole sum.
__device__ __forceinline__ int prefix(int v, int* s_wave, int& total) {
  const int lane = threadIdx.x % kWave, w = threadIdx.x / kWave;
  int x = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(x, o, kWave);
    if (lane >= o) x += y;
  }
  __syncthreads();  // s_wave may still be read by an earlier call
  if (lane == kWave - 1) s_wave[w] = x;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int i = 0; i < kThreads / kWave; ++i) {
    if (i < w) before += s_wave[i];
    total += s_wave[i];
  }
  return before + x - v;
}

// A sequence number in range, named once in s_row[0 .. n).
__device__ __forceinline__ bool sound(const int* s_row, int i, int n_seqs) {
  const int r = s_row[i];
  bool ok = r >= 0 && r < n_seqs;
  for (int j = 0; j < i; ++j) ok &= s_row[j] != r;
  return ok;
}

// Row of entry e, where row i has the entries s_at[i] .. s_at[i + 1] - 1.
__device__ __forceinline__ int row_of(const int* s_at, int n, int e) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (s_at[mid] <= e) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ void report(const TableArgs& a, int status, int pairs, int pages, int left) {
  a.result[0] = status;
  a.result[1] = pairs;
  a.result[2] = pages;
  a.result[3] = left;
}

__global__ __launch_bounds__(kThreads) void reserve_kernel(TableArgs a) {
  __shared__ int s_row[kRows], s_open[kRows], s_at[kRows], s_have[kRows], s_wave[kThreads / kWave];
  const int i = threadIdx.x;
  s_row[i] = i < a.n ? a.rows[i] : kPadding;
  const bool mine = s_row[i] != kPadding;
  __syncthreads();
  bool ok = !mine || sound(s_row, i, a.n_seqs);
  const int row = mine && ok ? s_row[i] : -1;
  const int add = row >= 0 ? a.more[i] : 0;
  const int len = row >= 0 ? a.length[row] : 0;
  const int64_t end = (int64_t)len + add;
  ok = ok && add >= 0 && len >= 0 && end <= (int64_t)a.max_pages * kPage;
  const int n_free = a.free_pages[0];
  int* const table = a.table + (int64_t)max(row, 0) * a.max_pages;
  // the page that the sequence ends in, if it ends inside one and will grow
  int open = -1, holders = 0;
  if (row >= 0 && ok && add > 0 && len % kPage) {
    open = table[len / kPage];
    if (open < 0 || open >= a.n_pages) ok = false;
    else holders = a.refs[open];
  }
  s_open[i] = open;
  ok = ok && n_free >= 0 && n_free <= a.n_pages;
  if (!__syncthreads_and(ok)) {
    if (i < a.n) a.start[i] = -1;
    if (i == 0) report(a, LLA_PAGES_BAD, 0, 0, n_free);
    return;
  }
  // each earlier row with the same open page took a copy if this one can
  int before = 0;
  if (open >= 0)
    for (int j = 0; j < i; ++j) before += s_open[j] == open;
  const bool copy = open >= 0 && holders - before > 1;
  const int have = pages_of(len) - (copy ? 1 : 0);
  const int need = row >= 0 ? pages_of(end) - have : 0;
  int total, pairs;
  const int at = prefix(need, s_wave, total);
  const int pair = prefix(copy ? 1 : 0, s_wave, pairs);
  if (total > n_free) {
    if (i < a.n) a.start[i] = -1;
    if (i == 0) report(a, LLA_PAGES_FULL, 0, 0, n_free);
    return;
  }
  s_at[i] = at;
  s_have[i] = have;
  if (row >= 0) {
    if (copy) {
      atomicSub(&a.refs[open], 1);
      a.pairs[2 * pair] = open;
      a.pairs[2 * pair + 1] = a.free_pages[n_free - at];  // the row's first
    }
    a.start[i] = len;
    a.length[row] = (int)end;
  } else if (i < a.n) {
    a.start[i] = -1;
  }
  __syncthreads();
  for (int e = i; e < total; e += kThreads) {
    const int r = row_of(s_at, a.n, e);
    const int page = a.free_pages[n_free - e];
    a.table[(int64_t)s_row[r] * a.max_pages + s_have[r] + e - s_at[r]] = page;
    if (page >= 0 && page < a.n_pages) a.refs[page] = 1;
  }
  if (i == 0) {
    a.free_pages[0] = n_free - total;
    report(a, LLA_PAGES_OK, pairs, total, n_free - total);
  }
}

__global__ __launch_bounds__(kThreads) void fork_kernel(TableArgs a) {
  __shared__ int s_row[kRows], s_src[kRows], s_at[kRows], s_wave[kThreads / kWave];
  const int i = threadIdx.x;
  s_row[i] = i < a.n ? a.rows[i] : kPadding;
  const bool mine = s_row[i] != kPadding;
  s_src[i] = mine ? a.more[i] : -1;
  __syncthreads();
  bool ok = true;
  int len = 0;
  if (mine) {
    const int src = s_src[i];
    ok = sound(s_row, i, a.n_seqs) && src >= 0 && src < a.n_seqs;
    for (int j = 0; j < a.n; ++j) ok &= s_row[j] != src;
    if (ok) {
      len = a.length[src];
      ok = a.length[s_row[i]] == 0 && len >= 0 && len <= (int64_t)a.max_pages * kPage;
    }
  }
  if (!__syncthreads_and(ok)) {
    if (i == 0) report(a, LLA_PAGES_BAD, 0, 0, a.free_pages[0]);
    return;
  }
  int entries;
  s_at[i] = prefix(pages_of(len), s_wave, entries);
  if (mine) a.length[s_row[i]] = len;
  __syncthreads();
  for (int e = i; e < entries; e += kThreads) {
    const int r = row_of(s_at, a.n, e), k = e - s_at[r];
    const int page = a.table[(int64_t)s_src[r] * a.max_pages + k];
    a.table[(int64_t)s_row[r] * a.max_pages + k] = page;
    if (page >= 0 && page < a.n_pages) atomicAdd(&a.refs[page], 1);
  }
  if (i == 0) report(a, LLA_PAGES_OK, 0, 0, a.free_pages[0]);
}

// Freeing goes over all (row, page) entries.  Holders are counted down; the
// entry that takes the last one gives the page back, unless several entries of
// the call name that page: then the first of them does, which is found by the
// least rank, lowered by 2^31, that lands in refs.  Pages given back are laid onto
// the stack, the last first.
__global__ __launch_bounds__(kThreads) void free_kernel(TableArgs a) {
  constexpr int kHeld = 8;   // entries of a thread whose pages it keeps
  constexpr int kNamed = (int)0x80000000;
  __shared__ int s_row[kRows], s_at[kRows], s_wave[kThreads / kWave];
  const int i = threadIdx.x;
  s_row[i] = i < a.n ? a.rows[i] : kPadding;
  const bool mine = s_row[i] != kPadding;
  __syncthreads();
  bool ok = true;
  int len = 0;
  const int n_free = a.free_pages[0];
  if (mine) {
    ok = sound(s_row, i, a.n_seqs);
    if (ok) len = a.length[s_row[i]];
    ok = ok && len >= 0 && len <= (int64_t)a.max_pages * kPage;
  }
  ok = ok && n_free >= 0 && n_free <= a.n_pages;
  if (!__syncthreads_and(ok)) {
    if (i == 0) report(a, LLA_PAGES_BAD, 0, 0, n_free);
    return;
  }
  int entries;
  s_at[i] = prefix(pages_of(len), s_wave, entries);
  __syncthreads();
  auto entry = [&](int e) -> int32_t* {
    const int r = row_of(s_at, a.n, e);
    return a.table + (int64_t)s_row[r] * a.max_pages + (e - s_at[r]);
  };
  auto page_at = [&](int e) {
    const int page = e < entries ? *entry(e) : -1;
    return page >= 0 && page < a.n_pages ? page : -1;
  };
  auto each = [&](auto f) {
    for (int e = i; e < entries; e += kThreads) {
      const int page = page_at(e);
      if (page >= 0) f(e, page);
    }
  };
  auto holders = [&](int page) {
    return __hip_atomic_load(&a.refs[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  // lays down the pages of this round's threads that give one back (the last
  // first, so the first is on top once all `total` are there)
  int done = 0;
  auto lay = [&](int page, bool back, int total) {
    int round;
    const int at = done + prefix(back ? 1 : 0, s_wave, round);
    if (back && at < total) a.free_pages[n_free + total - at] = page;
    done += round;
  };
  const int room = a.n_pages - n_free;  // (more than this only if a table was damaged)
  int total;
  bool again = entries > kHeld * kThreads;
  if (!again) {
    int page[kHeld], old[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) page[k] = k * kThreads < entries ? page_at(i + k * kThreads) : -1;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      old[k] = 2;
      if (page[k] >= 0) old[k] = atomicSub(&a.refs[page[k]], 1);
    }
    wait_stores_in_l2();
    __syncthreads();
    int twice = 0, back = 0;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      if (k * kThreads >= entries) break;
      back += old[k] == 1;
      if (page[k] >= 0 && old[k] != 1) twice |= holders(page[k]) <= 0;
    }
    again = __syncthreads_or(twice);
    if (!again) {
      prefix(back, s_wave, total);
      total = min(total, room);
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
        if (k * kThreads < entries) lay(page[k], old[k] == 1, total);
    }
  } else {
    each([&](int, int page) { atomicSub(&a.refs[page], 1); });
    wait_stores_in_l2();
    __syncthreads();
  }
  if (again) {
    each([&](int e, int page) {
      if (holders(page) <= 0) atomicMin(&a.refs[page], kNamed + e);
    });
    wait_stores_in_l2();
    __syncthreads();
    int back = 0;
    each([&](int e, int page) { back += holders(page) == kNamed + e; });
    prefix(back, s_wave, total);
    total = min(total, room);
    for (int e0 = 0; e0 < entries; e0 += kThreads) {
      const int page = page_at(e0 + i);
      lay(page, page >= 0 && holders(page) == kNamed + e0 + i, total);
    }
    __syncthreads();
    each([&](int, int page) {
      if (holders(page) < 0) __hip_atomic_store(&a.refs[page], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    });
    __syncthreads();
  }
  for (int e = i; e < entries; e += kThreads) *entry(e) = -1;
  if (mine) a.length[s_row[i]] = 0;
  if (i == 0) {
    a.free_pages[0] = n_free + total;
    report(a, LLA_PAGES_OK, 0, total, n_free + total);
  }
}

// ---- whole pages ----

constexpr int kCopyThreads = 256;
typedef unsigned int Words4 __attribute__((ext_vector_type(4)));

// 768 pages of 524 KB (24 layers, 32 pairs, keys and values) in 80 us, 108 where the
// last-level cache holds others' lines (7.4 TB/s of reads and writes, 8 pages read by 4
// pairs each); one workgroup a page 180.  A workgroup copies kCopyBytes of one page of one layer (blockIdx.x: pair
// and piece of both pools' pages, blockIdx.y: layer).
constexpr int kCopyRun = 2, kCopyBytes = kCopyRun * kCopyThreads * 16;
__global__ __launch_bounds__(kCopyThreads) void copy_kernel(PageCopyArgs a, int pieces, int pieces_a) {
  const int i = blockIdx.x / pieces, piece = blockIdx.x - i * pieces;
  if (a.count && i >= *a.count) return;
  const int from = a.pairs[2 * i], to = a.pairs[2 * i + 1];
  if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages) return;
  const bool second = piece >= pieces_a;
  const int64_t bytes = a.bytes[second], at = (int64_t)(piece - (second ? pieces_a : 0)) * kCopyBytes;
  char* const pool = static_cast<char*>(a.pool[second]) + (int64_t)blockIdx.y * a.n_pages * bytes + at;
  const Words4* src = reinterpret_cast<const Words4*>(pool + from * bytes);
  Words4* dst = reinterpret_cast<Words4*>(pool + to * bytes);
  const int n = (int)min((int64_t)kCopyBytes, bytes - at) / 16;
  Words4 w[kCopyRun];
#pragma unroll
  for (int k = 0; k < kCopyRun; ++k) {
    const int e = threadIdx.x + k * kCopyThreads;
    if (e < n) w[k] = src[e];
  }
#pragma unroll
  for (int k = 0; k < kCopyRun; ++k) {
    const int e = threadIdx.x + k * kCopyThreads;
    if (e < n) __builtin_nontemporal_store(w[k], dst + e);
  }
}

// ---- tokens ----

// One workgroup per (sequence, destination page), key head and layer (blockIdx.z
// / 2), of the keys (blockIdx.z even) or the values.  Keys are whole rows; a
// value is one element of every feature row, so a wavefront collects the page's
// 64 tokens of a feature from the few lines that hold them and stores one.  Where
// few tokens are kept, the lines of values that they share with others bound it: a
// quarter of 8 x 4096 tokens of 16 heads of 128, bf16, reads nearly all of their
// 134 MB to move 34, and with the keys takes 54 us (190 MB fetched, 67 written: 4.8
// TB/s; heads side by side, so that pages that share lines meet in an L2, 54.4).
template <typename T>
__global__ __launch_bounds__(kCopyThreads) void gather_kernel(KvGatherArgs a, int blocks) {
  __shared__ int64_t s_from[kPage];  // element offset of the token's page and head, -1: none
  __shared__ int s_slot[kPage];
  const int j = blockIdx.x / blocks, pg = blockIdx.x % blocks, h = blockIdx.y, d = a.p.d, tid = threadIdx.x;
  const int n = a.n_keep ? max(0, min(a.n_keep[j], a.max_keep)) : a.max_keep;
  const int count = min(kPage, n - pg * kPage);
  const int src = a.src[j], dst = a.dst[j];
  if (count <= 0 || dst < 0 || dst >= a.p.n_seqs) return;
  const int page = a.p.table[(int64_t)dst * a.p.max_pages + pg];
  if (page < 0 || page >= a.p.n_pages) return;
  const int64_t layer = (int64_t)(blockIdx.z / 2) * a.p.n_pages, unit = (int64_t)kPage * d;
  if (tid < kPage) {
    int64_t from = -1;
    int slot = 0;
    if (tid < count && src >= 0 && src < a.p.n_seqs) {
      const int t = a.keep[(int64_t)j * a.max_keep + pg * kPage + tid];
      if (t >= 0 && t / kPage < a.p.max_pages) {
        const int f = a.p.table[(int64_t)src * a.p.max_pages + t / kPage];
        if (f >= 0 && f < a.p.n_pages) from = ((layer + f) * a.p.Hkv + h) * unit;
        slot = t % kPage;
      }
    }
    s_from[tid] = from;
    s_slot[tid] = slot;
  }
  __syncthreads();
  const int64_t at = ((layer + page) * a.p.Hkv + h) * unit;
  T none;
  store_out(&none, 0, __builtin_nanf(""));
  constexpr int kRun = 4;  // loads of a thread on their way
  if (blockIdx.z % 2 == 0) {
    constexpr int V = Elem<T>::kPer16B;
    T* const k = static_cast<T*>(a.p.k);
    const int chunks = d / V, all = count * chunks;
    for (int e0 = tid; e0 < all; e0 += kRun * kCopyThreads) {
      uint4 w[kRun];
#pragma unroll
      for (int x = 0; x < kRun; ++x) {
        const int e = min(e0 + x * kCopyThreads, all - 1), t = e / chunks, f = e - t * chunks;
        const int64_t from = s_from[t];
        w[x] = ld16(k + (from < 0 ? at : from + s_slot[t] * d) + f * V);
        if (from < 0) {
          const uint32_t u = sizeof(T) == 4 ? __float_as_uint(__builtin_nanf("")) : 0x7fc07fc0u;
          w[x] = uint4{u, u, u, u};
        }
      }
#pragma unroll
      for (int x = 0; x < kRun; ++x) {
        const int e = e0 + x * kCopyThreads;
        if (e < all)
          __builtin_nontemporal_store(__builtin_bit_cast(Words4, w[x]), reinterpret_cast<Words4*>(k + at + (int64_t)e * V));
      }
    }
    return;
  }
  T* const v = static_cast<T*>(a.p.v);
  const int t = tid % kPage;
  if (t >= count) return;
  const int64_t from = s_from[t];
  const T* in = v + (from < 0 ? at : from + s_slot[t]);
  T* out = v + at + t;
  constexpr int kWaves = kCopyThreads / kWave;
  for (int f0 = tid / kWave; f0 < d; f0 += kRun * kWaves) {
    T w[kRun];
#pragma unroll
    for (int x = 0; x < kRun; ++x) w[x] = in[min(f0 + x * kWaves, d - 1) * kPage];
#pragma unroll
    for (int x = 0; x < kRun; ++x) {
      const int f = f0 + x * kWaves;
      if (f < d) __builtin_nontemporal_store(from < 0 ? none : w[x], &out[f * kPage]);
    }
  }
}

}  // namespace

hipError_t launch_pages_reserve(const TableArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(reserve_kernel, dim3(1), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}
hipError_t launch_pages_fork(const TableArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(fork_kernel, dim3(1), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}
hipError_t launch_pages_free(const TableArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(free_kernel, dim3(1), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}
int64_t page_copy_pieces(int64_t a_bytes, int64_t b_bytes) {
  return (a_bytes + kCopyBytes - 1) / kCopyBytes + (b_bytes + kCopyBytes - 1) / kCopyBytes;
}
hipError_t launch_pages_copy(const PageCopyArgs& a, hipStream_t stream) {
  const int pieces = (int)page_copy_pieces(a.bytes[0], a.bytes[1]), first = (int)page_copy_pieces(a.bytes[0], 0);
  hipLaunchKernelGGL(copy_kernel, dim3((unsigned)a.n_pairs * pieces, a.layers), dim3(kCopyThreads), 0, stream, a, pieces,
                     first);
  return hipGetLastError();
}
hipError_t launch_kv_gather(const KvGatherArgs& a, hipStream_t stream) {
  const int blocks = (a.max_keep + kPage - 1) / kPage;
  const dim3 grid(a.B * blocks, a.p.Hkv, 2 * a.layers);
  if (a.p.dtype == LLA_BF16) hipLaunchKernelGGL(gather_kernel<bf16_t>, grid, dim3(kCopyThreads), 0, stream, a, blocks);
  else hipLaunchKernelGGL(gather_kernel<float>, grid, dim3(kCopyThreads), 0, stream, a, blocks);
  return hipGetLastError();
}

}  // namespace lla
