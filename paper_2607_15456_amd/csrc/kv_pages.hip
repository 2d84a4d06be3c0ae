// Bookkeeping of the paged K/V cache on the device: room for new tokens with
// copy on write, sharing, freeing, and the copies of pages and tokens.
//
// The three table calls each run in one workgroup of up to 1024 sequences: the
// rows' needs are a prefix sum, so the outcome is that of one row after another
// in any run, with no lock and no order of atomics that shows.  They move a few
// words a page; what they cost is a launch and a chain of dependent loads.

#include "kv_internal.h"
#include "lla_device.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

constexpr int kRows = LLA_KV_MAX_ROWS, kThreads = 1024;

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
__device__ __forceinline__ bool sound(const int* s_row, int n, int i, int n_seqs) {
  const int r = s_row[i];
  bool ok = r >= 0 && r < n_seqs;
  for (int j = 0; j < i; ++j) ok &= s_row[j] != r;
  return ok;
}

__device__ __forceinline__ void report(const TableArgs& a, int status, int pairs, int pages, int left) {
  a.result[0] = status;
  a.result[1] = pairs;
  a.result[2] = pages;
  a.result[3] = left;
}

__global__ __launch_bounds__(kThreads) void reserve_kernel(TableArgs a) {
  __shared__ int s_row[kRows], s_open[kRows], s_wave[kThreads / kWave];
  const int i = threadIdx.x;
  const bool mine = i < a.n;
  s_row[i] = mine ? a.rows[i] : -1;
  __syncthreads();
  bool ok = !mine || sound(s_row, a.n, i, a.n_seqs);
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
    if (mine) a.start[i] = -1;
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
    if (mine) a.start[i] = -1;
    if (i == 0) report(a, LLA_PAGES_FULL, 0, 0, n_free);
    return;
  }
  if (row >= 0) {
    for (int k = 0; k < need; ++k) {
      const int page = a.free_pages[n_free - (at + k)];
      table[have + k] = page;
      if (page >= 0 && page < a.n_pages) a.refs[page] = 1;
    }
    if (copy) {
      atomicSub(&a.refs[open], 1);
      a.pairs[2 * pair] = open;
      a.pairs[2 * pair + 1] = table[have];
    }
    a.start[i] = len;
    a.length[row] = (int)end;
  }
  __syncthreads();
  if (i == 0) {
    a.free_pages[0] = n_free - total;
    report(a, LLA_PAGES_OK, pairs, total, n_free - total);
  }
}

__global__ __launch_bounds__(kThreads) void fork_kernel(TableArgs a) {
  __shared__ int s_row[kRows];
  const int i = threadIdx.x;
  const bool mine = i < a.n;
  s_row[i] = mine ? a.rows[i] : -1;
  __syncthreads();
  bool ok = true;
  int src = -1;
  if (mine) {
    src = a.more[i];
    ok = sound(s_row, a.n, i, a.n_seqs) && src >= 0 && src < a.n_seqs;
    for (int j = 0; j < a.n; ++j) ok &= s_row[j] != src;
    if (ok) ok = a.length[s_row[i]] == 0 && a.length[src] >= 0 && a.length[src] <= (int64_t)a.max_pages * kPage;
  }
  if (!__syncthreads_and(ok)) {
    if (i == 0) report(a, LLA_PAGES_BAD, 0, 0, a.free_pages[0]);
    return;
  }
  if (mine) {
    const int len = a.length[src];
    const int32_t* from = a.table + (int64_t)src * a.max_pages;
    int32_t* to = a.table + (int64_t)s_row[i] * a.max_pages;
    for (int k = 0; k < pages_of(len); ++k) {
      const int page = from[k];
      to[k] = page;
      if (page >= 0 && page < a.n_pages) atomicAdd(&a.refs[page], 1);
    }
    a.length[s_row[i]] = len;
  }
  if (i == 0) report(a, LLA_PAGES_OK, 0, 0, a.free_pages[0]);
}

// Freeing in three steps over all (row, page) entries: holders are counted
// down; of the entries whose page has none left, the first names it (its rank,
// lowered by 2^31, is the least that lands in refs); the named pages are laid
// onto the stack, the last first.
__global__ __launch_bounds__(kThreads) void free_kernel(TableArgs a) {
  __shared__ int s_row[kRows], s_at[kRows], s_wave[kThreads / kWave];
  const int i = threadIdx.x;
  const bool mine = i < a.n;
  s_row[i] = mine ? a.rows[i] : -1;
  __syncthreads();
  bool ok = true;
  int len = 0;
  const int n_free = a.free_pages[0];
  if (mine) {
    ok = sound(s_row, a.n, i, a.n_seqs);
    if (ok) len = a.length[s_row[i]];
    ok = ok && len >= 0 && len <= (int64_t)a.max_pages * kPage;
  }
  ok = ok && n_free >= 0 && n_free <= a.n_pages;
  if (!__syncthreads_and(ok)) {
    if (i == 0) report(a, LLA_PAGES_BAD, 0, 0, n_free);
    return;
  }
  int entries;
  s_at[i] = prefix(mine ? pages_of(len) : 0, s_wave, entries);
  __syncthreads();
  // entry e of all: its row (the last whose first entry is at or before e) and page
  auto entry = [&](int e) -> int32_t* {
    int lo = 0, hi = a.n - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (s_at[mid] <= e) lo = mid;
      else hi = mid - 1;
    }
    return a.table + (int64_t)s_row[lo] * a.max_pages + (e - s_at[lo]);
  };
  auto page_at = [&](int e) {
    const int page = *entry(e);
    return page >= 0 && page < a.n_pages ? page : -1;
  };
  for (int e = i; e < entries; e += kThreads) {
    const int page = page_at(e);
    if (page >= 0) atomicSub(&a.refs[page], 1);
  }
  wait_stores_in_l2();
  __syncthreads();
  constexpr int kNamed = (int)0x80000000;
  for (int e = i; e < entries; e += kThreads) {
    const int page = page_at(e);
    if (page >= 0 && __hip_atomic_load(&a.refs[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) <= 0)
      atomicMin(&a.refs[page], kNamed + e);
  }
  wait_stores_in_l2();
  __syncthreads();
  int back = 0;  // pages given back by earlier rounds
  for (int e0 = 0; e0 < entries; e0 += kThreads) {
    const int e = e0 + i;
    const int page = e < entries ? page_at(e) : -1;
    const bool named =
        page >= 0 && __hip_atomic_load(&a.refs[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == kNamed + e;
    int round;
    const int at = back + prefix(named ? 1 : 0, s_wave, round);
    (void)at;
    back += round;
  }
  const int total = min(back, a.n_pages - n_free);
  int done = 0;
  for (int e0 = 0; e0 < entries; e0 += kThreads) {
    const int e = e0 + i;
    const int page = e < entries ? page_at(e) : -1;
    const bool named =
        page >= 0 && __hip_atomic_load(&a.refs[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == kNamed + e;
    int round;
    const int at = done + prefix(named ? 1 : 0, s_wave, round);
    if (named && at < total) a.free_pages[n_free + total - at] = page;
    done += round;
  }
  __syncthreads();
  for (int e = i; e < entries; e += kThreads) {
    const int page = page_at(e);
    if (page >= 0 && __hip_atomic_load(&a.refs[page], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < 0)
      __hip_atomic_store(&a.refs[page], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  for (int e = i; e < entries; e += kThreads) *entry(e) = -1;
  if (mine) a.length[s_row[i]] = 0;
  if (i == 0) {
    a.free_pages[0] = n_free + total;
    report(a, LLA_PAGES_OK, 0, total, n_free + total);
  }
}

// ---- whole pages ----

constexpr int kCopyThreads = 256;

__global__ __launch_bounds__(kCopyThreads) void copy_kernel(PageCopyArgs a) {
  const int i = blockIdx.x;
  if (a.count && i >= *a.count) return;
  const int from = a.pairs[2 * i], to = a.pairs[2 * i + 1];
  if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages) return;
  for (int x = 0; x < 2; ++x) {
    char* const pool = static_cast<char*>(a.pool[x]) + (int64_t)blockIdx.y * a.n_pages * a.bytes[x];
    const uint4* src = reinterpret_cast<const uint4*>(pool + from * a.bytes[x]);
    uint4* dst = reinterpret_cast<uint4*>(pool + to * a.bytes[x]);
    for (int64_t e = threadIdx.x; e < a.bytes[x] / 16; e += kCopyThreads) dst[e] = src[e];
  }
}

// ---- tokens ----

// One workgroup per (sequence, destination page), key head and layer.
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
  const int64_t layer = (int64_t)blockIdx.z * a.p.n_pages, unit = (int64_t)kPage * d;
  T* k = static_cast<T*>(a.p.k);
  T* v = static_cast<T*>(a.p.v);
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
  for (int e = tid; e < count * d; e += kCopyThreads) {
    const int t = e / d, f = e - t * d;
    k[at + e] = s_from[t] < 0 ? none : k[s_from[t] + s_slot[t] * d + f];
  }
  for (int e = tid; e < kPage * d; e += kCopyThreads) {
    const int f = e / kPage, t = e - f * kPage;
    if (t < count) v[at + e] = s_from[t] < 0 ? none : v[s_from[t] + f * kPage + s_slot[t]];
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
hipError_t launch_pages_copy(const PageCopyArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(copy_kernel, dim3(a.n_pairs, a.layers), dim3(kCopyThreads), 0, stream, a);
  return hipGetLastError();
}
hipError_t launch_kv_gather(const KvGatherArgs& a, hipStream_t stream) {
  const int blocks = (a.max_keep + kPage - 1) / kPage;
  const dim3 grid(a.B * blocks, a.p.Hkv, a.layers);
  if (a.p.dtype == LLA_BF16) hipLaunchKernelGGL(gather_kernel<bf16_t>, grid, dim3(kCopyThreads), 0, stream, a, blocks);
  else hipLaunchKernelGGL(gather_kernel<float>, grid, dim3(kCopyThreads), 0, stream, a, blocks);
  return hipGetLastError();
}

}  // namespace lla
