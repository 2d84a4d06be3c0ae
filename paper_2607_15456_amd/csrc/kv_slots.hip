// Packed batches over the paged K/V cache: from request lengths to offsets, positions
// and slots, which neighbours share leading pages, and the write of packed keys and
// values to their slots.
//
// The maps are a few words a token, so a launch and a chain of dependent reads bound
// them: lengths, a prefix sum, the entry's start and row, its page.  Every workgroup
// sums all lengths for itself, so one launch does.

#include "kv_internal.h"
#include "kv_tile.h"
#include "rotary.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

constexpr int kThreads = 256;

// ---- offsets, entries, positions, slots ----

__global__ __launch_bounds__(kThreads) void slots_kernel(KvSlotsArgs a) {
  constexpr int kEach = kMostEntries / kThreads;
  __shared__ int s_off[kMostEntries + 1];
  __shared__ int s_wave[kThreads / kWave];
  const int tid = threadIdx.x;
  int n[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = tid * kEach + i;
    n[i] = b < a.B ? max(0, min(a.n_new[b], a.total)) : 0;  // (a length past the room ends there)
    sum += n[i];
  }
  int at = prefix_sum<kThreads>(sum, s_wave);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int b = tid * kEach + i;
    if (b < a.B) s_off[b] = min(at, a.total);
    at = add_up(at, n[i]);
    if (b == a.B - 1) s_off[a.B] = min(at, a.total);
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int b = tid; b <= a.B; b += kThreads) a.offset[b] = s_off[b];
  const int t = blockIdx.x * kThreads + tid;
  if (t >= a.total) return;
  int entry = -1, pos = -1;
  int64_t slot = -1;
  if (t < s_off[a.B]) {
    entry = last_at_most(s_off, a.B, t);
    const int i = t - s_off[entry], start = a.start[entry], row = a.rows ? a.rows[entry] : entry;
    const int64_t place = start < 0 ? -1 : (int64_t)start + i;
    const int64_t turned = a.pos0 ? (int64_t)a.pos0[entry] + i : place;
    if (place >= 0 && turned >= 0 && turned <= 0x7fffffff) pos = (int)turned;
    if (place >= 0 && row >= 0 && row < a.n_seqs && place < (int64_t)a.max_pages * kPage) {
      const int page = a.table[(int64_t)row * a.max_pages + place / kPage];
      if (page >= 0 && page < a.n_pages) slot = (int64_t)page * kPage + place % kPage;
    }
  }
  a.entry[t] = entry;
  a.pos[t] = pos;
  a.slot[t] = slot;
}

// ---- shared leading pages ----

// Places that a sequence holds, 0 where it is none.
__device__ __forceinline__ int held(const PagesSharedArgs& a, int b, int& row) {
  row = a.rows ? a.rows[b] : b;
  if (row < 0 || row >= a.n_seqs) return 0;
  return (int)max((int64_t)0, min((int64_t)a.length[row], (int64_t)a.max_pages * kPage));
}

// Places at which entry b > 0 and the one before it read the same pages, by a wavefront.
__device__ __forceinline__ int common(const PagesSharedArgs& a, int b) {
  const int lane = threadIdx.x % kWave;
  int row, other;
  const int n = held(a, b, row), most = min(n, held(a, b - 1, other)), pages = (most + kPage - 1) / kPage;
  if (row == other) return most;
  const int32_t* x = a.table + (int64_t)row * a.max_pages;
  const int32_t* y = a.table + (int64_t)other * a.max_pages;
  int same = pages;
  for (int p0 = 0; p0 < pages; p0 += kWave) {
    const int p = p0 + lane, page = p < pages ? x[p] : -1;
    const bool off = p < pages && (page != y[p] || page < 0 || page >= a.n_pages);
    const uint64_t stop = __ballot(off);
    if (stop) {
      same = p0 + __builtin_ctzll(stop);
      break;
    }
  }
  return min(most, same * kPage);
}

constexpr int kGroupThreads = 1024, kAlone = 64;  // entries up to which one workgroup does both parts

__global__ __launch_bounds__(kWave) void common_kernel(PagesSharedArgs a) {
  const int b = blockIdx.x, n = b ? common(a, b) : 0;
  if (threadIdx.x == 0) a.shared[b] = n;
}

// Runs of entries that have enough in common with the one before, and the least of a run.
template <bool All>
__global__ __launch_bounds__(kGroupThreads) void groups_kernel(PagesSharedArgs a) {
  constexpr int kWaves = kGroupThreads / kWave;
  __shared__ int s_common[kMostEntries], s_least[kMostEntries], s_wave[kWaves], s_start[kMostEntries];
  const int b = threadIdx.x;
  if constexpr (All) {
    for (int x = threadIdx.x / kWave; x < a.B; x += kWaves) {
      const int n = x ? common(a, x) : 0;
      if (threadIdx.x % kWave == 0) s_common[x] = n;
    }
  } else if (b < a.B) {
    s_common[b] = a.shared[b];
  }
  s_least[b] = 0x7fffffff;
  __syncthreads();
  const bool joined = b < a.B && s_common[b] > 0 && s_common[b] >= a.least;
  const int run = prefix_sum<kGroupThreads>(b < a.B && !joined ? 1 : 0, s_wave) + (joined ? 0 : 1) - 1;
  if (b < a.B && !joined) s_start[run] = b;
  if (joined) atomicMin(&s_least[run], s_common[b]);
  __syncthreads();
  if (b < a.B) {
    a.lead[b] = s_start[run];
    a.shared[b] = s_least[run] == 0x7fffffff ? 0 : s_least[run];
  }
}

// ---- packed keys and values to their slots ----

constexpr int kTokens = 64, kCols = 128;

// 64 packed tokens of one key head, its keys or its values.  Values go through LDS: a
// token is one element of every feature row, and neighbouring tokens mostly neighbours there.
template <typename T, int N, bool Interleaved>
__global__ __launch_bounds__(kThreads) void write_slots_kernel(KvWriteSlotsArgs a) {
  constexpr int kWords = kCols * (int)sizeof(T) / 4 + 1;  // of a staged row: columns meet different banks
  __shared__ uint32_t s_v[kTokens * kWords];
  const int h = blockIdx.x % a.p.Hkv, t0 = blockIdx.x / a.p.Hkv * kTokens, d = a.p.d, tid = threadIdx.x;
  const int count = min(kTokens, a.total - t0);
  const int64_t places = (int64_t)a.p.n_pages * kPage;
  // where slot s of the head's unit is, in elements of a page row
  auto unit = [&](int64_t s) { return ((s / kPage) * a.p.Hkv + h) * (int64_t)kPage * d; };
  if (blockIdx.y == 0) {
    const T* k = static_cast<const T*>(a.k) + t0 * a.kt + (int64_t)h * d;
    const int parts = Part<T, N, Interleaved>::count(a.rot, d - a.rot);
    for (int x = tid; x < count * parts; x += kThreads) {
      const int i = x / parts;
      Part<T, N, Interleaved> p(x - i * parts, a.rot, d);
      p.load(k + i * a.kt);
      const int64_t s = a.slot[t0 + i];
      Turn<N> t;
      if (p.turned) {
        double freq[N];
        p.load_freq(freq, a.freq);
        t.at((double)a.pos[t0 + i], freq, a.magnitude, 1.f);
      }
      p.turn(t);
      if (s >= 0 && s < places) p.store(static_cast<T*>(a.p.k) + unit(s) + s % kPage * d);
    }
    return;
  }
  const int lane = tid % kWave, w = tid / kWave;
  const int64_t s = lane < count ? a.slot[t0 + lane] : -1;
  T* const to = s >= 0 && s < places ? static_cast<T*>(a.p.v) + unit(s) + s % kPage : nullptr;
  for (int f0 = 0; f0 < d; f0 += kCols) {
    constexpr int V = Elem<T>::kPer16B;
    const int cols = min(kCols, d - f0), chunks = cols / V;
    const T* v = static_cast<const T*>(a.v) + t0 * a.vt + (int64_t)h * d + f0;
    if (f0) __syncthreads();
    for (int x = tid; x < count * chunks; x += kThreads) {
      const int i = x / chunks, c = x - i * chunks;
      const uint4 y = ld16(v + i * a.vt + c * V);
      uint32_t* p = s_v + i * kWords + c * 4;
      p[0] = y.x, p[1] = y.y, p[2] = y.z, p[3] = y.w;
    }
    __syncthreads();
    if (to) {
      for (int f = w; f < cols; f += kThreads / kWave)
        to[(int64_t)(f0 + f) * kPage] = reinterpret_cast<const T*>(s_v + lane * kWords)[f];
    }
  }
}

template <typename T, int N, bool Interleaved>
hipError_t launch(const KvWriteSlotsArgs& a, hipStream_t stream) {
  const unsigned blocks = (unsigned)((a.total + kTokens - 1) / kTokens) * a.p.Hkv;
  hipLaunchKernelGGL((write_slots_kernel<T, N, Interleaved>), dim3(blocks, 2), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}
template <typename T, bool Interleaved>
hipError_t launch(const KvWriteSlotsArgs& a, hipStream_t stream) {
  if constexpr (sizeof(T) == 2) {
    if (a.rot % 16 == 0) return launch<T, 8, Interleaved>(a, stream);
  }
  return launch<T, 4, Interleaved>(a, stream);
}

}  // namespace

hipError_t launch_kv_slots(const KvSlotsArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(slots_kernel, dim3((unsigned)((a.total + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_pages_shared(const PagesSharedArgs& a, hipStream_t stream) {
  if (a.B <= kAlone) {
    hipLaunchKernelGGL(groups_kernel<true>, dim3(1), dim3(kGroupThreads), 0, stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(common_kernel, dim3(a.B), dim3(kWave), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(groups_kernel<false>, dim3(1), dim3(kGroupThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_kv_write_slots(const KvWriteSlotsArgs& a, hipStream_t stream) {
  if (a.p.dtype == LLA_BF16) return a.interleaved ? launch<bf16_t, true>(a, stream) : launch<bf16_t, false>(a, stream);
  return a.interleaved ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
}

}  // namespace lla
