// Write of new tokens' keys and values into their sequences' pages, the keys
// turned to their positions on the way.
//
// Bound by memory: every element is read and written once.  Keys are rows of the
// page as they are rows of the input; values turn from token rows into the
// page's feature rows.

#include "kv_internal.h"
#include "rotary.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

constexpr int kThreads = 256;

// Where the tokens of entry b go: the first place, the position it is turned to, and
// how many there are.
struct Entry {
  int row, n;
  int64_t first, turned;
  __device__ __forceinline__ Entry(const KvWriteArgs& a, int b) {
    row = a.rows ? a.rows[b] : b;
    first = a.start[b];
    turned = a.pos ? a.pos[b] : first;
    n = a.n_new ? max(0, min(a.n_new[b], a.M)) : a.M;
    if (first < 0 || row < 0 || row >= a.p.n_seqs) n = 0;
  }
  // page number of the sequence's page `slot`, -1 where it has none
  __device__ __forceinline__ int page(const KvWriteArgs& a, int64_t slot) const {
    if (slot >= a.p.max_pages) return -1;
    const int p = a.p.table[(int64_t)row * a.p.max_pages + slot];
    return p < a.p.n_pages ? p : -1;
  }
};

// Few tokens: one thread per (token, head) and part of the key row or 8 value
// features (stored one by one: a token is one element of every feature row).
template <typename T, int N, bool Interleaved>
__global__ __launch_bounds__(kThreads) void write_few_kernel(KvWriteArgs a) {
  typedef Part<T, N, Interleaved> KeyPart;
  const int d = a.p.d, parts = KeyPart::count(a.rot, d - a.rot), units = parts + d / 8;
  const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t at = idx / units;  // (b, m, h)
  const int u = (int)(idx - at * units);
  if (at >= (int64_t)a.B * a.M * a.p.Hkv) return;
  const int h = (int)(at % a.p.Hkv), bm = (int)(at / a.p.Hkv), b = bm / a.M, m = bm - b * a.M;
  // the input is requested before the chain of entry, page and angle
  KeyPart p(u, a.rot, d);
  Run<T, 8> r;
  double freq[N];
  const bool key = u < parts;
  if (key) {
    p.load(static_cast<const T*>(a.k) + b * a.kb + m * a.km + (int64_t)h * d);
    if (p.turned) p.load_freq(freq, a.freq);
  } else {
    r = Run<T, 8>::load(static_cast<const T*>(a.v) + b * a.vb + m * a.vm + (int64_t)h * d + 8 * (u - parts));
  }
  const Entry e(a, b);
  if (m >= e.n) return;
  const int64_t pos = e.first + m;
  const int page = e.page(a, pos / kPage), t = (int)(pos % kPage);
  if (page < 0) return;
  const int64_t unit = ((int64_t)page * a.p.Hkv + h) * kPage * d;
  if (key) {
    Turn<N> turn;
    if (p.turned) turn.at((double)(e.turned + m), freq, a.magnitude, 1.f);
    p.turn(turn);
    p.store(static_cast<T*>(a.p.k) + unit + t * d);
  } else {
    T* vp = static_cast<T*>(a.p.v) + unit + t;
#pragma unroll
    for (int i = 0; i < 8; ++i) store_out(vp, (8 * (u - parts) + i) * kPage, r.get(i));
  }
}

// Prompts: a workgroup takes the tokens of one entry that fall into one page, for
// one key head, its keys or its values.  Values go through LDS, up to 128 features
// at a time, read there by columns, 16 bytes of a feature row at a time.  Small
// workgroups keep many loads in flight: prompts of 4001 to 2501 tokens, 16 heads of
// 128, not in a cache take 47 us (4.4 TB/s; a large copy runs at 5.0); a workgroup with
// one angle for 2, 4 or 16 heads takes 1, 5, 40 us more, plain stores 2.
template <typename T, int N, bool Interleaved>
__global__ __launch_bounds__(kThreads) void write_page_kernel(KvWriteArgs a, int blocks) {
  constexpr int V = Elem<T>::kPer16B, kCols = 128;
  // 16-byte chunk c of token t at chunk c ^ (t / V): runs of a column meet different banks
  __shared__ __align__(16) T s_v[kPage * kCols];
  auto at = [](int t, int f) { return t * kCols + (f / V ^ t / V) * V + f % V; };
  // heads side by side, as a token's rows are (52 -> 47 us against pages side by side)
  const int h = blockIdx.x % a.p.Hkv, wg = blockIdx.x / a.p.Hkv;
  const int b = wg / blocks, d = a.p.d, tid = threadIdx.x;
  const Entry e(a, b);
  const int64_t slot = e.first / kPage + wg % blocks;
  // tokens [m0, m1), at positions t0 .. t1 - 1 of the page
  const int64_t base = slot * kPage - e.first;
  const int m0 = (int)max((int64_t)0, base), m1 = (int)min((int64_t)e.n, base + kPage);
  if (m0 >= m1) return;
  const int page = e.page(a, slot);  // (needed by the stores: the rows are requested beside it)
  const int t0 = (int)(m0 - base), t1 = t0 + (m1 - m0), count = m1 - m0;
  const int64_t unit = ((int64_t)page * a.p.Hkv + h) * kPage * d;

  if (blockIdx.y == 0) {
    const T* k = static_cast<const T*>(a.k) + b * a.kb + m0 * a.km + (int64_t)h * d;
    T* kp = static_cast<T*>(a.p.k) + unit + t0 * d;
    const int parts = Part<T, N, Interleaved>::count(a.rot, d - a.rot);
    for (int x = tid; x < count * parts; x += kThreads) {
      const int i = x / parts;
      Part<T, N, Interleaved> p(x - i * parts, a.rot, d);
      p.load(k + i * a.km);
      Turn<N> t;
      if (p.turned) {
        double freq[N];
        p.load_freq(freq, a.freq);
        t.at((double)(e.turned + m0 + i), freq, a.magnitude, 1.f);
      }
      p.turn(t);
      if (page >= 0) p.store_past(kp + i * d);
    }
    return;
  }

  for (int f0 = 0; f0 < d; f0 += kCols) {
    const int cols = min(kCols, d - f0), chunks = cols / V;
    const T* v = static_cast<const T*>(a.v) + b * a.vb + m0 * a.vm + (int64_t)h * d + f0;
    T* vp = static_cast<T*>(a.p.v) + unit + f0 * kPage;
    if (f0) __syncthreads();
    for (int x = tid; x < count * chunks; x += kThreads) {
      const int i = x / chunks, f = x - i * chunks;
      *reinterpret_cast<uint4*>(s_v + at(t0 + i, f * V)) = ld16(v + i * a.vm + f * V);
    }
    __syncthreads();
    if (page < 0) return;
    // 64 / V runs of a feature row side by side, so a row's lines are written together
    constexpr int kRuns = kPage / V;
    for (int x = tid; x < cols * kRuns; x += kThreads) {
      const int f = x / kRuns, t = (x - f * kRuns) * V;
      if (t + V <= t0 || t >= t1) continue;
      if (t >= t0 && t + V <= t1) {
        Run<T, V> r;
#pragma unroll
        for (int i = 0; i < V; ++i) {
          if constexpr (sizeof(T) == 4) r.w[i] = __float_as_uint(s_v[at(t + i, f)]);
          else if (i % 2 == 0) r.w[i / 2] = s_v[at(t + i, f)] | (uint32_t(s_v[at(t + i + 1, f)]) << 16);
        }
        r.store_past(vp + f * kPage + t);
      } else {
        for (int i = max(t, t0); i < min(t + V, t1); ++i) vp[f * kPage + i] = s_v[at(i, f)];
      }
    }
  }
}

// From kPaged tokens an entry the page kernel is the faster one (32 entries, 16 heads of 128,
// bf16, few / page: 2 tokens 6.0 / 6.5 us, 4 6.9 / 6.7, 8 9.6 / 6.2, 15 12.3 / 9.4).
constexpr int kPaged = 4;

template <typename T, int N, bool Interleaved>
hipError_t launch(const KvWriteArgs& a, hipStream_t stream) {
  const int d = a.p.d;
  if (a.M < kPaged) {
    const int units = Part<T, N, Interleaved>::count(a.rot, d - a.rot) + d / 8;
    const int64_t runs = (int64_t)a.B * a.M * a.p.Hkv * units;
    hipLaunchKernelGGL((write_few_kernel<T, N, Interleaved>), dim3((unsigned)((runs + kThreads - 1) / kThreads)),
                       dim3(kThreads), 0, stream, a);
    return hipGetLastError();
  }
  const int blocks = (a.M + 2 * kPage - 2) / kPage;  // pages that M positions can touch
  hipLaunchKernelGGL((write_page_kernel<T, N, Interleaved>), dim3((unsigned)a.B * blocks * a.p.Hkv, 2), dim3(kThreads), 0, stream, a,
                     blocks);
  return hipGetLastError();
}

template <typename T, bool Interleaved>
hipError_t launch(const KvWriteArgs& a, hipStream_t stream) {
  if constexpr (sizeof(T) == 2) {
    if (a.rot % 16 == 0) return launch<T, 8, Interleaved>(a, stream);
  }
  return launch<T, 4, Interleaved>(a, stream);
}

}  // namespace

hipError_t launch_kv_write(const KvWriteArgs& a, hipStream_t stream) {
  if (a.p.dtype == LLA_BF16) return a.interleaved ? launch<bf16_t, true>(a, stream) : launch<bf16_t, false>(a, stream);
  return a.interleaved ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
}

}  // namespace lla
