// Write of new tokens' keys and values into their sequences' pages, the keys
// turned to their positions on the way.
//
// A workgroup takes the new tokens of one entry that fall into one page, for
// one key head.  Keys are rows of the page as they are rows of the input; values
// turn from token rows into the page's feature rows.

#include "kv_internal.h"
#include "rotary.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

constexpr int kThreads = 256;

template <typename T, bool Interleaved>
__global__ __launch_bounds__(kThreads) void write_kernel(KvWriteArgs a, int blocks) {
  const int b = blockIdx.x / blocks, h = blockIdx.y, d = a.p.d, tid = threadIdx.x;
  const int row = a.rows ? a.rows[b] : b;
  const int64_t first = a.start[b];
  if (first < 0 || row < 0 || row >= a.p.n_seqs) return;
  const int n = a.n_new ? max(0, min(a.n_new[b], a.M)) : a.M;
  const int64_t slot = first / kPage + blockIdx.x % blocks;  // page of the sequence
  if (slot >= a.p.max_pages) return;
  // tokens [m0, m1) at positions t0 .. of the page
  const int64_t base = slot * kPage - first;
  const int m0 = (int)max((int64_t)0, base), m1 = (int)min((int64_t)n, base + kPage);
  if (m0 >= m1) return;
  const int t0 = (int)(m0 - base);
  const int page = a.p.table[(int64_t)row * a.p.max_pages + slot];
  if (page < 0 || page >= a.p.n_pages) return;
  const int64_t at = ((int64_t)page * a.p.Hkv + h) * kPage * d;
  T* kp = static_cast<T*>(a.p.k) + at;
  T* vp = static_cast<T*>(a.p.v) + at;
  const T* k = static_cast<const T*>(a.k) + b * a.kb + (int64_t)h * d;
  const T* v = static_cast<const T*>(a.v) + b * a.vb + (int64_t)h * d;
  const int half = a.rot / 2, turned = half / 4, units = turned + (d - a.rot) / 8;
  for (int e = tid; e < (m1 - m0) * units; e += kThreads) {
    const int i = e / units, u = e - i * units, m = m0 + i;
    const T* x = k + m * a.km;
    T* y = kp + (t0 + i) * d;
    if (u < turned) {
      Turn<4> t;
      t.at((double)(first + m), a.freq + 4 * u, a.magnitude, 1.f);
      Pairs<T, 4, Interleaved> p;
      p.load(x, 4 * u, half);
      p.turn(t);
      p.store(y, 4 * u, half);
    } else {
      const int f = a.rot + 8 * (u - turned);
      Run<T, 8>::load(x + f).store(y + f);
    }
  }
  for (int e = tid; e < kPage * d; e += kThreads) {
    const int f = e / kPage, t = e - f * kPage, m = m0 + t - t0;
    if (m >= m0 && m < m1) vp[e] = v[m * a.vm + f];
  }
}

}  // namespace

hipError_t launch_kv_write(const KvWriteArgs& a, hipStream_t stream) {
  const int blocks = (a.M + 2 * kPage - 2) / kPage;  // pages that M positions can touch
  const dim3 grid(a.B * blocks, a.p.Hkv);
  if (a.p.dtype == LLA_BF16) {
    if (a.interleaved) hipLaunchKernelGGL((write_kernel<bf16_t, true>), grid, dim3(kThreads), 0, stream, a, blocks);
    else hipLaunchKernelGGL((write_kernel<bf16_t, false>), grid, dim3(kThreads), 0, stream, a, blocks);
  } else {
    if (a.interleaved) hipLaunchKernelGGL((write_kernel<float, true>), grid, dim3(kThreads), 0, stream, a, blocks);
    else hipLaunchKernelGGL((write_kernel<float, false>), grid, dim3(kThreads), 0, stream, a, blocks);
  }
  return hipGetLastError();
}

}  // namespace lla
