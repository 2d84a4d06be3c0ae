// Rotary positions of query or key rows in either pairing, over part of the
// head, with given frequencies; with the sign of the angle turned, the
// transposed rotation of a backward pass.
//
//   y[pair i] = magnitude * R(p * freq[i]) x[pair i],   y[rest] = x[rest]
//
// Bound by memory: 6 flops a pair against 8 bytes in bf16.

#include "kv_internal.h"
#include "rotary.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ int64_t position(const RotaryArgs& a, int b, int m) {
  if (!a.pos) return (int64_t)a.pos0 + m;
  if (a.pos_tokens) return (int64_t)a.pos[(int64_t)b * a.M + m] + a.pos0;
  return (int64_t)a.pos[b] + a.pos0 + m;
}

// One thread per (token, part of its rows) and chunk of heads (blockIdx.y).
template <typename T, int N, bool Interleaved>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, int parts, int heads_per) {
  const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t tok = idx / parts;
  if (tok >= (int64_t)a.B * a.M) return;
  const int b = (int)(tok / a.M), m = (int)(tok - (int64_t)b * a.M);
  const int h0 = blockIdx.y * heads_per, h1 = min(a.H, h0 + heads_per);
  const T* x = static_cast<const T*>(a.x) + b * a.xb + m * a.xm;
  T* y = static_cast<T*>(a.y) + b * a.yb + m * a.ym;
  Part<T, N, Interleaved> p((int)(idx - tok * parts), a.rot, a.d);
  p.load(x + h0 * a.xh);  // on its way while the angle is formed
  Turn<N> t;
  if (p.turned) {
    double freq[N];
    p.load_freq(freq, a.freq);
    t.at((double)position(a, b, m), freq, a.magnitude, a.sign);
  }
  for (int h = h0;;) {
    p.turn(t);
    p.store(y + h * a.yh);
    if (++h >= h1) break;
    p.load(x + h * a.xh);
  }
}

// Few rows get a thread for each head, so that they spread over the device; from
// kMany runs on a thread turns kHeads heads with one angle.  4 x 8192 tokens of 16
// heads of 128, bf16, not in a cache: one head 71 us, two 50, four 50 (5.2 TB/s; a
// large copy runs at 5.0), four with two or four of them loaded together 51, 52,
// non-temporal stores 69; 3 x 1501 tokens of 16 heads of 96, fp32, 64 turned: one 13.8,
// four 15.3.
constexpr int64_t kMany = 1 << 21;
constexpr int kHeads = 4;

template <typename T, int N, bool Interleaved>
hipError_t launch(const RotaryArgs& a, hipStream_t stream) {
  const int parts = Part<T, N, Interleaved>::count(a.rot, a.x == a.y ? 0 : a.d - a.rot);
  const int64_t runs = (int64_t)a.B * a.M * parts;
  const int heads_per = runs * a.H < kMany ? 1 : kHeads;
  hipLaunchKernelGGL((rotary_kernel<T, N, Interleaved>),
                     dim3((unsigned)((runs + kThreads - 1) / kThreads), (a.H + heads_per - 1) / heads_per), dim3(kThreads), 0,
                     stream, a, parts, heads_per);
  return hipGetLastError();
}

template <typename T, bool Interleaved>
hipError_t launch(const RotaryArgs& a, hipStream_t stream) {
  // pairs of a thread: 16 bytes of each half of a bf16 row where rot/2 allows it
  if (sizeof(T) == 2 && a.rot % 16 == 0) return launch<T, 8, Interleaved>(a, stream);
  return launch<T, 4, Interleaved>(a, stream);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  if (a.dtype == LLA_BF16) return a.interleaved ? launch<bf16_t, true>(a, stream) : launch<bf16_t, false>(a, stream);
  return a.interleaved ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
}

}  // namespace lla
