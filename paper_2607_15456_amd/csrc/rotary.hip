// Rotary positions of query or key rows in either pairing, over part of the
// head, with given frequencies; with the sign of the angle turned, the
// transposed rotation of a backward pass.
//
//   y[pair i] = magnitude * R(p * freq[i]) x[pair i],   y[rest] = x[rest]
//
// Memory-bound: 6 flops a pair against 8 bytes in bf16.

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

// One thread per (token, run of N pairs or of 2N copied features) and chunk of
// heads (blockIdx.y).
template <typename T, int N, bool Interleaved>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, int units, int heads_per) {
  const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t tok = idx / units;
  if (tok >= (int64_t)a.B * a.M) return;
  const int u = (int)(idx - tok * units);
  const int b = (int)(tok / a.M), m = (int)(tok - (int64_t)b * a.M);
  const int h0 = blockIdx.y * heads_per, h1 = min(a.H, h0 + heads_per);
  const T* x = static_cast<const T*>(a.x) + b * a.xb + m * a.xm + h0 * a.xh;
  T* y = static_cast<T*>(a.y) + b * a.yb + m * a.ym + h0 * a.yh;
  const int half = a.rot / 2, turned = half / N;
  if (u < turned) {
    Turn<N> t;
    t.at((double)position(a, b, m), a.freq + u * N, a.magnitude, a.sign);
    for (int h = h0; h < h1; ++h, x += a.xh, y += a.yh) {
      Pairs<T, N, Interleaved> p;
      p.load(x, u * N, half);
      p.turn(t);
      p.store(y, u * N, half);
    }
  } else {
    const int f = a.rot + 8 * (u - turned);  // copied features, 8 a thread
    for (int h = h0; h < h1; ++h, x += a.xh, y += a.yh) Run<T, 8>::load(x + f).store(y + f);
  }
}

template <typename T, int N, bool Interleaved>
hipError_t launch(const RotaryArgs& a, hipStream_t stream) {
  const bool in_place = a.x == a.y;
  const int units = a.rot / 2 / N + (in_place ? 0 : (a.d - a.rot) / 8);
  const int64_t blocks = ((int64_t)a.B * a.M * units + kThreads - 1) / kThreads;
  const int heads_per = a.H;
  hipLaunchKernelGGL((rotary_kernel<T, N, Interleaved>), dim3((unsigned)blocks, (a.H + heads_per - 1) / heads_per),
                     dim3(kThreads), 0, stream, a, units, heads_per);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  if (a.dtype == LLA_BF16) {
    return a.interleaved ? launch<bf16_t, 4, true>(a, stream) : launch<bf16_t, 4, false>(a, stream);
  }
  return a.interleaved ? launch<float, 4, true>(a, stream) : launch<float, 4, false>(a, stream);
}

}  // namespace lla
