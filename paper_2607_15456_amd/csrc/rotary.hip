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

// One thread per (token, run of N pairs or of 8 copied features) and chunk of
// heads (blockIdx.y), HU heads' rows in flight at a time: their loads are issued
// before any store (y may be x), the first ones before the angle is formed.
template <typename T, int N, bool Interleaved, int HU>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, int units, int heads_per) {
  const int64_t idx = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t tok = idx / units;
  if (tok >= (int64_t)a.B * a.M) return;
  const int u = (int)(idx - tok * units);
  const int b = (int)(tok / a.M), m = (int)(tok - (int64_t)b * a.M);
  const int h0 = blockIdx.y * heads_per, h1 = min(a.H, h0 + heads_per);
  const T* x = static_cast<const T*>(a.x) + b * a.xb + m * a.xm;
  T* y = static_cast<T*>(a.y) + b * a.yb + m * a.ym;
  const int half = a.rot / 2, turned = half / N;
  if (u < turned) {
    Turn<N> t;
    for (int h = h0; h < h1; h += HU) {
      Pairs<T, N, Interleaved> p[HU];
#pragma unroll
      for (int k = 0; k < HU; ++k) p[k].load(x + min(h + k, h1 - 1) * a.xh, u * N, half);
      if (h == h0) {
        double freq[N];
        load_freq(freq, a.freq + u * N);
        t.at((double)position(a, b, m), freq, a.magnitude, a.sign);
      }
#pragma unroll
      for (int k = 0; k < HU; ++k) {
        p[k].turn(t);
        if (h + k < h1) p[k].store(y + (h + k) * a.yh, u * N, half);
      }
    }
  } else {
    const int f = a.rot + 8 * (u - turned);
    for (int h = h0; h < h1; h += HU) {
      Run<T, 8> p[HU];
#pragma unroll
      for (int k = 0; k < HU; ++k) p[k] = Run<T, 8>::load(x + min(h + k, h1 - 1) * a.xh + f);
#pragma unroll
      for (int k = 0; k < HU; ++k)
        if (h + k < h1) p[k].store(y + (h + k) * a.yh + f);
    }
  }
}

template <typename T, int N, bool Interleaved>
hipError_t launch(const RotaryArgs& a, hipStream_t stream) {
  constexpr int kHeads = 4;
  const int units = a.rot / 2 / N + (a.x == a.y ? 0 : (a.d - a.rot) / 8);
  const int64_t runs = (int64_t)a.B * a.M * units;
  const unsigned blocks = (unsigned)((runs + kThreads - 1) / kThreads);
  // heads of a thread: as many as leave the device kOccupy threads, so that few
  // tokens spread over it and many form each angle once
  const int64_t kOccupy = (int64_t)device_cu_count() * 1024;
  const int64_t want = runs * a.H / kOccupy;
  if (want < kHeads) {
    hipLaunchKernelGGL((rotary_kernel<T, N, Interleaved, 1>), dim3(blocks, a.H), dim3(kThreads), 0, stream, a, units, 1);
  } else {
    const int per = (int)(want < a.H ? want : a.H);
    hipLaunchKernelGGL((rotary_kernel<T, N, Interleaved, kHeads>), dim3(blocks, (a.H + per - 1) / per), dim3(kThreads), 0,
                       stream, a, units, per);
  }
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
