// Rotary pairs on the device: the angle of a position and the turn of a run of
// pairs, shared by the embedding of queries (rotary.hip) and the write of keys
// into their pages (kv_write.hip).
//
// A thread holds the N pairs of one token and turns them for one head after
// another, so the angle (64-bit product and reduction, about 60 instructions a
// pair with sine and cosine) is paid once per token, not once per head.
#pragma once

#include "lla_device.h"

namespace lla {

// Runs of N elements in the widest accesses that divide them.
template <typename T, int N>
struct Run {
  static constexpr int kBytes = N * (int)sizeof(T);
  typedef uint32_t Words __attribute__((ext_vector_type(kBytes / 4)));
  Words w;
  __device__ __forceinline__ static Run load(const void* p) { return Run{*static_cast<const Words*>(p)}; }
  __device__ __forceinline__ void store(void* p) const { *static_cast<Words*>(p) = w; }
  __device__ __forceinline__ float get(int i) const;
  __device__ __forceinline__ void set(int i, float v);
};
template <typename T, int N>
__device__ __forceinline__ float Run<T, N>::get(int i) const {
  if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
  else return i & 1 ? bf16_hi(w[i / 2]) : bf16_lo(w[i / 2]);
}
template <typename T, int N>
__device__ __forceinline__ void Run<T, N>::set(int i, float v) {
  if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(v);
  else w[i / 2] = i & 1 ? (w[i / 2] & 0xffffu) | (uint32_t(f32_to_bf16(v)) << 16)
                        : (w[i / 2] & 0xffff0000u) | f32_to_bf16(v);
}

// magnitude * (cos, sin) of position * freq, the angle reduced to [-pi, pi] in
// 64 bits (positions reach 2^31) and evaluated in 32.
template <int N>
struct Turn {
  float c[N], s[N];
  __device__ __forceinline__ void at(double pos, const double* freq, float magnitude, float sign) {
    constexpr double kTwoPi = 6.283185307179586476925286766559;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double ang = pos * freq[i];
      const double r = ang - rint(ang * (1.0 / kTwoPi)) * kTwoPi;
      float sn, cs;
      sincosf((float)r, &sn, &cs);
      c[i] = magnitude * cs;
      s[i] = magnitude * sign * sn;
    }
  }
};

// The N pairs from pair p0 on of the row at x, turned, to the row at y (which
// may be x): features (i, i + half), or (2i, 2i + 1) when interleaved.
template <typename T, int N, bool Interleaved>
struct Pairs {
  Run<T, N> a, b;  // half-split: features p0 .., half + p0 ..; interleaved: 2 p0 .., 2 p0 + N ..
  __device__ __forceinline__ static int first(int p0) { return Interleaved ? 2 * p0 : p0; }
  __device__ __forceinline__ static int second(int p0, int half) { return Interleaved ? 2 * p0 + N : half + p0; }
  __device__ __forceinline__ void load(const T* x, int p0, int half) {
    a = Run<T, N>::load(x + first(p0));
    b = Run<T, N>::load(x + second(p0, half));
  }
  __device__ __forceinline__ void turn(const Turn<N>& t) {
    if constexpr (Interleaved) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        Run<T, N>& r = i < N / 2 ? a : b;
        const int j = 2 * (i % (N / 2));
        const float u = r.get(j), v = r.get(j + 1);
        r.set(j, u * t.c[i] - v * t.s[i]);
        r.set(j + 1, v * t.c[i] + u * t.s[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float u = a.get(i), v = b.get(i);
        a.set(i, u * t.c[i] - v * t.s[i]);
        b.set(i, v * t.c[i] + u * t.s[i]);
      }
    }
  }
  __device__ __forceinline__ void store(T* y, int p0, int half) const {
    a.store(y + first(p0));
    b.store(y + second(p0, half));
  }
};

}  // namespace lla
