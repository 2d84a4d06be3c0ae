// Rotary pairs on the device: the angle of a position and the turn of a run of
// pairs, shared by the embedding of queries (rotary.hip) and the write of keys
// into their pages (kv_write.hip).
//
// A thread holds the N pairs of one token and turns them for several heads, so
// the angle (64-bit product and reduction, sine and cosine) is paid once.
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
  // with the non-temporal policy
  __device__ __forceinline__ void store_past(void* p) const { __builtin_nontemporal_store(w, static_cast<Words*>(p)); }
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

// cos and sin of an angle: in 64 bits the angle is brought to within pi/4 of a
// multiple j of pi/2 (positions reach 2^31: the product is right to 2^-22 there),
// in 32 their series about 0 are summed (the first terms left out are below
// 2e-9) and go by j's quarter.  About 30 instructions, half of the library's
// sincosf, which has to be ready for any argument.
__device__ __forceinline__ void cos_sin(double angle, float& c, float& s) {
  constexpr double kHalfPi = 1.5707963267948966192313216916398;
  const double j = rint(angle * (1.0 / kHalfPi));
  const float y = (float)__builtin_fma(-j, kHalfPi, angle), z = y * y;
  const int quarter = (int)(j - 4.0 * rint(j * 0.25));  // -2 .. 2
  float sn = __builtin_fmaf(z, 1.f / 362880.f, -1.f / 5040.f);
  sn = __builtin_fmaf(sn, z, 1.f / 120.f);
  sn = __builtin_fmaf(sn, z, -1.f / 6.f);
  sn = __builtin_fmaf(sn * z, y, y);
  float cs = __builtin_fmaf(z, -1.f / 3628800.f, 1.f / 40320.f);
  cs = __builtin_fmaf(cs, z, -1.f / 720.f);
  cs = __builtin_fmaf(cs, z, 1.f / 24.f);
  cs = __builtin_fmaf(cs, z, -0.5f);
  cs = __builtin_fmaf(cs, z, 1.f);
  const float u = quarter & 1 ? sn : cs, v = quarter & 1 ? cs : sn;
  c = (quarter + 1) & 2 ? -u : u;
  s = quarter & 2 ? -v : v;
}

// magnitude * (cos, sin) of position * freq for N pairs.
template <int N>
struct Turn {
  float c[N], s[N];
  __device__ __forceinline__ void at(double pos, const double (&freq)[N], float magnitude, float sign) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float sn, cs;
      cos_sin(pos * freq[i], cs, sn);
      c[i] = magnitude * cs;
      s[i] = magnitude * sign * sn;
    }
  }
};
template <int N>
__device__ __forceinline__ void load_freq(double (&f)[N], const double* p) {
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = p[i];
}

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
  __device__ __forceinline__ void store_past(T* y, int p0, int half) const {
    a.store_past(y + first(p0));
    b.store_past(y + second(p0, half));
  }
};

}  // namespace lla
