// Rotary pairs on the device: the angle of a position and the turn of a run of
// pairs, shared by the embedding of queries (rotary.hip) and the write of keys
// into their pages (kv_write.hip).
//
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
// A thread's part of a row: a run of N features and the one as far behind it as
// half of the turned features, or half of the copied ones, are wide, so that
// neighbouring threads touch neighbouring runs.  Half-split these are N pairs;
// interleaved, N/2 pairs each; copied, the second may lie past the row's end.
// Turned and copied parts are moved alike: a wavefront that holds both does not
// branch.
template <typename T, int N, bool Interleaved>
struct Part {
  bool turned, second;
  int a_at, b_at;
  // parts of `copied` features, and of a row
  __host__ __device__ __forceinline__ static int copies(int copied) { return (copied + 2 * N - 1) / (2 * N); }
  __host__ __device__ __forceinline__ static int count(int rot, int copied) { return rot / 2 / N + copies(copied); }
  __device__ __forceinline__ Part(int u, int rot, int d) {
    const int pairs = rot / 2 / N;
    turned = u < pairs;
    a_at = turned ? u * N : rot + (u - pairs) * N;
    b_at = a_at + (turned ? rot / 2 : copies(d - rot) * N);
    second = b_at < d;
  }
  // the row's pair that is this part's i-th
  __device__ __forceinline__ int pair(int i) const {
    return !Interleaved ? a_at + i : i < N / 2 ? a_at / 2 + i : b_at / 2 + i - N / 2;
  }
  __device__ __forceinline__ void load_freq(double (&f)[N], const double* p) const {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = p[pair(i)];
  }

  Run<T, N> a, b;
  __device__ __forceinline__ void load(const T* x) {
    a = Run<T, N>::load(x + a_at);
    b = Run<T, N>::load(x + (second ? b_at : a_at));
  }
  __device__ __forceinline__ void turn(const Turn<N>& t) {
    Run<T, N> p = a, q = b;
    if constexpr (Interleaved) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        Run<T, N>& r = i < N / 2 ? p : q;
        const int j = 2 * (i % (N / 2));
        const float u = r.get(j), v = r.get(j + 1);
        r.set(j, u * t.c[i] - v * t.s[i]);
        r.set(j + 1, v * t.c[i] + u * t.s[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float u = p.get(i), v = q.get(i);
        p.set(i, u * t.c[i] - v * t.s[i]);
        q.set(i, v * t.c[i] + u * t.s[i]);
      }
    }
    if (turned) {
      a = p;
      b = q;
    }
  }
  __device__ __forceinline__ void store(T* y) const {
    a.store(y + a_at);
    if (second) b.store(y + b_at);
  }
  __device__ __forceinline__ void store_past(T* y) const {
    a.store_past(y + a_at);
    if (second) b.store_past(y + b_at);
  }
};

}  // namespace lla
