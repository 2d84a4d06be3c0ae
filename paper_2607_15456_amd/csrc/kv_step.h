// A wavefront's step of attention over the paged K/V cache: a page or a part of one
// from memory through its LDS into both products, and the arithmetic of partial
// softmaxes, shared by the decode (kv_decode.hip) and the attention of packed tokens
// and shared prompts (kv_tile_small.h).
#pragma once

#include "kv_internal.h"
#include "lla_device.h"

namespace lla {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t BufRsrc;

constexpr int kTile = 16;     // columns of a product: query heads
// Wavefronts of a workgroup, at most: four, so that two workgroups fit a compute
// unit; up to a width of 64, whose steps are small, eight where no second workgroup comes (24 x 17
// pages, 8 key heads of 64: 16.0 -> 15.1 us; at 128 no gain, 28.8 -> 29.5 on 4 x 4096).
constexpr int kWaves = 4;
constexpr int most_waves(int d) { return d <= 64 ? 2 * kWaves : kWaves; }
constexpr float kLazy = 8.f;  // log2 by which a step may exceed the running maximum
constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ BufRsrc make_rsrc(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, bytes, 0x00020000);
}
// (2: the non-temporal policy)
__device__ __forceinline__ uint4 buf_ld16(BufRsrc r, int voff, int soff) {
  return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, voff, soff, 2));
}
// Uniform read of an index array (nothing in a launch writes one).
typedef const int __attribute__((address_space(4))) ConstInt;
__device__ __forceinline__ int uniform(const int32_t* p, int64_t i) {
  return reinterpret_cast<ConstInt*>(reinterpret_cast<uintptr_t>(p))[i];
}

// Orders a wavefront's LDS accesses on either side: lanes read what others wrote.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// ---- one step of a wavefront ----
//
// A step's keys, then its values, go from memory to registers as whole
// consecutive kilobytes (read once: non-temporal), from there to the
// wavefront's own LDS, and from there to the matrix instructions as operands: 16
// bytes of a row a lane.  Straight from memory, an operand load touches 64 bytes
// of each of 16 rows, which the memory answers 12% more slowly (32 x 4096 tokens of 16 heads of
// 128: 191 us; the same bytes consecutive and non-temporal 168).  16-byte chunks
// of a row are stored at chunk ^ swizzle(row), so that the 8 lanes that LDS
// serves at a time meet different banks.

// bf16: a page, half of one where two tiles' accumulators of a wide head leave no
// registers for more (its values then come in 64-byte pieces).
template <int D, int NT>
struct StepBf16 {
  static constexpr int kTok = NT * D > 384 ? 32 : 64, kTiles = kTok / 16, kBytes = 2;
  static constexpr int KS = D / 32, FT = D / 16, UU = kTok / 32;
  static constexpr int kLoads = kTok * D * 2 / 1024;  // of the keys, and of the values
  static constexpr int kKeyChunks = D / 8, kValChunks = kTok / 8;
  uint4 q[NT][KS], k[kLoads], v[kLoads];

  __device__ __forceinline__ void load_q(int n, const void* row, int g, bool in) {
#pragma unroll
    for (int s = 0; s < KS; ++s)
      q[n][s] = in ? ld16(static_cast<const bf16_t*>(row) + 32 * s + 8 * g) : uint4{0, 0, 0, 0};
  }
  // lanes that read keys at a time hold rows 0 .. 3 and 8 .. 11 of 16
  __device__ __forceinline__ static int key_at(int row, int chunk) {
    const int i = (row & 3) | ((row >> 1) & 4);
    return (row * kKeyChunks + (chunk ^ (kKeyChunks % 8 ? i >> 1 : i))) * 16;
  }
  __device__ __forceinline__ static int val_at(int row, int chunk) {
    return (row * kValChunks + (chunk ^ (kValChunks == 8 ? row & 7 : (row >> 1) & 3))) * 16;
  }
  __device__ __forceinline__ void load_k(BufRsrc r, int tok, int lane) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) k[j] = buf_ld16(r, lane * 16, tok * D * 2 + j * 1024);
  }
  __device__ __forceinline__ void load_v(BufRsrc r, int tok, int lane) {
    constexpr int kRows = kWave / kValChunks;  // feature rows of a load
    const int at = lane / kValChunks * (kPage * 2) + lane % kValChunks * 16;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) v[j] = buf_ld16(r, at, tok * 2 + j * kRows * kPage * 2);
  }
  __device__ __forceinline__ void stage_k(char* lds, int lane) const {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = j * kWave + lane;
      *reinterpret_cast<uint4*>(lds + key_at(i / kKeyChunks, i % kKeyChunks)) = k[j];
    }
  }
  // tokens not attended become zero, whatever their slots hold
  template <typename Seen>
  __device__ __forceinline__ void mask_values(const Seen& seen, int lane) {
    uint32_t keep[4];
    const int t = lane % kValChunks * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      keep[i] = (seen(t + 2 * i) ? 0xffffu : 0u) | (seen(t + 2 * i + 1) ? 0xffff0000u : 0u);
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
      v[j] = uint4{v[j].x & keep[0], v[j].y & keep[1], v[j].z & keep[2], v[j].w & keep[3]};
  }
  // mask_values, and values that are not finite become zero, too; whether the lane had such
  template <typename Seen>
  __device__ __forceinline__ bool finite_values(const Seen& seen, int lane) {
    uint32_t all = 0;
    mask_values(seen, lane);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t odd = ((w[i] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;  // (exponents of ones carry over)
        all |= odd;
        w[i] &= ~((odd << 1) - (odd >> 15));  // (a half word of ones for its bit)
      }
      v[j] = uint4{w[0], w[1], w[2], w[3]};
    }
    return all != 0;
  }
  __device__ __forceinline__ void stage_v(char* lds, int lane) const {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = j * kWave + lane;
      *reinterpret_cast<uint4*>(lds + val_at(i / kValChunks, i % kValChunks)) = v[j];
    }
  }
  // token of register i of tile t in this lane, from the step's first
  __device__ __forceinline__ static int token(int t, int i, int g) { return 32 * (t / 2) + 8 * g + 4 * (t % 2) + i; }
  __device__ __forceinline__ void scores(const char* lds, int c, int g, f32x4 (&sc)[NT][kTiles]) const {
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
#pragma unroll
      for (int n = 0; n < NT; ++n) sc[n][t] = f32x4{0.f};
      const int row = 32 * (t / 2) + 8 * (c / 4) + 4 * (t % 2) + c % 4;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const bf16x8 x =
            __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(lds + key_at(row, 4 * s + g)));
#pragma unroll
        for (int n = 0; n < NT; ++n)
          sc[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, __builtin_bit_cast(bf16x8, q[n][s]), sc[n][t], 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ void values(const char* lds, int c, int g, const f32x4 (&p)[NT][kTiles],
                                         f32x4 (&o)[NT][FT]) const {
#pragma unroll
    for (int u = 0; u < UU; ++u) {
      bf16x8 hi[NT], mid[NT], lo[NT];  // 8 bits each of a weight's 24
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = p[n][2 * u + e / 4][e % 4];
          hi[n][e] = (__bf16)x;
          const float y = x - (float)hi[n][e];
          mid[n][e] = (__bf16)y;
          lo[n][e] = (__bf16)(y - (float)mid[n][e]);
        }
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        const bf16x8 w =
            __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(lds + val_at(16 * f + c, 4 * u + g)));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          o[n][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, hi[n], o[n][f], 0, 0, 0);
          o[n][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, mid[n], o[n][f], 0, 0, 0);
          o[n][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, lo[n], o[n][f], 0, 0, 0);
        }
      }
    }
  }
};

// fp32: half a page, or a quarter.
template <int D, int NT>
struct StepF32 {
  static constexpr int kTok = NT * D > 384 ? 16 : 32, kTiles = kTok / 16, kBytes = 4;
  static constexpr int KS = D / 16, FT = D / 16;
  static constexpr int kLoads = kTok * D * 4 / 1024;
  static constexpr int kKeyChunks = D / 4, kValChunks = kTok / 4;
  f32x4 q[NT][KS], k[kLoads], v[kLoads];

  __device__ __forceinline__ void load_q(int n, const void* row, int g, bool in) {
#pragma unroll
    for (int s = 0; s < KS; ++s)
      q[n][s] = in ? *reinterpret_cast<const f32x4*>(static_cast<const float*>(row) + 16 * s + 4 * g) : f32x4{0.f};
  }
  __device__ __forceinline__ static int key_at(int row, int chunk) { return (row * kKeyChunks + (chunk ^ (row & 7))) * 16; }
  __device__ __forceinline__ static int val_at(int row, int chunk) {
    return (row * kValChunks + (chunk ^ (kValChunks == 8 ? row & 7 : (row >> 1) & 3))) * 16;
  }
  __device__ __forceinline__ void load_k(BufRsrc r, int tok, int lane) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) k[j] = __builtin_bit_cast(f32x4, buf_ld16(r, lane * 16, tok * D * 4 + j * 1024));
  }
  __device__ __forceinline__ void load_v(BufRsrc r, int tok, int lane) {
    constexpr int kRows = kWave / kValChunks;
    const int at = lane / kValChunks * (kPage * 4) + lane % kValChunks * 16;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) v[j] = __builtin_bit_cast(f32x4, buf_ld16(r, at, tok * 4 + j * kRows * kPage * 4));
  }
  __device__ __forceinline__ void stage_k(char* lds, int lane) const {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = j * kWave + lane;
      *reinterpret_cast<f32x4*>(lds + key_at(i / kKeyChunks, i % kKeyChunks)) = k[j];
    }
  }
  template <typename Seen>
  __device__ __forceinline__ void mask_values(const Seen& seen, int lane) {
    const int t = lane % kValChunks * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool in = seen(t + e);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) v[j][e] = in ? v[j][e] : 0.f;
    }
  }
  template <typename Seen>
  __device__ __forceinline__ bool finite_values(const Seen& seen, int lane) {
    bool any = false;
    mask_values(seen, lane);
#pragma unroll
    for (int j = 0; j < kLoads; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool odd = (__float_as_uint(v[j][e]) & 0x7f800000u) == 0x7f800000u;
        any |= odd;
        v[j][e] = odd ? 0.f : v[j][e];
      }
    return any;
  }
  __device__ __forceinline__ void stage_v(char* lds, int lane) const {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const int i = j * kWave + lane;
      *reinterpret_cast<f32x4*>(lds + val_at(i / kValChunks, i % kValChunks)) = v[j];
    }
  }
  __device__ __forceinline__ static int token(int t, int i, int g) { return 16 * t + 4 * g + i; }
  __device__ __forceinline__ void scores(const char* lds, int c, int g, f32x4 (&sc)[NT][kTiles]) const {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) sc[n][t] = f32x4{0.f};
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const f32x4 y = *reinterpret_cast<const f32x4*>(lds + key_at(16 * t + c, 4 * s + g));
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            sc[n][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[e], q[n][s][e], sc[n][t], 0, 0, 0);
      }
  }
  __device__ __forceinline__ void values(const char* lds, int c, int g, const f32x4 (&p)[NT][kTiles],
                                         f32x4 (&o)[NT][FT]) const {
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        const f32x4 y = *reinterpret_cast<const f32x4*>(lds + val_at(16 * f + c, 4 * t + g));
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int n = 0; n < NT; ++n)
            o[n][f] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[e], p[n][t][e], o[n][f], 0, 0, 0);
      }
  }
};

// score * scale - base, the product rounded as the maximum's was: a fused one would
// leave the maximum's rounding, which past 2^31 is more than exp2 has a result for.
__device__ __forceinline__ float below(float score, float scale, float base) {
#pragma clang fp contract(off)
  const float x = score * scale;
  return x - base;
}

// One (m, l, o[]) into another: o2 and l2 were weighed by 2^-m2.
template <int FT>
__device__ __forceinline__ void join(float& m, float& l, f32x4 (&o)[FT], float m2, float l2, const float* o2) {
  const float to = fmaxf(m, m2), base = to == neg_inf() ? 0.f : to;
  const float x = __builtin_amdgcn_exp2f(m - base), y = __builtin_amdgcn_exp2f(m2 - base);
  m = to;
  l = l * x + l2 * y;
#pragma unroll
  for (int f = 0; f < FT; ++f) {
    const f32x4 w = *reinterpret_cast<const f32x4*>(o2 + 16 * f);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[f][i] = o[f][i] * x + w[i] * y;
  }
}

// Bytes that a wavefront leaves for its neighbour to join.
constexpr size_t join_bytes(int d, int tiles) { return (size_t)tiles * kTile * (d + 6) * sizeof(float); }

}  // namespace lla
