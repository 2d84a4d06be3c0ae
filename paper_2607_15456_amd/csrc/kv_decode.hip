// Decode attention over the paged K/V cache: one query per (entry, query head),
// grouped onto the key heads, over the pages that the page table names.
//
//   s_n = scale q . k_n,  o = sum_n softmax(s)_n v_n
//
// Every key and value is read once for all query heads of its group, so the
// bytes of the attended pages bound it: 2 d elements a token and key head, 4 d
// flops a token and query head.
//
// A workgroup takes up to 32 query heads of one (entry, key head) and a slice of
// its pages; a wavefront takes steps of 64 tokens (fp32: 32), every W-th of the
// slice's, with both products on the matrix instructions:
//
//   S^T [tokens x heads] = K Q^T      A: 16 bytes of a key row (token-major)
//   O^T [features x heads] += V^T P^T A: 16 bytes of a value row (feature-major)
//
// In a 16 x 16 accumulator lane (c, g) = (lane % 16, lane / 16) holds rows 4g ..
// 4g + 3 of column c, a query head: maximum and sum stay with the lane until the
// end, and its weights are the next product's B operand without a lane exchange
// once the token of each row is chosen so (bf16: rows 4g' + i of the two tiles of
// 32 tokens are tokens 8g' + i and 8g' + 4 + i; fp32: row and token are the same,
// and product e of a tile takes element e of every lane's 16 bytes).  Groups of
// fewer than 16 heads leave columns empty: at 16 columns the products take about
// a tenth of the time that their operands take to arrive.
//
// The running maximum is raised only when a step exceeds it by more than 2^8, so
// the accumulator is rarely rescaled.  bf16 weights enter as three bf16, which hold all
// of their 24 bits (two, 2^-17, made bf16 results fall to the neighbouring value more
// often; the third costs at most 2%: 24 x 17 pages of width 64 14.7 -> 15.0 us, 32 x
// 4096 tokens of 128 none).

#include <algorithm>

#include "kv_internal.h"
#include "lla_device.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

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

// Tokens that an entry attends, [0, first) and [last, n), and their pages: the
// sequence's pages 0 .. lead - 1, then lead + skip .. .
struct Span {
  int n, first, last, lead, skip, pages;
  __device__ __forceinline__ Span(int len, int sink, int window) {
    n = len;
    const bool cut = window > 0 && (int64_t)sink + window < n;
    first = cut ? sink : n;
    last = cut ? n - window : n;
    const int all = (n + kPage - 1) / kPage;
    lead = cut ? (first + kPage - 1) / kPage : all;
    skip = cut ? max(0, last / kPage - lead) : 0;
    pages = all - skip;
  }
  __device__ __forceinline__ int page(int i) const { return i < lead ? i : i + skip; }
  __device__ __forceinline__ bool seen(int t) const { return t < first || (t >= last && t < n); }
  // all tokens t .. t + count - 1
  __device__ __forceinline__ bool whole(int t, int count) const {
    return t + count <= first || (t >= last && t + count <= n);
  }
};

// Pages that each slice of an entry takes.  The split is of the entry's own pages: the
// bound, which a captured step sets for a sequence's whole life, says how many slices
// there may be (a sequence of 4096 tokens, 16 key heads, bound 131,072: 47 us with the
// bound's slices, 14 with its own; 24 x 1000 tokens of 8 heads of 64, bound 8192: 17.4, 18.3).
__device__ __forceinline__ int slice_pages(const KvDecodeArgs& a, int pages) {
  if (a.slices == 1) return pages;
  // the quotient: pages < 2^21 and slices <= 512, so the product with 2^32 / slices,
  // rounded up, is off by less than 1 / slices
  return max(a.least, (int)__umulhi((unsigned)(pages + a.slices - 1), a.inverse));
}

// Entry b's tokens: 0 for padding, -1 where its row or length is out of range.
__device__ __forceinline__ int entry_tokens(const KvDecodeArgs& a, int b, int& row) {
  row = a.rows ? uniform(a.rows, b) : b;
  if (row < 0 || row >= a.p.n_seqs) return a.rows && row == -1 ? 0 : -1;
  const int n = uniform(a.length, row);
  return n < 0 || n > a.n_ctx ? -1 : n;
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

// ---- output rows ----

// Four features from f on of row i (d wide).
__device__ __forceinline__ void store4(const KvDecodeArgs& a, int64_t i, int f, f32x4 v) {
  const int64_t at = i * a.p.d + f;
  if (a.out_dtype == LLA_BF16) {
    uint2 w;
    w.x = f32_to_bf16(v[0]) | (uint32_t(f32_to_bf16(v[1])) << 16);
    w.y = f32_to_bf16(v[2]) | (uint32_t(f32_to_bf16(v[3])) << 16);
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.out) + at) = w;
  } else {
    *reinterpret_cast<f32x4*>(static_cast<float*>(a.out) + at) = v;
  }
}

// Partial of a slice: d sums, the maximum (log2 units), the sum of weights, padding.
__device__ __forceinline__ float* partial(const KvDecodeArgs& a, int64_t row, int slice) {
  return a.part + (row * a.slices + slice) * (a.p.d + 4);
}

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

// NT tiles of 16 query heads.  Two wavefronts a SIMD; one above a width of 128,
// where steps are twice as large, so as many bytes are on their way, and with two
// tiles, whose accumulators need the registers.
template <template <int, int> class StepOf, int D, int NT>
__global__ __launch_bounds__(most_waves(D) * kWave, D <= 128 && NT * D <= 128 ? 2 : 1) void decode_kernel(KvDecodeArgs a) {
  typedef StepOf<D, NT> Step;
  constexpr int kStepBytes = Step::kTok * D * Step::kBytes;
  constexpr int FT = D / 16, kSteps = kPage / Step::kTok, kTiles = Step::kTiles;
  constexpr int kRow = D + 4, kCols = NT * kTile;
  // the wavefronts' steps, then what they join
  extern __shared__ __align__(16) char s_raw[];
  const int W = blockDim.x / kWave;  // 1, 2, 4 or 8
  float* const s_o = reinterpret_cast<float*>(s_raw);
  float(*const s_ml)[2][kCols] = reinterpret_cast<float(*)[2][kCols]>(s_o + W / 2 * kCols * kRow);
  const int tid = threadIdx.x, lane = tid % kWave, c = lane % 16, g = lane / 16;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  char* const lds = s_raw + w * kStepBytes;
  const int units = a.B * a.p.Hkv;
  const int slice = blockIdx.x / units, unit = blockIdx.x - slice * units;
  const int b = unit / a.p.Hkv, kvh = unit - b * a.p.Hkv;
  const int group = a.H / a.p.Hkv;
  const int h0 = blockIdx.y * kCols + c;  // tile x's column: head h0 + 16 x of the group
  const int64_t out_row = (int64_t)b * a.H + kvh * group + h0;

  int row;
  const int n = entry_tokens(a, b, row);
  const Span sp(max(n, 0), a.sink, a.window);
  const int per = slice_pages(a, sp.pages), pb = slice * per, pe = min(sp.pages, pb + per);
  if (n <= 0 || pb >= pe) {
    if (n <= 0 && slice == 0 && w == 0 && a.slices == 1) {
      const float none = n < 0 ? __builtin_nanf("") : 0.f;
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        if (h0 + x * kTile >= group) continue;
#pragma unroll
        for (int f = 0; f < FT; ++f) store4(a, out_row + x * kTile, 16 * f + 4 * g, f32x4{none, none, none, none});
        if (a.lse && g == 0) a.lse[out_row + x * kTile] = n < 0 ? none : neg_inf();
      }
    }
    return;
  }

  Step st;
  constexpr int kHeadBytes = kPage * D * Step::kBytes;
  const int32_t* table = a.p.table + (int64_t)row * a.p.max_pages;
  bool bad = false;
  // step t of the slice's: where its page's keys and values are
  auto block = [&](int t) -> int64_t {
    int page = uniform(table, sp.page(t / kSteps));
    bad |= page < 0 || page >= a.p.n_pages;
    page = page < 0 || page >= a.p.n_pages ? 0 : page;
    return ((int64_t)page * a.p.Hkv + kvh) * kHeadBytes;
  };
  auto keys = [&](int64_t at) { return make_rsrc(static_cast<const char*>(a.p.k) + at, kHeadBytes); };
  auto vals = [&](int64_t at) { return make_rsrc(static_cast<const char*>(a.p.v) + at, kHeadBytes); };

  int t = pb * kSteps + w;
  const int end = pe * kSteps;
  float m[NT], l[NT];
  f32x4 o[NT][FT];
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    m[x] = neg_inf();
    l[x] = 0.f;
#pragma unroll
    for (int f = 0; f < FT; ++f) o[x][f] = f32x4{0.f};
  }
  if (t < end) {
    const int64_t at = block(t);
    const int tok = t % kSteps * Step::kTok;
    st.load_k(keys(at), tok, lane);
    st.load_v(vals(at), tok, lane);
  }
#pragma unroll
  for (int x = 0; x < NT; ++x)
    st.load_q(x, static_cast<const char*>(a.q) + (out_row + x * kTile) * D * Step::kBytes, g, h0 + x * kTile < group);
  // A step's keys are requested as soon as the keys before have left their
  // registers for LDS, its values likewise.
  for (; t < end; t += W) {
    const bool more = t + W < end;
    const int tok = (t + W) % kSteps * Step::kTok;
    const int64_t next = more ? block(t + W) : 0;
    f32x4 sc[NT][kTiles];
    st.stage_k(lds, lane);
    if (more) st.load_k(keys(next), tok, lane);
    wave_lds_order();
    st.scores(lds, c, g, sc);
    wave_lds_order();
    const int t0 = sp.page(t / kSteps) * kPage + t % kSteps * Step::kTok;
    const bool whole = sp.whole(t0, Step::kTok);
    if (!whole) {
#pragma unroll
      for (int y = 0; y < kTiles; ++y)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!sp.seen(t0 + Step::token(y, i, g))) {
#pragma unroll
            for (int x = 0; x < NT; ++x) sc[x][y][i] = neg_inf();
          }
    }
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      float pm = neg_inf();
#pragma unroll
      for (int y = 0; y < kTiles; ++y)
#pragma unroll
        for (int i = 0; i < 4; ++i) pm = fmaxf(pm, sc[x][y][i]);
      pm = fmaxf(pm, xor_shfl(pm, 16));
      pm = fmaxf(pm, xor_shfl(pm, 32)) * a.qscale;
      if (__any(pm > m[x] + kLazy)) {
        const float to = fmaxf(m[x], pm);
        const float alpha = m[x] == neg_inf() ? 0.f : __builtin_amdgcn_exp2f(m[x] - to);
        l[x] *= alpha;
#pragma unroll
        for (int f = 0; f < FT; ++f) o[x][f] *= alpha;
        m[x] = to;
      }
      const float base = m[x] == neg_inf() ? 0.f : m[x];
#pragma unroll
      for (int y = 0; y < kTiles; ++y)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sc[x][y][i] = __builtin_amdgcn_exp2f(below(sc[x][y][i], a.qscale, base));
          l[x] += sc[x][y][i];
        }
    }
    if (!whole) st.mask_values([&](int k) { return sp.seen(t0 + k); }, lane);
    st.stage_v(lds, lane);
    if (more) st.load_v(vals(next), tok, lane);
    wave_lds_order();
    st.values(lds, c, g, sc, o);
    wave_lds_order();
  }
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    l[x] += xor_shfl(l[x], 16);
    l[x] += xor_shfl(l[x], 32);
    if (bad) l[x] = __builtin_nanf("");
  }

  // join the wavefronts, the upper half into the lower
  if (W > 1) __syncthreads();
  for (int half = W / 2; half >= 1; half /= 2) {
    if (w >= half && w < 2 * half) {
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        const int col = x * kTile + c;
        float* so = s_o + ((w - half) * kCols + col) * kRow + 4 * g;
#pragma unroll
        for (int f = 0; f < FT; ++f) *reinterpret_cast<f32x4*>(so + 16 * f) = o[x][f];
        if (g == 0) {
          s_ml[w - half][0][col] = m[x];
          s_ml[w - half][1][col] = l[x];
        }
      }
    }
    __syncthreads();
    if (w < half) {
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        const int col = x * kTile + c;
        join<FT>(m[x], l[x], o[x], s_ml[w][0][col], s_ml[w][1][col], s_o + (w * kCols + col) * kRow + 4 * g);
      }
    }
    if (half > 1) __syncthreads();
  }
  if (w != 0) return;
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    if (h0 + x * kTile >= group) continue;
    const int64_t at = out_row + x * kTile;
    if (a.slices > 1) {
      float* part = partial(a, at, slice);
#pragma unroll
      for (int f = 0; f < FT; ++f) *reinterpret_cast<f32x4*>(part + 16 * f + 4 * g) = o[x][f];
      if (g == 0) {
        part[D] = m[x];
        part[D + 1] = l[x];
      }
    } else {
#pragma unroll
      for (int f = 0; f < FT; ++f) store4(a, at, 16 * f + 4 * g, o[x][f] / l[x]);
      if (a.lse && g == 0) a.lse[at] = ((m[x] == neg_inf() ? 0.f : m[x]) + __builtin_amdgcn_logf(l[x])) * kLn2;
    }
  }
}

// Joins the slices of one (entry, query head): their weights 2^(m_s - m) first, a
// slice a thread, then four features a thread of every R-th slice.
constexpr int kJoinThreads = 256, kMaxSlices = 512;
__global__ __launch_bounds__(kJoinThreads) void join_kernel(KvDecodeArgs a) {
  constexpr int kJoinWaves = kJoinThreads / kWave;
  __shared__ __align__(16) float s_o[kJoinThreads * 4];
  __shared__ float s_w[kMaxSlices], s_red[2][kJoinWaves];
  const int64_t row_out = blockIdx.x;
  const int b = blockIdx.x / a.H, tid = threadIdx.x, d = a.p.d, lanes = d / 4;
  int row;
  const int n = entry_tokens(a, b, row);
  const Span sp(max(n, 0), a.sink, a.window);
  const int per = slice_pages(a, sp.pages), slices = (sp.pages + per - 1) / per;
  float ms[kMaxSlices / kJoinThreads], ls[kMaxSlices / kJoinThreads], m = neg_inf(), l = 0.f;
#pragma unroll
  for (int i = 0; i < kMaxSlices / kJoinThreads; ++i) {
    const int s = tid + i * kJoinThreads;
    ms[i] = neg_inf();
    ls[i] = 0.f;
    if (s < slices) {
      ms[i] = partial(a, row_out, s)[d];
      ls[i] = partial(a, row_out, s)[d + 1];
    }
    m = fmaxf(m, ms[i]);
  }
#pragma unroll
  for (int x = kWave / 2; x; x >>= 1) m = fmaxf(m, xor_shfl(m, x));
  if (tid % kWave == 0) s_red[0][tid / kWave] = m;
  __syncthreads();
#pragma unroll
  for (int x = 0; x < kJoinWaves; ++x) m = fmaxf(m, s_red[0][x]);
  const float base = m == neg_inf() ? 0.f : m;
#pragma unroll
  for (int i = 0; i < kMaxSlices / kJoinThreads; ++i) {
    const float w = __builtin_amdgcn_exp2f(ms[i] - base);
    s_w[tid + i * kJoinThreads] = w;
    l += ls[i] * w;
  }
#pragma unroll
  for (int x = kWave / 2; x; x >>= 1) l += xor_shfl(l, x);
  if (tid % kWave == 0) s_red[1][tid / kWave] = l;
  __syncthreads();
  l = 0.f;
#pragma unroll
  for (int x = 0; x < kJoinWaves; ++x) l += s_red[1][x];

  const int R = kJoinThreads / lanes, r = tid / lanes, f = tid % lanes;
  f32x4 o = f32x4{0.f};
  if (r < R) {
    const float* part = partial(a, row_out, 0) + 4 * f;
#pragma unroll 4
    for (int s = r; s < slices; s += R) o += *reinterpret_cast<const f32x4*>(part + (int64_t)s * (d + 4)) * s_w[s];
  }
  *reinterpret_cast<f32x4*>(&s_o[4 * tid]) = o;
  __syncthreads();
  if (r == 0) {
    for (int x = 1; x < R; ++x) o += *reinterpret_cast<const f32x4*>(&s_o[4 * (tid + x * lanes)]);
    const float none = n < 0 ? __builtin_nanf("") : 0.f;
    const bool empty = n <= 0;
    store4(a, row_out, 4 * f, empty ? f32x4{none, none, none, none} : o / l);
    if (a.lse && f == 0) a.lse[row_out] = n < 0 ? none : empty ? neg_inf() : (base + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

// Tiles of a workgroup: two from 17 query heads a group on (16 x 4096 tokens, 8 key
// heads, bf16, one tile / two: 20 heads a group 92 / 64 us, 64 133 / 115; width 256,
// 20 heads 187 / 135).
int query_tiles(int group) { return group > kTile ? 2 : 1; }
int query_blocks(int group) { return (group + kTile * query_tiles(group) - 1) / (kTile * query_tiles(group)); }

template <template <int, int> class StepOf, int D, int NT>
void launch_tiles(const KvDecodeArgs& a, hipStream_t stream) {
  typedef StepOf<D, NT> Step;
  const dim3 grid(a.B * a.p.Hkv * a.slices, query_blocks(a.H / a.p.Hkv));
  // wavefronts: no more than a slice has steps; of eight, each with a second one
  const int64_t steps = (int64_t)a.per * (kPage / Step::kTok);
  const bool alone = (int64_t)grid.x * grid.y <= device_cu_count();
  const int W = steps > most_waves(D) && alone ? most_waves(D) : steps >= kWaves ? kWaves : steps >= 2 ? 2 : 1;
  const size_t lds = std::max<size_t>((size_t)W * Step::kTok * D * Step::kBytes, W / 2 * join_bytes(D, NT));
  hipLaunchKernelGGL((decode_kernel<StepOf, D, NT>), grid, dim3(W * kWave), lds, stream, a);
}
template <template <int, int> class StepOf, int D>
void launch_step(const KvDecodeArgs& a, hipStream_t stream) {
  if (query_tiles(a.H / a.p.Hkv) == 2) launch_tiles<StepOf, D, 2>(a, stream);
  else launch_tiles<StepOf, D, 1>(a, stream);
}

template <int D>
hipError_t launch(const KvDecodeArgs& a, hipStream_t stream) {
  if (a.p.dtype == LLA_BF16) launch_step<StepBf16, D>(a, stream);
  else launch_step<StepF32, D>(a, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.slices == 1) return e;
  hipLaunchKernelGGL(join_kernel, dim3(a.B * a.H), dim3(kJoinThreads), 0, stream, a);
  return hipGetLastError();
}

int wave_pages(const KvDecodeArgs& a) { return a.p.dtype == LLA_BF16 ? kWaves : kWaves / 2; }  // of a step a wavefront

// Slices of a context, at most.  Long ones: as many as give each compute unit two
// workgroups, if a slice keeps kLong pages; otherwise one workgroup a unit, since
// a join costs a launch (4 us) and has to save more.  Measured (width 128, bf16
// but for the first; unsplit / split, us):
//   1 x 512 tokens, fp32, 16 key heads 21.5 / 10.9 (a page a slice), bf16 11.7 / 8.5
//   1 x 32,768, 2 key heads            312 / 15.9 (4 pages; 2 pages 17.9)
//   4 x 4096, 16 key heads             48.3 / 28.8 (16 pages; 8 pages 29.4)
//   24 of 17 pages, 8 key heads of 64  15.1 / 19.7
// and of 128 KB of keys and values or less, 8 wavefronts to a workgroup from 9 steps on:
//   512 tokens, 8 key heads of 64, bf16 1 x 7.7 / 7.6, 16 x 8.7 / 10.8, 320 tokens 7.3 / 7.7
//   1 x 512, 700, 1024, 8 of 32, bf16  5.9, 7.0, 7.5 / 7.6, 8.4, 7.8
//   256 tokens, 8 of 64, fp32          4 x 8.4 / 9.1
//   20 x 1024 .. 4096, 16 key heads    88 / 80;  12 x 2250 .. 9000, 8 key heads 102 / 59
//   40 x 4096, 16 key heads (640 workgroups) 219 / 218
int most_slices(const KvDecodeArgs& a, int units, int pages, int cus) {
  constexpr int kLong = 16, kAlone = 128 << 10;
  // a step a wavefront; of narrow heads, what eight wavefronts read in two steps or less
  const int bytes = a.p.d * (a.p.dtype == LLA_BF16 ? 256 : 512);
  if (pages <= wave_pages(a) || (most_waves(a.p.d) > kWaves && units <= cus && pages <= kAlone / bytes)) return 1;
  const int want = (2 * cus + units - 1) / units;
  return std::min(pages < (int64_t)want * kLong ? std::max(1, cus / units) : want, kMaxSlices);
}
// Most pages that an entry attends.
int most_pages(const KvDecodeArgs& a) {
  const int all = (a.n_ctx + kPage - 1) / kPage;
  const int64_t budget = ((int64_t)a.sink + kPage - 1) / kPage + ((int64_t)a.window + kPage - 1) / kPage + 1;
  return a.window ? (int)std::min<int64_t>(all, budget) : all;
}
int units_of(const KvDecodeArgs& a) { return a.p.Hkv * query_blocks(a.H / a.p.Hkv); }  // of an entry
size_t partial_bytes(const KvDecodeArgs& a, int B, int slices) {
  return slices == 1 ? 0 : (size_t)B * a.H * slices * (a.p.d + 4) * sizeof(float);
}
}  // namespace

size_t kv_decode_shape(KvDecodeArgs& a) {
  const int pages = most_pages(a), want = most_slices(a, a.B * units_of(a), pages, device_cu_count());
  a.per = (pages + want - 1) / want;
  a.slices = (pages + a.per - 1) / a.per;
  a.least = std::min(a.per, wave_pages(a));
  a.inverse = a.slices == 1 ? 0 : (unsigned)(((1ull << 32) + a.slices - 1) / a.slices);
  return partial_bytes(a, a.B, a.slices);
}

// With more pages there are no fewer slices wanted, with more entries there may be: the
// most of any number of them (none are split from 2 workgroups a compute unit on).
size_t kv_decode_workspace(const KvDecodeArgs& a) {
  const int pages = most_pages(a), cus = device_cu_count(), units = units_of(a);
  size_t most = 0;
  for (int B = 1; B <= a.B && (int64_t)B * units < 2 * cus; ++B)
    most = std::max(most, partial_bytes(a, B, std::min(pages, most_slices(a, B * units, pages, cus))));
  return most;
}

hipError_t launch_kv_decode(const KvDecodeArgs& a, hipStream_t stream) {
  switch (a.p.d) {
    case 32: return launch<32>(a, stream);
    case 64: return launch<64>(a, stream);
    case 96: return launch<96>(a, stream);
    case 128: return launch<128>(a, stream);
    case 160: return launch<160>(a, stream);
    case 192: return launch<192>(a, stream);
    case 224: return launch<224>(a, stream);
    default: return launch<256>(a, stream);
  }
}

}  // namespace lla
