// Attention of large tiles over the paged K/V cache, bf16: 256 rows (128 above a width of
// 128) that read the same pages for one key head.  Prompts and pieces of prompts
// (kv_large_packed.hip) and the queries of many entries over one shared prompt
// (kv_large_shared.hip).
//
// Bound by the matrix units: 4 d flops a pair of row and token, of which the weights' half is
// done three times for all of their bits (4 prompts of 4096 tokens, 16 heads of 128, 539 us: 510
// TFLOP/s, 1.02 PFLOP/s with the three, where a large library product reaches 1.15).  A
// wavefront holds 32 rows, a workgroup eight of them (four); a step of 64 tokens (32) is
// staged in LDS once for all, the next one on its way in registers.
// Both products are 32 x 32 tiles with the rows as columns:
//
//   S^T [tokens x rows] = K Q^T           A: 16 bytes of a key row (token-major)
//   O^T [features x rows] += V^T P^T      A: 16 bytes of a value row (feature-major)
//
// Lane (c, hf) = (lane % 32, lane / 32) of an accumulator holds rows 8 (i / 4) + 4 hf + i % 4
// of column c, so a row's maximum and sum take one exchange between the halves, and the
// weights are the next product's B operand as they are: row r of a tile of 32 tokens is
// token r with bits 2 and 3 exchanged, so that registers 8u .. 8u + 7 of half hf are
// tokens 16u + 8hf ...
#pragma once

#include <type_traits>

#include "kv_step.h"
#include "kv_tile.h"
#include "../../include/lla_kv.h"

namespace lla {

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int D>
struct LargeTile {
  static constexpr int kWaves = D <= 128 ? 8 : 4, kThreads = kWaves * kWave, kCols = kWaves * 32;
  static constexpr int kTok = D <= 128 ? 64 : 32, kSteps = kPage / kTok;
  static constexpr int KT = kTok / 32, FT = D / 32, KQ = D / 16;
  static constexpr int kKeyChunks = D / 8, kValChunks = kTok / 8;
  static constexpr int kUnits = 2 * kTok * D * 2 / 1024, J = kUnits / kWaves;  // kilobytes: of a step, of a wavefront
  static_assert(kUnits % kWaves == 0);

  // 16 bytes behind every row: the 8 lanes that LDS serves at a time meet different banks,
  // and all of a lane's operands lie at fixed distances from one address
  static constexpr int kKeyRow = D * 2 + 16, kValRow = kTok * 2 + 16;
  static constexpr int kBuffer = kTok * kKeyRow + D * kValRow;
  __device__ __forceinline__ static int key_at(int row, int chunk) { return row * kKeyRow + chunk * 16; }
  __device__ __forceinline__ static int val_at(int row, int chunk) { return kTok * kKeyRow + row * kValRow + chunk * 16; }

  // ---- staging ----
  uint4 r[J];
  // k, v: a step's first key, and its first token's value in feature row 0
  __device__ __forceinline__ void load(const char* k, const char* v, int w, int lane) {
    constexpr int kRow = kPage * 2, kUnitRows = kWave / kValChunks;
    const uint32_t val = lane / kValChunks * kRow + lane % kValChunks * 16;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int u = j * kWaves + w;
      const bool key = u < kUnits / 2;
      const char* from = key ? k + u * 1024 : v + (u - kUnits / 2) * kUnitRows * kRow;
      r[j] = ld16(from + (key ? lane * 16u : val));
    }
  }
  // Values that are not finite become zero; whether one was of a token that some row attends.
  template <typename Seen>
  __device__ __forceinline__ bool drop_nonfinite(int w, int lane, const Seen& seen) {
    bool any = false;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (j * kWaves + w < kUnits / 2) continue;
      uint32_t x[4] = {r[j].x, r[j].y, r[j].z, r[j].w};
      uint32_t lows = 0, highs = 0;  // a value is not finite where its 8 bits of exponent are ones
      bool bad = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        lows |= (x[i] & 0x7f80u) == 0x7f80u ? 1u << i : 0u;
        highs |= (x[i] & 0x7f800000u) == 0x7f800000u ? 1u << i : 0u;
      }
      bad = (lows | highs) != 0;
      if (!__any(bad)) continue;
      const int t = lane % kValChunks * 8;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool lo = lows >> i & 1, hi = highs >> i & 1;
        any |= (lo && seen(t + 2 * i)) || (hi && seen(t + 2 * i + 1));
        x[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
      }
      r[j] = uint4{x[0], x[1], x[2], x[3]};
    }
    return any;
  }
  __device__ __forceinline__ void stage(char* lds, int w, int lane) const {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int u = j * kWaves + w;
      const unsigned i = (u < kUnits / 2 ? u : u - kUnits / 2) * kWave + lane;
      *reinterpret_cast<uint4*>(lds + (u < kUnits / 2 ? key_at(i / kKeyChunks, i % kKeyChunks)
                                                      : val_at(i / kValChunks, i % kValChunks))) = r[j];
    }
  }

  // ---- products ----
  uint4 q[KQ];
  __device__ __forceinline__ void load_q(const bf16_t* row, int hf, bool in) {
#pragma unroll
    for (int s = 0; s < KQ; ++s) q[s] = in ? ld16(row + (2 * s + hf) * 8) : uint4{0, 0, 0, 0};
  }
  // token of register i of tile t in half 0, from the step's first; half 1's is 8 behind
  __device__ __forceinline__ static constexpr int token(int t, int i) { return 32 * t + 16 * (i / 8) + i % 8; }
  // A step's operands are read ahead of the products that take them, which then issue one
  // after another: the keys' (above a width of 128 in two parts), and the values' while
  // the exponentials are taken.
  static constexpr int kParts = D <= 128 ? 1 : 2, kQPart = KQ / kParts;
  static constexpr int kVals = 2 * KT * FT;  // of values: 16 tokens by 32 features each
  static_assert(KQ % kParts == 0);
  __device__ __forceinline__ void scores(const char* lds, int c, int hf, f32x16 (&sc)[KT]) const {
    const int row = (c & 19) | ((c & 4) << 1) | ((c & 8) >> 1);
#pragma unroll
    for (int t = 0; t < KT; ++t) sc[t] = f32x16{0.f};
#pragma unroll
    for (int part = 0; part < kParts; ++part) {
      uint4 x[kQPart][KT];
#pragma unroll
      for (int s = 0; s < kQPart; ++s)
#pragma unroll
        for (int t = 0; t < KT; ++t)
          x[s][t] = *reinterpret_cast<const uint4*>(lds + key_at(32 * t + row, 2 * (part * kQPart + s) + hf));
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < kQPart; ++s)
#pragma unroll
        for (int t = 0; t < KT; ++t)
          sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x[s][t]),
                                                          __builtin_bit_cast(bf16x8, q[part * kQPart + s]), sc[t], 0, 0, 0);
    }
  }
  // operand n of the values: tokens of group n / FT, features 32 (n % FT) ..
  __device__ __forceinline__ static uint4 value_operand(const char* lds, int c, int hf, int n) {
    return *reinterpret_cast<const uint4*>(lds + val_at(32 * (n % FT) + c, 2 * (n / FT) + hf));
  }
  // o += V^T P^T; returns the sum of this lane's weights.  A weight enters the product with its 24 bits, as three bf16:
  // rounded to one or two it would save half or a quarter of the step's products (4 prompts of 4096
  // tokens, 16 heads of 128: 348, 450 and 548 us with one, two and three), and would make what an
  // entry gets go by the kind of tile that its batch gives it.
  template <int kAhead>
  __device__ __forceinline__ float values(const char* lds, const uint4 (&ahead)[kAhead], int c, int hf, const f32x16 (&p)[KT],
                                          f32x16 (&o)[FT]) const {
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < 2 * KT; ++u) {
      bf16x8 w[3];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float x = p[u / 2][8 * (u % 2) + e];
        sum += x;
#pragma unroll
        for (int n = 0; n < 3; ++n) {
          w[n][e] = (__bf16)x;
          x -= (float)w[n][e];
        }
      }
#pragma unroll
      for (int f = 0; f < FT; ++f) {
        const int i = u * FT + f;
        const uint4 x = i < kAhead ? ahead[i < kAhead ? i : 0] : value_operand(lds, c, hf, i);
#pragma unroll
        for (int n = 0; n < 3; ++n)
          o[f] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), w[n], o[f], 0, 0, 0);
      }
    }
    return sum;
  }
};

// The greater of a lane's value and its other half's, NaN if either is.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Maxima above which a score's product is rounded before the maximum is taken from it, as
// the maximum's was: one fused with the difference is off by the product's rounding, at
// most 2^-8 of a power below (1 operation instead of 2 for each score).
constexpr float kFar = 65536.f;

template <int D, TileMode Mode>
__global__ __launch_bounds__(LargeTile<D>::kThreads) void large_tile_kernel(KvTileArgs args) {
  typedef LargeTile<D> L;
  constexpr int kCols = L::kCols, kThreads = L::kThreads, KT = L::KT, FT = L::FT, kTok = L::kTok;
  constexpr int kHeadBytes = kPage * D * 2;
  __shared__ int s_first[kMostEntries + 1], s_runs[kMostEntries + 1];
  __shared__ int s_wave[kThreads / kWave];
  __shared__ int s_odd;  // whether values of tokens that only some rows attend were not finite
  extern __shared__ __align__(16) char s_raw[];
  const int tid = threadIdx.x, lane = tid % kWave, c = lane % 32, hf = lane / 32;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);

  constexpr int64_t kFarTile = 1 << 28;
  const int group = args.H / args.p.Hkv;
  int last_from = 0;  // the last tile's number in its sequence, at most
  if constexpr (Mode == kPacked) {
    // (a start past the bound counts as at it: the search for a tile ends at last_from)
    for (int b = tid; b < args.B; b += kThreads)
      s_runs[b] = (int)min((int64_t)max(0, min(args.start[b], args.n_ctx)) * group / kCols, kFarTile);
    count_packed<kThreads>(args, kCols, args.small_rows, 0x7fffffff, s_first, s_wave);
    last_from = (int)(min((int64_t)args.n_ctx * group / kCols, kFarTile) + (int64_t)args.total * group / kCols) + 1;
  } else {
    count_shared<kThreads>(args, s_runs, nullptr, s_first, s_wave);
  }
  for (int item = blockIdx.x;; item += gridDim.x) {
    Tile t;
    int kvh, pb, pe;
    {
      const KvTileArgs& a = args_again();
      const int tiles = tiles_of(a.large, s_first[a.B]), slices = tile_slices(a.large, tiles * a.p.Hkv);
      if (item >= tiles * a.p.Hkv * slices) break;
      const int unit = item / a.p.Hkv, slice = unit / tiles, tile = tiles - 1 - (unit - slice * tiles);
      kvh = item - unit * a.p.Hkv;
      int b = last_at_most(s_first, a.B, tile), nth = tile - s_first[b];
      if constexpr (Mode == kPacked) {
        if (slices == 1 && a.B > 1) HeavyFirst{s_first, s_runs, a.B}.find(unit, last_from, b, nth);
      }
      t.at<Mode>(a, b, kCols, nth, Mode == kPacked ? 1 : run_entries(a, s_runs, b));
      const int per = slice_pages(a.large.least, t.keys.pages, slices);
      pb = slice * per;
      pe = min(t.keys.pages, pb + per);
      if (t.state != kFine || pb >= pe) {
        const int col = 32 * w + c;
        if (Mode == kPacked && slice == 0 && col < t.rows) {
          int64_t q_at, out_at;
          t.row_keys<Mode>(a, kvh, col, q_at, out_at);
          const float none = t.state == kNone ? __builtin_nanf("") : 0.f;
          for (int f = 4 * hf; f < D; f += 8) store_row4(a, out_at, f, f32x4{none, none, none, none});
          if (a.lse && hf == 0) a.lse[out_at] = t.state == kNone ? none : neg_inf();
        }
        continue;
      }
    }
    L st;
    RowKeys rk;
    TileKeys mine = t.keys;  // of this wavefront's rows, for the steps that it need not take or mask
    const char *k_pool, *v_pool;
    const int32_t* table;
    int n_pages;
    int64_t page_bytes;
    float qscale;
    {
      const KvTileArgs& a = args_again();
      int64_t q_at, unused;
      const int col = 32 * w + c;
      rk = t.row_keys<Mode>(a, kvh, min(col, t.rows - 1), q_at, unused);
      st.load_q(static_cast<const bf16_t*>(a.q) + q_at, hf, col < t.rows);
      // (rows are in the order of their tokens)
      mine.p_min = __builtin_amdgcn_readfirstlane(rk.p);
      mine.p_max = __builtin_amdgcn_readlane(rk.p, 31);
      mine.low_min = __builtin_amdgcn_readfirstlane(rk.low);
      mine.low_max = __builtin_amdgcn_readlane(rk.low, 31);
      k_pool = static_cast<const char*>(a.p.k) + (int64_t)kvh * kHeadBytes;
      v_pool = static_cast<const char*>(a.p.v) + (int64_t)kvh * kHeadBytes;
      table = a.p.table + (int64_t)t.row * a.p.max_pages;
      n_pages = a.p.n_pages;
      page_bytes = (int64_t)a.p.Hkv * kHeadBytes;
      qscale = a.qscale;
    }
    const bool idle = 32 * w >= t.rows;
    const int sink = t.keys.sink;
    // Pages of the slice, 64 at a time in the lanes of a register: -1 where there is none.
    // Steps are asked for one after another.
    int list = -1;
    auto page_of = [&](int s) {
      const int i = s / L::kSteps - pb;
      if (i % kWave == 0 && s % L::kSteps == 0) {
        list = -1;
        if (pb + i + lane < pe) {
          const int page = table[t.keys.page(pb + i + lane)];
          list = (unsigned)page >= (unsigned)n_pages ? -1 : page;
        }
      }
      return __builtin_amdgcn_readlane(list, i % kWave);
    };
    auto first_token = [&](int s) { return t.keys.page(s / L::kSteps) * kPage + s % L::kSteps * kTok; };
    auto request = [&](int page, int s) {
      const int64_t at = max(page, 0) * page_bytes;
      const int tok = s % L::kSteps * kTok;
      st.load(k_pool + at + tok * D * 2, v_pool + at + tok * 2, w, lane);
    };
    // Step s to its buffer; values that are not finite stay out of it where not all rows attend the step's tokens.
    auto put = [&](int s, bool whole) {
      if (!whole) {
        const int t0 = first_token(s);
        const RowKeys most{t.keys.p_max, t.keys.low_min};
        const bool odd = st.drop_nonfinite(w, lane, [&](int k) { return most.seen(t0 + k, sink); });
        if (__any(odd) && lane == 0) s_odd = 1;
      }
      st.stage(s_raw + (s & 1) * L::kBuffer, w, lane);
    };

    int s = pb * L::kSteps;
    const int end = pe * L::kSteps;
    float m = neg_inf(), l = 0.f;
    bool far = false;
    f32x16 o[FT];
#pragma unroll
    for (int f = 0; f < FT; ++f) o[f] = f32x16{0.f};
    // (the last tile's is 0 here, or all have read it: a barrier of add_nonfinite's is between)
    if (tid == 0) s_odd = 0;
    int now = page_of(s), next = s + 1 < end ? page_of(s + 1) : -1;
    bool whole = t.keys.whole(first_token(s), kTok);
    request(now, s);
    __syncthreads();
    put(s, whole);
    __syncthreads();

    // One step; with kMasked, of tokens that not all of the tile's rows attend, or of no page.
    auto step = [&](auto masked) {
      constexpr bool kMasked = decltype(masked)::value;
      const int t0 = kMasked ? first_token(s) : 0;
      if (idle || (kMasked && (now < 0 || !RowKeys{mine.p_max, mine.low_min}.any(t0, kTok, sink)))) {
        if (kMasked && now < 0 && rk.any(t0, kTok, sink)) l = __builtin_nanf("");
        return;
      }
      const char* lds = s_raw + (s & 1) * L::kBuffer;
      f32x16 sc[KT];
      st.scores(lds, c, hf, sc);
      constexpr int kAhead = kMasked ? FT : D <= 128 ? L::kVals : L::kVals / 2;
      uint4 ahead[kAhead];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ahead[i] = L::value_operand(lds, c, hf, i);
      __builtin_amdgcn_sched_barrier(0);
      if (kMasked && !mine.whole(t0, kTok)) {
        // token i of half 0 is attended up to p, below the sink or from low on
        const int p = rk.p - t0 - 8 * hf, low = rk.low - t0 - 8 * hf, first = sink - t0 - 8 * hf;
        if (mine.low_max == 0) {
#pragma unroll
          for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[x][i] = L::token(x, i) <= p ? sc[x][i] : neg_inf();
        } else {
#pragma unroll
          for (int x = 0; x < KT; ++x)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int n = L::token(x, i);
              sc[x][i] = n <= p && (n < first || n >= low) ? sc[x][i] : neg_inf();
            }
        }
      }
      float pm = sc[0][0];
#pragma unroll
      for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) pm = __builtin_elementwise_maximum(pm, sc[x][i]);
      pm = max_halves(pm) * qscale;
      if (__any(pm > m + kLazy)) {
        const float to = fmaxf(m, pm);
        const float alpha = m == neg_inf() ? 0.f : __builtin_amdgcn_exp2f(m - to);
        l *= alpha;
#pragma unroll
        for (int f = 0; f < FT; ++f) o[f] *= alpha;
        m = to;
        far = __any(fabsf(m) > kFar && m != neg_inf());
      }
      const float base = m == neg_inf() ? 0.f : m;
      if (far) {
#pragma unroll
        for (int x = 0; x < KT; ++x)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[x][i] = below(sc[x][i], qscale, base);
      }
      const float by = far ? 1.f : qscale, less = far ? 0.f : -base;
#pragma unroll
      for (int x = 0; x < KT; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[x][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x][i], by, less));
      l += st.values(lds, ahead, c, hf, sc, o);
    };
    // the next step's pages are asked for before a step and put after it
    while (s < end) {
      if (whole) {
        // steps from here on whose tokens all rows attend
        const int t0 = first_token(s), i = s / L::kSteps;
        const int to = t0 >= t.keys.low_max ? t.keys.p_min + 1 : min(sink, t.keys.p_min + 1);
        const int last = min(end, (i < t.keys.lead ? t.keys.lead : t.keys.pages) * L::kSteps);
        for (int n = min(last - s, (to - t0) / kTok); n > 1 && now >= 0 && next >= 0; --n) {
          request(next, s + 1);
          const int after = s + 2 < end ? page_of(s + 2) : -1;
          step(std::false_type{});
          put(s + 1, true);
          ++s;
          now = next;
          next = after;
          __syncthreads();
        }
      }
      const bool more = s + 1 < end;
      if (more) request(next, s + 1);
      const int after = s + 2 < end ? page_of(s + 2) : -1;
      step(std::true_type{});
      whole = more && t.keys.whole(first_token(s + 1), kTok);
      if (more) put(s + 1, whole);
      ++s;
      now = next;
      next = after;
      __syncthreads();
    }

    const KvTileArgs& a = args_again();
    const bool odd = s_odd != 0, direct = Mode == kPacked && pb == 0 && pe == t.keys.pages;
    float* const part = partial_row(a.large.part, item, kCols, 0, D);
    l += xor_shfl(l, 32);
    const int col = 32 * w + c;
    if (col < t.rows) {
      int64_t q_at, out_at;
      t.row_keys<Mode>(a, kvh, col, q_at, out_at);
      if (t.past_bound<Mode>(a, col)) l = __builtin_nanf("");
      if (direct) {
        const float by = 1.f / l;
#pragma unroll
        for (int f = 0; f < FT; ++f)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = o[f][4 * y + e] * by;
            store_row4(a, out_at, 32 * f + 8 * y + 4 * hf, v);
          }
        if (a.lse && hf == 0) a.lse[out_at] = ((m == neg_inf() ? 0.f : m) + __builtin_amdgcn_logf(l)) * kLn2;
      } else {
        float* to = part + col * (D + 4);
#pragma unroll
        for (int f = 0; f < FT; ++f)
#pragma unroll
          for (int y = 0; y < 4; ++y)
            *reinterpret_cast<f32x4*>(to + 32 * f + 8 * y + 4 * hf) =
                f32x4{o[f][4 * y], o[f][4 * y + 1], o[f][4 * y + 2], o[f][4 * y + 3]};
        if (hf == 0) {
          to[D] = m;
          to[D + 1] = l;
        }
      }
    }
    if (odd) add_nonfinite<Mode, bf16_t, D, kThreads>(a, t, kvh, pb, pe, direct ? nullptr : part);
  }
}

template <int D, TileMode Mode>
hipError_t launch_large(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  typedef LargeTile<D> L;
  hipLaunchKernelGGL((large_tile_kernel<D, Mode>), dim3(grid), dim3(L::kThreads), 2 * L::kBuffer, stream, a);
  return hipGetLastError();
}
// Widths of up to 128, and above, which are built apart.
template <TileMode Mode>
hipError_t launch_large_narrow(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  switch (a.p.d) {
    case 32: return launch_large<32, Mode>(a, grid, stream);
    case 64: return launch_large<64, Mode>(a, grid, stream);
    case 96: return launch_large<96, Mode>(a, grid, stream);
    default: return launch_large<128, Mode>(a, grid, stream);
  }
}
template <TileMode Mode>
hipError_t launch_large_wide(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  switch (a.p.d) {
    case 160: return launch_large<160, Mode>(a, grid, stream);
    case 192: return launch_large<192, Mode>(a, grid, stream);
    case 224: return launch_large<224, Mode>(a, grid, stream);
    default: return launch_large<256, Mode>(a, grid, stream);
  }
}

}  // namespace lla
