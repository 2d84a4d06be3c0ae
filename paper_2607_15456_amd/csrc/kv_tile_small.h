// Attention of small tiles over the paged K/V cache: up to 32 rows that read the same
// pages for one key head, in the steps of kv_step.h, a wavefront a page (fp32: half a
// page) at a time.  The few new tokens of a packed entry (kv_tile_packed.hip), the
// queries that read one shared prompt, and an entry's own tokens behind it
// (kv_tile_shared.hip).
//
// Bound by memory: every page is read once for the tile's rows.
#pragma once

#include <algorithm>

#include "kv_step.h"
#include "kv_tile.h"
#include "../../include/lla_kv.h"

namespace lla {

// Values that are not finite, which the matrix product of a step with rows that attend
// only some of its tokens has left out: added to the rows that attend them (a product
// with a weight of zero would give NaN to the others).  v: the step's first token of
// feature row 0.
template <typename T, int NT, int FT, typename Seen>
__device__ __forceinline__ void add_nonfinite(const T* v, int count, int g, const Seen& seen, f32x4 (&o)[NT][FT]) {
#pragma unroll 1
  for (int k = 0; k < count; ++k) {
    bool in[NT];
#pragma unroll
    for (int x = 0; x < NT; ++x) in[x] = seen(x, k);
#pragma unroll
    for (int f = 0; f < FT; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y = Elem<T>::get(v, (size_t)(16 * f + 4 * g + i) * kPage + k);
        if ((__float_as_uint(y) & 0x7f800000u) != 0x7f800000u) continue;
#pragma unroll
        for (int x = 0; x < NT; ++x)
          if (in[x]) o[x][f][i] += y;
      }
  }
}

// Packed: entries of few rows.  Otherwise the few queries of a run over their shared
// prompt, and every entry's own tokens, in one launch.
template <template <int, int> class StepOf, int D, int NT, bool Packed>
__global__ __launch_bounds__(kWaves* kWave, D <= 128 && NT * D <= 128 ? 2 : 1) void small_tile_kernel(KvTileArgs a) {
  typedef StepOf<D, NT> Step;
  typedef std::conditional_t<Step::kBytes == 2, bf16_t, float> T;
  constexpr int kStepBytes = Step::kTok * D * Step::kBytes;
  constexpr int FT = D / 16, kSteps = kPage / Step::kTok, kTiles = Step::kTiles;
  constexpr int kRow = D + 4, kCols = NT * kTile, kThreads = kWaves * kWave, W = kWaves;
  __shared__ int s_first[kMostEntries + 1], s_runs[Packed ? 1 : kMostEntries + 1];
  __shared__ int64_t s_wave[kThreads / kWave];
  // the wavefronts' steps, then what they join
  extern __shared__ __align__(16) char s_raw[];
  float* const s_o = reinterpret_cast<float*>(s_raw);
  float(*const s_ml)[2][kCols] = reinterpret_cast<float(*)[2][kCols]>(s_o + W / 2 * kCols * kRow);
  const int tid = threadIdx.x, lane = tid % kWave, c = lane % 16, g = lane / 16;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  char* const lds = s_raw + w * kStepBytes;
  const int group = a.H / a.p.Hkv, blocks = (group + kCols - 1) / kCols;

  // An entry's own tokens come first: how many tiles over prompts there are takes a count.
  const int64_t own_items = Packed ? 0 : (int64_t)a.B * blocks * a.p.Hkv * a.own_slices;
  int tiles = -1, slices = 1;
  for (int64_t i = blockIdx.x;; i += gridDim.x) {
    const bool own = !Packed && i < own_items;
    if (!own && tiles < 0) {
      if constexpr (Packed) count_packed<kThreads>(a, kCols, 0, a.small_rows, s_first, s_wave);
      else count_shared<kThreads>(a, s_runs, s_first, nullptr, s_wave);
      tiles = tiles_of(a.small, s_first[a.B]);
      slices = tile_slices(a.small, (int64_t)tiles * a.p.Hkv);
    }
    const int64_t item = own ? i : i - own_items;
    if (!own && item >= (int64_t)tiles * a.p.Hkv * slices) break;
    const int kvh = (int)(item % a.p.Hkv), unit = (int)(item / a.p.Hkv), of = own ? a.B * blocks : tiles;
    const int slice = unit / of, tile = of - 1 - (unit - slice * of);
    float* const part = own ? a.own_part : a.small.part;
    Tile t;
    if (own) {
      t.at<kOwn>(a, tile / blocks, kCols, tile % blocks);
    } else {
      const int b = last_at_most(s_first, a.B, tile);
      if constexpr (Packed) t.at<kPacked>(a, b, kCols, tile - s_first[b]);
      else t.at<kPrefix>(a, b, kCols, tile - s_first[b], run_entries(a, s_runs, b));
    }
    const int per = slice_pages(a.small.least, t.keys.pages, own ? a.own_slices : slices), pb = slice * per,
              pe = min(t.keys.pages, pb + per);
    const bool direct = Packed && per >= t.keys.pages;
    constexpr TileMode Mode = Packed ? kPacked : kOwn;  // (rows of both kinds of shared tiles are entries)
    RowKeys rk[NT];
    int64_t q_at[NT], out_at[NT];
    bool in[NT];
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      const int col = x * kTile + c;
      in[x] = col < t.rows;
      rk[x] = t.row_keys<Mode>(a, kvh, min(col, t.rows - 1), q_at[x], out_at[x]);
    }
    if (t.state != kFine || pb >= pe) {
      if (Packed && slice == 0 && w == 0) {
        const float none = t.state == kNone ? __builtin_nanf("") : 0.f;
#pragma unroll
        for (int x = 0; x < NT; ++x) {
          if (!in[x]) continue;
#pragma unroll
          for (int f = 0; f < FT; ++f) store_row4(a, out_at[x], 16 * f + 4 * g, f32x4{none, none, none, none});
          if (a.lse && g == 0) a.lse[out_at[x]] = t.state == kNone ? none : neg_inf();
        }
      }
      continue;
    }

    Step st;
    constexpr int kHeadBytes = kPage * D * Step::kBytes;
    const int32_t* table = a.p.table + (int64_t)t.row * a.p.max_pages;
    // step s of the tile's: where its page's keys and values are (-1: nowhere)
    auto block = [&](int s) -> int64_t {
      const int page = uniform(table, t.keys.page(s / kSteps));
      return page < 0 || page >= a.p.n_pages ? -1 : ((int64_t)page * a.p.Hkv + kvh) * kHeadBytes;
    };
    auto keys = [&](int64_t at) { return make_rsrc(static_cast<const char*>(a.p.k) + max(at, (int64_t)0), kHeadBytes); };
    auto vals = [&](int64_t at) { return make_rsrc(static_cast<const char*>(a.p.v) + max(at, (int64_t)0), kHeadBytes); };

    int s = pb * kSteps + w;
    const int end = pe * kSteps;
    int64_t now = -1;
    float m[NT], l[NT];
    f32x4 o[NT][FT];
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      m[x] = neg_inf();
      l[x] = 0.f;
#pragma unroll
      for (int f = 0; f < FT; ++f) o[x][f] = f32x4{0.f};
    }
    if (s < end) {
      now = block(s);
      const int tok = s % kSteps * Step::kTok;
      st.load_k(keys(now), tok, lane);
      st.load_v(vals(now), tok, lane);
    }
#pragma unroll
    for (int x = 0; x < NT; ++x) st.load_q(x, static_cast<const T*>(a.q) + q_at[x], g, in[x]);
    for (; s < end; s += W) {
      const bool more = s + W < end;
      const int tok = (s + W) % kSteps * Step::kTok;
      const int64_t next = more ? block(s + W) : -1;
      f32x4 sc[NT][kTiles];
      st.stage_k(lds, lane);
      if (more) st.load_k(keys(next), tok, lane);
      wave_lds_order();
      st.scores(lds, c, g, sc);
      wave_lds_order();
      const int t0 = t.keys.page(s / kSteps) * kPage + s % kSteps * Step::kTok;
      const bool good = now >= 0, whole = good && t.keys.whole(t0, Step::kTok);
      if (!whole) {
#pragma unroll
        for (int x = 0; x < NT; ++x) {
#pragma unroll
          for (int y = 0; y < kTiles; ++y)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (!good || !rk[x].seen(t0 + Step::token(y, i, g), t.keys.sink)) sc[x][y][i] = neg_inf();
          if (!good && rk[x].any(t0, Step::kTok, t.keys.sink)) l[x] = __builtin_nanf("");
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
      bool odd = false;  // values that are not finite among tokens that only some rows attend
      if (!whole) {
        const RowKeys most{t.keys.p_max, t.keys.low_min};
        st.mask_values([&](int k) { return good && most.seen(t0 + k, t.keys.sink); }, lane);
        if (Packed) odd = __any(st.drop_nonfinite());
      }
      st.stage_v(lds, lane);
      if (more) st.load_v(vals(next), tok, lane);
      wave_lds_order();
      st.values(lds, c, g, sc, o);
      wave_lds_order();
      if (Packed && odd)
        add_nonfinite<T, NT, FT>(reinterpret_cast<const T*>(static_cast<const char*>(a.p.v) + now) + t0 % kPage, Step::kTok,
                                 g, [&](int x, int k) { return rk[x].seen(t0 + k, t.keys.sink); }, o);
      now = next;
    }
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      l[x] += xor_shfl(l[x], 16);
      l[x] += xor_shfl(l[x], 32);
      if (in[x] && t.past_bound<Mode>(a, x * kTile + c)) l[x] = __builtin_nanf("");
    }

    // join the wavefronts, the upper half into the lower
    __syncthreads();
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
      __syncthreads();
    }
    if (w == 0) {
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        if (!in[x]) continue;
        if (direct) {
#pragma unroll
          for (int f = 0; f < FT; ++f) store_row4(a, out_at[x], 16 * f + 4 * g, o[x][f] / l[x]);
          if (a.lse && g == 0) a.lse[out_at[x]] = ((m[x] == neg_inf() ? 0.f : m[x]) + __builtin_amdgcn_logf(l[x])) * kLn2;
        } else {
          float* to = partial_row(part, item, kCols, x * kTile + c, D);
#pragma unroll
          for (int f = 0; f < FT; ++f) *reinterpret_cast<f32x4*>(to + 16 * f + 4 * g) = o[x][f];
          if (g == 0) {
            to[D] = m[x];
            to[D + 1] = l[x];
          }
        }
      }
    }
  }
}

template <template <int, int> class StepOf, int D, int NT, bool Packed>
hipError_t launch_small(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  typedef StepOf<D, NT> Step;
  const size_t lds = std::max<size_t>((size_t)kWaves * Step::kTok * D * Step::kBytes, kWaves / 2 * join_bytes(D, NT));
  hipLaunchKernelGGL((small_tile_kernel<StepOf, D, NT, Packed>), dim3(grid), dim3(kWaves * kWave), lds, stream, a);
  return hipGetLastError();
}

template <int NT, bool Packed, template <int, int> class StepOf>
hipError_t launch_small_width(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  switch (a.p.d) {
    case 32: return launch_small<StepOf, 32, NT, Packed>(a, grid, stream);
    case 64: return launch_small<StepOf, 64, NT, Packed>(a, grid, stream);
    case 96: return launch_small<StepOf, 96, NT, Packed>(a, grid, stream);
    case 128: return launch_small<StepOf, 128, NT, Packed>(a, grid, stream);
    case 160: return launch_small<StepOf, 160, NT, Packed>(a, grid, stream);
    case 192: return launch_small<StepOf, 192, NT, Packed>(a, grid, stream);
    case 224: return launch_small<StepOf, 224, NT, Packed>(a, grid, stream);
    default: return launch_small<StepOf, 256, NT, Packed>(a, grid, stream);
  }
}
template <int NT, bool Packed>
hipError_t launch_small_type(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  return a.p.dtype == LLA_BF16 ? launch_small_width<NT, Packed, StepBf16>(a, grid, stream)
                               : launch_small_width<NT, Packed, StepF32>(a, grid, stream);
}

}  // namespace lla
