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

// Packed: entries of few rows.  Otherwise the few queries of a run over their shared
// prompt, and every entry's own tokens, in one launch.
template <template <int, int> class StepOf, int D, int NT, bool Packed>
__global__ __launch_bounds__(kWaves* kWave, D <= 128 && NT * D <= 128 ? 2 : 1) void small_tile_kernel(KvTileArgs args) {
  typedef StepOf<D, NT> Step;
  typedef std::conditional_t<Step::kBytes == 2, bf16_t, float> T;
  constexpr int kStepBytes = Step::kTok * D * Step::kBytes;
  constexpr int FT = D / 16, kSteps = kPage / Step::kTok, kTiles = Step::kTiles;
  constexpr int kRow = D + 4, kCols = NT * kTile, kThreads = kWaves * kWave, W = kWaves;
  __shared__ int s_first[kMostEntries + 1], s_runs[Packed ? 1 : kMostEntries + 1];
  __shared__ int s_wave[kThreads / kWave];
  // the wavefronts' steps, then what they join
  extern __shared__ __align__(16) char s_raw[];
  float* const s_o = reinterpret_cast<float*>(s_raw);
  float(*const s_ml)[2][kCols] = reinterpret_cast<float(*)[2][kCols]>(s_o + W / 2 * kCols * kRow);
  const int tid = threadIdx.x, lane = tid % kWave, c = lane % 16, g = lane / 16;
  const int w = __builtin_amdgcn_readfirstlane(tid / kWave);
  char* const lds = s_raw + w * kStepBytes;
  constexpr TileMode Mode = Packed ? kPacked : kOwn;  // (rows of both kinds of shared tiles are entries)
  // An entry's own tokens come first: how many tiles over prompts there are takes a count.
  int tiles = -1, slices = 1;
  for (int i = blockIdx.x;; i += gridDim.x) {
    Tile t;
    bool own;
    int kvh, pb, pe;
    {
      const KvTileArgs& a = args_again();
      const int group = a.H / a.p.Hkv, blocks = (group + kCols - 1) / kCols;
      const int own_items = Packed ? 0 : a.B * blocks * a.p.Hkv * a.own_slices;
      own = !Packed && i < own_items;
      if (!own && tiles < 0) {
        if constexpr (Packed) count_packed<kThreads>(a, kCols, 0, a.small_rows, s_first, s_wave);
        else count_shared<kThreads>(a, s_runs, s_first, nullptr, s_wave);
        tiles = tiles_of(a.small, s_first[a.B]);
        slices = tile_slices(a.small, tiles * a.p.Hkv);
      }
      const int item = own ? i : i - own_items;
      if (!own && item >= tiles * a.p.Hkv * slices) break;
      const int unit = item / a.p.Hkv, of = own ? a.B * blocks : tiles;
      kvh = item - unit * a.p.Hkv;
      const int slice = unit / of, tile = of - 1 - (unit - slice * of);
      if (own) {
        t.at<kOwn>(a, tile / blocks, kCols, tile % blocks);
      } else {
        const int b = last_at_most(s_first, a.B, tile);
        if constexpr (Packed) t.at<kPacked>(a, b, kCols, tile - s_first[b]);
        else t.at<kPrefix>(a, b, kCols, tile - s_first[b], run_entries(a, s_runs, b));
      }
      const int per = slice_pages(a.small.least, t.keys.pages, own ? a.own_slices : slices);
      pb = slice * per;
      pe = min(t.keys.pages, pb + per);
      if (t.state != kFine || pb >= pe) {
        if (Packed && slice == 0 && w == 0) {
          const float none = t.state == kNone ? __builtin_nanf("") : 0.f;
#pragma unroll
          for (int x = 0; x < NT; ++x) {
            if (x * kTile + c >= t.rows) continue;
            int64_t q_at, out_at;
            t.row_keys<Mode>(a, kvh, x * kTile + c, q_at, out_at);
            for (int f = 0; f < FT; ++f) store_row4(a, out_at, 16 * f + 4 * g, f32x4{none, none, none, none});
            if (a.lse && g == 0) a.lse[out_at] = t.state == kNone ? none : neg_inf();
          }
        }
        continue;
      }
    }

    Step st;
    RowKeys rk[NT];
    const char *k_pool, *v_pool;
    const int32_t* table;
    int n_pages;
    int64_t page_bytes;
    float qscale;
    const void* q;
    int64_t q_at[NT];
    {
      const KvTileArgs& a = args_again();
      int64_t unused;
#pragma unroll
      for (int x = 0; x < NT; ++x) rk[x] = t.row_keys<Mode>(a, kvh, min(x * kTile + c, t.rows - 1), q_at[x], unused);
      constexpr int kHeadBytes = kPage * D * Step::kBytes;
      // (all of a workgroup's lanes agree on them: a page's resource stays in scalar registers)
      k_pool = scalar(static_cast<const char*>(a.p.k) + (int64_t)kvh * kHeadBytes);
      v_pool = scalar(static_cast<const char*>(a.p.v) + (int64_t)kvh * kHeadBytes);
      table = scalar(a.p.table + (int64_t)t.row * a.p.max_pages);
      n_pages = __builtin_amdgcn_readfirstlane(a.p.n_pages);
      page_bytes = (int64_t)__builtin_amdgcn_readfirstlane(a.p.Hkv) * kHeadBytes;
      qscale = a.qscale;
      q = a.q;
    }
    // step s of the tile's: where its page is in the pools (-1: nowhere)
    auto block = [&](int s) -> int64_t {
      const int page = uniform(table, t.keys.page(s / kSteps));
      return (unsigned)page >= (unsigned)n_pages ? -1 : page * page_bytes;
    };
    auto keys = [&](int64_t at) { return make_rsrc(k_pool + max(at, (int64_t)0), kPage * D * Step::kBytes); };
    auto vals = [&](int64_t at) { return make_rsrc(v_pool + max(at, (int64_t)0), kPage * D * Step::kBytes); };

    int s = pb * kSteps + w;
    const int end = pe * kSteps;
    bool odd = false;  // values that are not finite among tokens that only some rows attend
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
    for (int x = 0; x < NT; ++x) st.load_q(x, static_cast<const T*>(q) + q_at[x], g, x * kTile + c < t.rows);
    // A step's keys are requested as soon as the keys before have left their registers for
    // LDS, its values likewise.
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
        pm = fmaxf(pm, xor_shfl(pm, 32)) * qscale;
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
            sc[x][y][i] = __builtin_amdgcn_exp2f(below(sc[x][y][i], qscale, base));
            l[x] += sc[x][y][i];
          }
      }
      // Values of tokens that not all rows attend: weights of zero keep them out of the rows
      // that do not, if they are finite.  Shared tiles' rows all attend the same.
      if (!whole) {
        const RowKeys most{t.keys.p_max, t.keys.low_min};
        auto attended = [&](int k) { return good && most.seen(t0 + k, t.keys.sink); };
        if constexpr (Packed) odd |= st.finite_values(attended, lane);
        else st.mask_values(attended, lane);
      }
      st.stage_v(lds, lane);
      if (more) st.load_v(vals(next), tok, lane);
      wave_lds_order();
      st.values(lds, c, g, sc, o);
      wave_lds_order();
      now = next;
    }
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      l[x] += xor_shfl(l[x], 16);
      l[x] += xor_shfl(l[x], 32);
    }

    // join the wavefronts, the upper half into the lower
    const bool any_odd = __syncthreads_or(odd);
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
    const KvTileArgs& a = args_again();
    const bool whole = Packed && pb == 0 && pe == t.keys.pages;
    const int own_items = Packed ? 0 : a.B * ((a.H / a.p.Hkv + kCols - 1) / kCols) * a.p.Hkv * a.own_slices;
    float* const part = partial_row(own ? a.own_part : a.small.part, own ? i : i - own_items, kCols, 0, D);
    if (w == 0) {
#pragma unroll
      for (int x = 0; x < NT; ++x) {
        const int col = x * kTile + c;
        if (col >= t.rows) continue;
        if (t.past_bound<Mode>(a, col)) l[x] = __builtin_nanf("");
        if (whole) {
          int64_t q_unused, out_at;
          t.row_keys<Mode>(a, kvh, col, q_unused, out_at);
#pragma unroll
          for (int f = 0; f < FT; ++f) store_row4(a, out_at, 16 * f + 4 * g, o[x][f] / l[x]);
          if (a.lse && g == 0) a.lse[out_at] = ((m[x] == neg_inf() ? 0.f : m[x]) + __builtin_amdgcn_logf(l[x])) * kLn2;
        } else {
          float* to = part + col * (D + 4);
#pragma unroll
          for (int f = 0; f < FT; ++f) *reinterpret_cast<f32x4*>(to + 16 * f + 4 * g) = o[x][f];
          if (g == 0) {
            to[D] = m[x];
            to[D + 1] = l[x];
          }
        }
      }
    }
    if constexpr (Packed) {
      if (any_odd) add_nonfinite<kPacked, T, D, kThreads>(a, t, kvh, pb, pe, whole ? nullptr : part);
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
  constexpr bool kNarrow = Packed && NT == 1;  // (wide heads of packed tokens take two tiles)
  switch (a.p.d) {
    case 32: return launch_small<StepOf, 32, NT, Packed>(a, grid, stream);
    case 64: return launch_small<StepOf, 64, NT, Packed>(a, grid, stream);
    case 96: return launch_small<StepOf, 96, NT, Packed>(a, grid, stream);
    default: break;
  }
  if constexpr (!kNarrow) {
    switch (a.p.d) {
      case 128: return launch_small<StepOf, 128, NT, Packed>(a, grid, stream);
      case 160: return launch_small<StepOf, 160, NT, Packed>(a, grid, stream);
      case 192: return launch_small<StepOf, 192, NT, Packed>(a, grid, stream);
      case 224: return launch_small<StepOf, 224, NT, Packed>(a, grid, stream);
      default: return launch_small<StepOf, 256, NT, Packed>(a, grid, stream);
    }
  }
  return hipErrorInvalidValue;
}
template <int NT, bool Packed>
hipError_t launch_small_type(const KvTileArgs& a, unsigned grid, hipStream_t stream) {
  return a.p.dtype == LLA_BF16 ? launch_small_width<NT, Packed, StepBf16>(a, grid, stream)
                               : launch_small_width<NT, Packed, StepF32>(a, grid, stream);
}

}  // namespace lla
