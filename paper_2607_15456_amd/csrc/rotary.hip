// Rotary positions of query or key rows in either pairing, over part of the
// head, with given frequencies; with the sign of the angle turned, the
// transposed rotation of a backward pass.
//
//   y[pair i] = magnitude * R(p * freq[i]) x[pair i],   y[rest] = x[rest]
//
// Bound by memory: 6 flops a pair against 8 bytes in bf16.  A workgroup takes a
// stretch of y: all heads of a token or two (or all tokens of a head, where y's
// heads are the outer dimension), a part of a row a thread.  What decides is that
// neighbouring threads touch neighbouring bytes: with a thread per part of a token
// and its heads one after another, 4 x 8192 tokens of 16 heads of 128, bf16, into a
// result that no cache holds took 73 us; now 50 (5.3 TB/s; a large copy runs at
// 5.0); two parts a thread 52, eight 74; non-temporal stores 48, but what reads
// the result next would miss the caches.  The angles of the workgroup's tokens are
// formed once, into LDS, while the rows are on their way.  One decode step's queries
// (32 x 16 heads) 3 to 4 us, a launch and a chain of two reads.

#include <algorithm>

#include "kv_internal.h"
#include "rotary.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 16;  // of a workgroup, at most

template <typename T, int N, bool Interleaved>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a, int parts, int tokens, int heads) {
  extern __shared__ __align__(16) float2 s_cs[];  // [tokens][pairs] magnitude (cos, sin)
  const int tid = threadIdx.x, pairs = a.rot / 2;
  const uint32_t t0 = blockIdx.x * tokens;  // (B M < 2^31)
  const int nt = min(tokens, (int)((uint32_t)a.B * a.M - t0));
  const int h0 = blockIdx.y * heads, nh = min(heads, a.H - h0);
  // position and frequency of pair i of the workgroup's; the first are read before
  // the rows, whose arrival they would otherwise wait for
  int64_t pos = 0;
  double freq = 0.0;
  auto read = [&](int i) {
    const int at = i / pairs;
    const uint32_t w = t0 + at, wb = w / (uint32_t)a.M;
    int given = 0;
    if (a.pos) given = a.pos[a.pos_tokens ? w : wb];
    freq = a.freq[i - at * pairs];
    pos = (int64_t)a.pos0 + (a.pos_tokens ? 0 : w - wb * a.M) + given;
  };
  if (tid < nt * pairs) read(tid);

  // this thread's token, head and part (the last threads of a workgroup may have none)
  const int items = nt * nh * parts, e = min(tid, items - 1), row = e / parts;
  const bool heads_inside = a.yh <= a.ym;
  const int in = heads_inside ? nh : nt, outer = row / in, inner = row - outer * in;
  const int tok = heads_inside ? outer : inner, head = h0 + (heads_inside ? inner : outer);
  const uint32_t t = t0 + tok, b = t / (uint32_t)a.M, m = t - b * a.M;
  Part<T, N, Interleaved> p(e - row * parts, a.rot, a.d);
  p.load(static_cast<const T*>(a.x) + b * a.xb + m * a.xm + head * a.xh);

  for (int i = tid; i < nt * pairs;) {
    float c, s;
    cos_sin((double)pos * freq, c, s);
    s_cs[i] = make_float2(a.magnitude * c, a.magnitude * a.sign * s);
    i += kThreads;
    if (i < nt * pairs) read(i);
  }
  __syncthreads();
  if (tid >= items) return;
  if (p.turned) {
    Turn<N> turn;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float2 cs = s_cs[tok * pairs + p.pair(i)];
      turn.c[i] = cs.x;
      turn.s[i] = cs.y;
    }
    p.turn(turn);
  }
  p.store(static_cast<T*>(a.y) + b * a.yb + m * a.ym + head * a.yh);
}

template <typename T, int N, bool Interleaved>
hipError_t launch(const RotaryArgs& a, hipStream_t stream) {
  const int parts = Part<T, N, Interleaved>::count(a.rot, a.x == a.y ? 0 : a.d - a.rot);
  const int64_t all = (int64_t)a.B * a.M;
  // a stretch of at most kThreads parts, the inner of tokens and heads first
  const int rows = kThreads / parts;
  int heads, tokens;
  if (a.yh <= a.ym) {
    heads = std::min(a.H, rows);
    tokens = (int)std::min<int64_t>({all, kTokens, rows / heads});
  } else {
    tokens = (int)std::min<int64_t>({all, kTokens, rows});
    heads = std::min(a.H, rows / tokens);
  }
  hipLaunchKernelGGL((rotary_kernel<T, N, Interleaved>),
                     dim3((unsigned)((all + tokens - 1) / tokens), (a.H + heads - 1) / heads), dim3(kThreads),
                     (size_t)tokens * (a.rot / 2) * sizeof(float2), stream, a, parts, tokens, heads);
  return hipGetLastError();
}

template <typename T, bool Interleaved>
hipError_t launch(const RotaryArgs& a, hipStream_t stream) {
  // pairs of a thread: 16 bytes of each half of a bf16 row where rot/2 allows it
  if constexpr (sizeof(T) == 2) {
    if (a.rot % 16 == 0) return launch<T, 8, Interleaved>(a, stream);
  }
  return launch<T, 4, Interleaved>(a, stream);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  if (a.dtype == LLA_BF16) return a.interleaved ? launch<bf16_t, true>(a, stream) : launch<bf16_t, false>(a, stream);
  return a.interleaved ? launch<float, true>(a, stream) : launch<float, false>(a, stream);
}

}  // namespace lla
