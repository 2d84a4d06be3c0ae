// Decode attention over the paged K/V cache: one query per (entry, query head),
// grouped onto the key heads, over the pages that the page table names.
//
//   s_n = scale q . k_n,  o = sum_n softmax(s)_n v_n
//
// One workgroup per (entry, query head); a wavefront takes every fourth page.
// Scores: a lane per token, 16 bytes of its key row at a time.  Values: a lane
// per feature row, 64 weights from LDS.  A wavefront keeps its own running
// maximum and sum; the four are joined in LDS.

#include "kv_internal.h"
#include "lla_device.h"
#include "../../include/lla_kv.h"

namespace lla {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;

// Pages and tokens that an entry attends: tokens [0, first) and [last, n).
struct Span {
  int n;                // tokens of the sequence
  int first, last;      // first: the sinks
  int lead, skip, pages;  // pages 0 .. lead-1, then lead + skip .. ; their number
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
};

__device__ __forceinline__ void store_row(const KvDecodeArgs& a, int64_t i, float v) {
  if (a.out_dtype == LLA_BF16) store_out(static_cast<bf16_t*>(a.out), i, v);
  else store_out(static_cast<float*>(a.out), i, v);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void decode_simple_kernel(KvDecodeArgs a) {
  __shared__ float s_q[kMaxHead];
  __shared__ float s_p[kWaves][kPage];
  __shared__ float s_o[kWaves][kMaxHead];
  __shared__ float s_m[kWaves], s_l[kWaves];
  __shared__ int s_bad;
  const int b = blockIdx.x / a.H, h = blockIdx.x % a.H, d = a.p.d;
  const int tid = threadIdx.x, lane = tid % kWave, w = tid / kWave;
  const int64_t row_out = (int64_t)blockIdx.x * d;
  const int row = a.rows ? a.rows[b] : b;
  int n = row >= 0 && row < a.p.n_seqs ? a.length[row] : row == -1 ? 0 : -1;
  if (n > a.n_ctx) n = -1;
  if (n <= 0) {
    for (int i = tid; i < d; i += kThreads) store_row(a, row_out + i, n < 0 ? __builtin_nanf("") : 0.f);
    if (a.lse && tid == 0) a.lse[blockIdx.x] = n < 0 ? __builtin_nanf("") : neg_inf();
    return;
  }
  const Span sp(n, a.sink, a.window);
  const int kvh = h / (a.H / a.p.Hkv);
  for (int i = tid; i < d; i += kThreads) s_q[i] = Elem<T>::get(static_cast<const T*>(a.q), row_out + i) * a.qscale;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  float m_run = neg_inf(), l_run = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i = w; i < sp.pages; i += kWaves) {
    const int pg = sp.page(i);
    const int page = a.p.table[(int64_t)row * a.p.max_pages + pg];
    if (page < 0 || page >= a.p.n_pages) {
      s_bad = 1;
      break;
    }
    const int64_t at = ((int64_t)page * a.p.Hkv + kvh) * kPage * d;
    const T* k = static_cast<const T*>(a.p.k) + at + lane * d;
    const T* v = static_cast<const T*>(a.p.v) + at;
    const bool seen = sp.seen(pg * kPage + lane);
    float s = 0.f;
    constexpr int V = Elem<T>::kPer16B;
    for (int j = 0; j < d; j += V) {
      float f[V];
      Elem<T>::unpack(ld16(k + j), f);
      for (int e = 0; e < V; ++e) s += f[e] * s_q[j + e];
    }
    if (!seen) s = neg_inf();
    float mx = s;
    for (int x = 32; x; x >>= 1) mx = fmaxf(mx, xor_shfl(mx, x));
    const float m_new = fmaxf(m_run, mx), m_use = m_new == neg_inf() ? 0.f : m_new;
    const float alpha = exp2f(m_run - m_use), p = exp2f(s - m_use);
    float ps = p;
    for (int x = 32; x; x >>= 1) ps += xor_shfl(ps, x);
    l_run = l_run * alpha + ps;
    m_run = m_new;
    s_p[w][lane] = p;
    __builtin_amdgcn_wave_barrier();
    for (int r = 0; r < 4; ++r) {
      const int f = lane + r * kWave;
      if (f < d) {
        float acc = 0.f;
        for (int t = 0; t < kPage; ++t)
          if (sp.seen(pg * kPage + t)) acc += s_p[w][t] * Elem<T>::get(v, f * kPage + t);
        o[r] = o[r] * alpha + acc;
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
  for (int r = 0; r < 4; ++r)
    if (lane + r * kWave < d) s_o[w][lane + r * kWave] = o[r];
  if (lane == 0) {
    s_m[w] = m_run;
    s_l[w] = l_run;
  }
  __syncthreads();
  float m = neg_inf(), l = 0.f;
  for (int x = 0; x < kWaves; ++x) m = fmaxf(m, s_m[x]);
  const float m_use = m == neg_inf() ? 0.f : m;
  for (int x = 0; x < kWaves; ++x) l += s_l[x] * exp2f(s_m[x] - m_use);
  if (s_bad) l = __builtin_nanf("");
  for (int i = tid; i < d; i += kThreads) {
    float acc = 0.f;
    for (int x = 0; x < kWaves; ++x) acc += s_o[x][i] * exp2f(s_m[x] - m_use);
    store_row(a, row_out + i, acc / l);
  }
  if (a.lse && tid == 0) a.lse[blockIdx.x] = (m_use + log2f(l)) * 0.69314718055994531f;
}

}  // namespace

size_t kv_decode_shape(KvDecodeArgs& a) {
  a.slices = 1;
  a.per = (a.n_ctx + kPage - 1) / kPage;
  return 0;
}

hipError_t launch_kv_decode(const KvDecodeArgs& a, hipStream_t stream) {
  const dim3 grid(a.B * a.H);
  if (a.p.dtype == LLA_BF16) hipLaunchKernelGGL(decode_simple_kernel<bf16_t>, grid, dim3(kThreads), 0, stream, a);
  else hipLaunchKernelGGL(decode_simple_kernel<float>, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace lla
