// C ABI of the paged K/V cache (lla_kv.h): host-side validation and dispatch.
// Every check runs before any launch.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <limits>

#include "../../include/lla_kv.h"
#include "kv_internal.h"

namespace {

constexpr int kMaxPages = 1 << 20;   // pages of one sequence
constexpr int kMaxPool = 1 << 30;    // pages of a pool
constexpr int kMaxGridY = 65535;     // workgroups along a grid's second and third dimension
constexpr int kMaxGridX = (1 << 24) - 1;  // and its first: below 2^32 threads, 256 a workgroup
constexpr double kLog2e = 1.4426950408889634;

bool ptr_ok(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool idx_ok(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool opt_idx_ok(const void* p) { return !p || idx_ok(p); }
bool dtype_ok(int t) { return t == LLA_F32 || t == LLA_BF16; }
int elem_bytes(int t) { return t == LLA_F32 ? 4 : 2; }
bool head_ok(int d) { return d >= 32 && d <= 256 && d % 32 == 0; }
bool rot_ok(int rot, int d) { return rot >= 8 && rot % 8 == 0 && rot <= LLA_MAX_ROPE && rot <= d; }
bool stride_ok(int64_t s, int dtype) { return s >= 0 && s * elem_bytes(dtype) % 16 == 0 && s < ((int64_t)1 << 40); }
bool tables_ok(int n_seqs, int max_pages, int n_pages) {
  return n_seqs >= 1 && max_pages >= 1 && max_pages <= kMaxPages && n_pages >= 1 && n_pages <= kMaxPool;
}
// freq goes with a rotation, is a double array, and stays away without one
bool freq_ok(int rot, const double* f) {
  return rot ? f && (reinterpret_cast<uintptr_t>(f) & 7u) == 0 : f == nullptr;
}
// Whether rows of d elements at these strides (n of each) each have a place of
// their own: every dimension steps over all that the narrower ones span.
bool rows_apart(int d, int n0, int64_t s0, int n1, int64_t s1, int n2, int64_t s2) {
  struct Dim {
    int n;
    int64_t s;
  } dim[3] = {{n0, s0}, {n1, s1}, {n2, s2}};
  std::sort(dim, dim + 3, [](const Dim& a, const Dim& b) { return a.s < b.s; });
  int64_t span = d;
  for (const Dim& x : dim) {
    if (x.n == 1) continue;
    if (x.s < span) return false;
    if (x.s > (std::numeric_limits<int64_t>::max() - span) / x.n) return false;
    span += x.s * (x.n - 1);
  }
  return true;
}
lla_status hip_status(hipError_t e) { return e == hipSuccess ? LLA_OK : LLA_ERR_HIP; }

bool decode_ok(int dtype, int B, int H, int H_kv, int d_head, int n_ctx, int sink, int window) {
  return dtype_ok(dtype) && B >= 1 && H >= 1 && H_kv >= 1 && H % H_kv == 0 && H / H_kv <= kMaxGridY &&
         (int64_t)B * H <= kMaxGridX && head_ok(d_head) && n_ctx >= 1 &&
         n_ctx <= kMaxPages * LLA_PAGE_TOKENS && sink >= 0 && window >= 0 &&
         (window > 0 || sink == 0);
}

lla::KvDecodeArgs decode_args(int dtype, int B, int H, int H_kv, int d_head, int n_ctx, int sink, int window) {
  lla::KvDecodeArgs a{};
  a.p.dtype = dtype;
  a.p.Hkv = H_kv;
  a.p.d = d_head;
  a.B = B;
  a.H = H;
  a.n_ctx = n_ctx;
  a.sink = sink;
  a.window = window;
  return a;
}

lla::TableArgs table_args(int n, const int32_t* rows, int n_seqs, int max_pages, int n_pages, int32_t* table,
                          int32_t* length, int32_t* refs, int32_t* free_pages, int32_t* result) {
  lla::TableArgs a{};
  a.n = n;
  a.n_seqs = n_seqs;
  a.max_pages = max_pages;
  a.n_pages = n_pages;
  a.rows = rows;
  a.table = table;
  a.length = length;
  a.refs = refs;
  a.free_pages = free_pages;
  a.result = result;
  return a;
}
bool table_args_ok(const lla::TableArgs& a) {
  return a.n >= 1 && a.n <= LLA_KV_MAX_ROWS && tables_ok(a.n_seqs, a.max_pages, a.n_pages) && idx_ok(a.rows) &&
         idx_ok(a.table) && idx_ok(a.length) && idx_ok(a.refs) && idx_ok(a.free_pages) && idx_ok(a.result);
}

}  // namespace

extern "C" {

int lla_kv_abi_version(void) { return LLA_KV_ABI_VERSION; }

lla_status lla_rope_frequencies(int d_rot, double base, int scaling, double factor, double original,
                                double beta_fast, double beta_slow, double* freq, double* magnitude) {
  if (!rot_ok(d_rot, d_rot) || !std::isfinite(base) || !(base > 1.0) || scaling < LLA_ROPE_PLAIN ||
      scaling > LLA_ROPE_YARN || !freq || !magnitude)
    return LLA_ERR_INVALID_ARG;
  if (scaling != LLA_ROPE_PLAIN && (!std::isfinite(factor) || !(factor >= 1.0))) return LLA_ERR_INVALID_ARG;
  if (scaling == LLA_ROPE_YARN && (!std::isfinite(original) || !(original >= 1.0) || !std::isfinite(beta_fast) ||
                                   !(beta_slow > 0.0) || !(beta_fast > beta_slow)))
    return LLA_ERR_INVALID_ARG;
  if (scaling == LLA_ROPE_NTK) {
    base *= std::pow(factor, (double)d_rot / (d_rot - 2));
    if (!std::isfinite(base)) return LLA_ERR_INVALID_ARG;
  }
  // YaRN: the (real) pair index that turns r times within `original` positions
  // solves original * base^(-2i/d) = 2 pi r; the ramp runs over whole indices
  const double kTwoPi = 6.283185307179586476925286766559;
  auto index_of = [&](double turns) { return d_rot * std::log(original / (kTwoPi * turns)) / (2.0 * std::log(base)); };
  double low = 0.0, high = 0.0;
  if (scaling == LLA_ROPE_YARN) {
    low = std::max(std::floor(index_of(beta_fast)), 0.0);
    high = std::min(std::ceil(index_of(beta_slow)), d_rot - 1.0);
  }
  for (int i = 0; i < d_rot / 2; ++i) {
    const double f = std::pow(base, -2.0 * i / d_rot);
    freq[i] = f;
    if (scaling == LLA_ROPE_LINEAR) freq[i] = f / factor;
    if (scaling == LLA_ROPE_YARN) {
      const double ramp = std::min(std::max((i - low) / std::max(high - low, 1e-3), 0.0), 1.0);
      freq[i] = f * (1.0 - ramp) + f / factor * ramp;
    }
  }
  *magnitude = scaling == LLA_ROPE_YARN ? 0.1 * std::log(factor) + 1.0 : 1.0;
  return LLA_OK;
}

lla_status lla_rope_positions(int dtype, int B, int M, int H, int d_head, int d_rot, int interleaved,
                              int transpose, const void* x, int64_t x_b, int64_t x_m, int64_t x_h,
                              const int32_t* pos, int pos_tokens, int pos0, const double* freq,
                              float magnitude, void* y, int64_t y_b, int64_t y_m, int64_t y_h,
                              void* stream) {
  if (!dtype_ok(dtype) || B < 1 || M < 1 || H < 1 || d_head < 8 || d_head > LLA_KV_MAX_ROW || d_head % 8 ||
      !rot_ok(d_rot, d_head) || !std::isfinite(magnitude))
    return LLA_ERR_INVALID_ARG;
  if (H > kMaxGridY || (int64_t)B * M > std::min(kMaxGridX, std::numeric_limits<int>::max() / H))
    return LLA_ERR_INVALID_ARG;
  if (!ptr_ok(x) || !ptr_ok(y) || !opt_idx_ok(pos) || !freq_ok(d_rot, freq)) return LLA_ERR_INVALID_ARG;
  for (int64_t s : {x_b, x_m, x_h, y_b, y_m, y_h})
    if (!stride_ok(s, dtype)) return LLA_ERR_INVALID_ARG;
  if (!rows_apart(d_head, B, y_b, M, y_m, H, y_h)) return LLA_ERR_INVALID_ARG;
  if (x == y && ((B > 1 && x_b != y_b) || (M > 1 && x_m != y_m) || (H > 1 && x_h != y_h)))
    return LLA_ERR_INVALID_ARG;
  lla::RotaryArgs a{};
  a.dtype = dtype;
  a.B = B;
  a.M = M;
  a.H = H;
  a.d = d_head;
  a.rot = d_rot;
  a.interleaved = interleaved != 0;
  a.x = x;
  a.xb = x_b;
  a.xm = x_m;
  a.xh = x_h;
  a.pos = pos;
  a.pos_tokens = pos && pos_tokens;  // (without pos, token m is at pos0 + m)
  a.pos0 = pos0;
  a.freq = freq;
  a.magnitude = magnitude;
  a.sign = transpose ? -1.f : 1.f;
  a.y = y;
  a.yb = y_b;
  a.ym = y_m;
  a.yh = y_h;
  return hip_status(lla::launch_rotary(a, static_cast<hipStream_t>(stream)));
}

lla_status lla_kv_write(int dtype, int B, int M, int H_kv, int d_head, int d_rot, int interleaved,
                        const void* k, int64_t k_b, int64_t k_m, const void* v, int64_t v_b,
                        int64_t v_m, const double* freq, float magnitude, int n_seqs, int max_pages,
                        int n_pages, const int32_t* table, const int32_t* rows, const int32_t* start,
                        const int32_t* n_new, void* k_pages, void* v_pages, void* stream) {
  return lla_kv_write_at(dtype, B, M, H_kv, d_head, d_rot, interleaved, k, k_b, k_m, v, v_b, v_m, freq, magnitude,
                         n_seqs, max_pages, n_pages, table, rows, start, nullptr, n_new, k_pages, v_pages, stream);
}

lla_status lla_kv_write_at(int dtype, int B, int M, int H_kv, int d_head, int d_rot, int interleaved,
                           const void* k, int64_t k_b, int64_t k_m, const void* v, int64_t v_b,
                           int64_t v_m, const double* freq, float magnitude, int n_seqs, int max_pages,
                           int n_pages, const int32_t* table, const int32_t* rows, const int32_t* start,
                           const int32_t* pos, const int32_t* n_new, void* k_pages, void* v_pages, void* stream) {
  if (!dtype_ok(dtype) || B < 1 || M < 1 || H_kv < 1 || H_kv > kMaxGridY || (int64_t)B * M > std::numeric_limits<int>::max() / H_kv ||
      (int64_t)B * (M / LLA_PAGE_TOKENS + 2) > kMaxGridX / H_kv || !head_ok(d_head) || (d_rot && !rot_ok(d_rot, d_head)) || !std::isfinite(magnitude) ||
      !tables_ok(n_seqs, max_pages, n_pages))
    return LLA_ERR_INVALID_ARG;
  if (!ptr_ok(k) || !ptr_ok(v) || !freq_ok(d_rot, freq) || !idx_ok(table) || !opt_idx_ok(rows) || !idx_ok(start) ||
      !opt_idx_ok(pos) || !opt_idx_ok(n_new) || !ptr_ok(k_pages) || !ptr_ok(v_pages))
    return LLA_ERR_INVALID_ARG;
  for (int64_t s : {k_b, k_m, v_b, v_m})
    if (!stride_ok(s, dtype)) return LLA_ERR_INVALID_ARG;
  lla::KvWriteArgs a{};
  a.p = {dtype, H_kv, d_head, n_seqs, max_pages, n_pages, table, k_pages, v_pages};
  a.B = B;
  a.M = M;
  a.rot = d_rot;
  a.interleaved = interleaved != 0;
  a.k = k;
  a.v = v;
  a.kb = k_b;
  a.km = k_m;
  a.vb = v_b;
  a.vm = v_m;
  a.freq = freq;
  a.magnitude = magnitude;
  a.rows = rows;
  a.start = start;
  a.pos = pos;
  a.n_new = n_new;
  return hip_status(lla::launch_kv_write(a, static_cast<hipStream_t>(stream)));
}

lla_status lla_kv_decode_workspace_bytes(int dtype, int B, int H, int H_kv, int d_head, int n_ctx,
                                         int sink, int window, size_t* bytes) {
  if (!decode_ok(dtype, B, H, H_kv, d_head, n_ctx, sink, window) || !bytes) return LLA_ERR_INVALID_ARG;
  *bytes = lla::kv_decode_workspace(decode_args(dtype, B, H, H_kv, d_head, n_ctx, sink, window));
  return LLA_OK;
}

lla_status lla_kv_decode_attn(int dtype, int out_dtype, int B, int H, int H_kv, int d_head,
                              int n_seqs, int max_pages, int n_pages, int n_ctx, int sink,
                              int window, const int32_t* table, const int32_t* length,
                              const int32_t* rows, const void* q, const void* k_pages,
                              const void* v_pages, float scale, void* out, float* lse,
                              void* workspace, size_t ws_bytes, void* stream) {
  if (!decode_ok(dtype, B, H, H_kv, d_head, n_ctx, sink, window) || !dtype_ok(out_dtype) ||
      !tables_ok(n_seqs, max_pages, n_pages) || n_ctx > (int64_t)max_pages * LLA_PAGE_TOKENS ||
      !std::isfinite((float)(scale * kLog2e)) || !(scale > 0.f))
    return LLA_ERR_INVALID_ARG;
  if (!idx_ok(table) || !idx_ok(length) || !opt_idx_ok(rows) || !ptr_ok(q) || !ptr_ok(k_pages) || !ptr_ok(v_pages) ||
      !ptr_ok(out) || !opt_idx_ok(lse))
    return LLA_ERR_INVALID_ARG;
  lla::KvDecodeArgs a = decode_args(dtype, B, H, H_kv, d_head, n_ctx, sink, window);
  const size_t need = lla::kv_decode_shape(a);
  if ((workspace == nullptr) != (ws_bytes == 0) || ws_bytes < need ||
      (workspace && (reinterpret_cast<uintptr_t>(workspace) & 15u)))
    return LLA_ERR_WORKSPACE;
  a.p = {dtype, H_kv, d_head, n_seqs, max_pages, n_pages, table, const_cast<void*>(k_pages),
         const_cast<void*>(v_pages)};
  a.out_dtype = out_dtype;
  a.length = length;
  a.rows = rows;
  a.q = q;
  a.qscale = (float)((double)scale * kLog2e);
  a.out = out;
  a.lse = lse;
  a.part = static_cast<float*>(workspace);
  return hip_status(lla::launch_kv_decode(a, static_cast<hipStream_t>(stream)));
}

lla_status lla_pages_reserve(int n, const int32_t* rows, const int32_t* add, int n_seqs, int max_pages,
                             int n_pages, int32_t* table, int32_t* length, int32_t* refs,
                             int32_t* free_pages, int32_t* start, int32_t* pairs, int32_t* result,
                             void* stream) {
  lla::TableArgs a = table_args(n, rows, n_seqs, max_pages, n_pages, table, length, refs, free_pages, result);
  if (!table_args_ok(a) || !idx_ok(add) || !idx_ok(start) || !idx_ok(pairs)) return LLA_ERR_INVALID_ARG;
  a.more = add;
  a.start = start;
  a.pairs = pairs;
  return hip_status(lla::launch_pages_reserve(a, static_cast<hipStream_t>(stream)));
}

lla_status lla_pages_fork(int n, const int32_t* src, const int32_t* dst, int n_seqs, int max_pages,
                          int n_pages, int32_t* table, int32_t* length, int32_t* refs,
                          const int32_t* free_pages, int32_t* result, void* stream) {
  lla::TableArgs a = table_args(n, dst, n_seqs, max_pages, n_pages, table, length, refs,
                                const_cast<int32_t*>(free_pages), result);
  if (!table_args_ok(a) || !idx_ok(src)) return LLA_ERR_INVALID_ARG;
  a.more = src;
  return hip_status(lla::launch_pages_fork(a, static_cast<hipStream_t>(stream)));
}

lla_status lla_pages_free(int n, const int32_t* rows, int n_seqs, int max_pages, int n_pages,
                          int32_t* table, int32_t* length, int32_t* refs, int32_t* free_pages,
                          int32_t* result, void* stream) {
  lla::TableArgs a = table_args(n, rows, n_seqs, max_pages, n_pages, table, length, refs, free_pages, result);
  if (!table_args_ok(a)) return LLA_ERR_INVALID_ARG;
  return hip_status(lla::launch_pages_free(a, static_cast<hipStream_t>(stream)));
}

lla_status lla_pages_copy(int layers, int n_pages, void* a, int64_t a_bytes, void* b, int64_t b_bytes,
                          const int32_t* pairs, int n_pairs, const int32_t* count, void* stream) {
  const int64_t kMost = (int64_t)1 << 40;
  if (layers < 1 || layers > kMaxGridY || n_pages < 1 || n_pages > kMaxPool || n_pairs < 1 || n_pairs > (1 << 20) ||
      a_bytes < 16 || a_bytes % 16 || a_bytes > kMost || b_bytes < 0 || b_bytes % 16 || b_bytes > kMost ||
      (b == nullptr) != (b_bytes == 0))
    return LLA_ERR_INVALID_ARG;
  if (!ptr_ok(a) || (b && !ptr_ok(b)) || !idx_ok(pairs) || !opt_idx_ok(count)) return LLA_ERR_INVALID_ARG;
  if (lla::page_copy_pieces(a_bytes, b_bytes) > kMaxGridX / n_pairs) return LLA_ERR_INVALID_ARG;
  lla::PageCopyArgs c{};
  c.layers = layers;
  c.n_pages = n_pages;
  c.n_pairs = n_pairs;
  c.pool[0] = a;
  c.pool[1] = b;
  c.bytes[0] = a_bytes;
  c.bytes[1] = b_bytes;
  c.pairs = pairs;
  c.count = count;
  return hip_status(lla::launch_pages_copy(c, static_cast<hipStream_t>(stream)));
}

lla_status lla_kv_gather(int dtype, int B, int max_keep, int layers, int H_kv, int d_head, int n_seqs,
                         int max_pages, int n_pages, const int32_t* table, const int32_t* src,
                         const int32_t* dst, const int32_t* keep, const int32_t* n_keep,
                         void* k_pages, void* v_pages, void* stream) {
  if (!dtype_ok(dtype) || B < 1 || max_keep < 1 || layers < 1 || layers > kMaxGridY / 2 || H_kv < 1 ||
      H_kv > kMaxGridY ||
      !head_ok(d_head) || !tables_ok(n_seqs, max_pages, n_pages) ||
      max_keep > (int64_t)max_pages * LLA_PAGE_TOKENS || (int64_t)B * max_keep > (1 << 30) ||
      (max_keep + LLA_PAGE_TOKENS - 1) / LLA_PAGE_TOKENS > kMaxGridX / B)
    return LLA_ERR_INVALID_ARG;
  if (!idx_ok(table) || !idx_ok(src) || !idx_ok(dst) || !idx_ok(keep) || !opt_idx_ok(n_keep) || !ptr_ok(k_pages) ||
      !ptr_ok(v_pages))
    return LLA_ERR_INVALID_ARG;
  lla::KvGatherArgs a{};
  a.p = {dtype, H_kv, d_head, n_seqs, max_pages, n_pages, table, k_pages, v_pages};
  a.B = B;
  a.max_keep = max_keep;
  a.layers = layers;
  a.src = src;
  a.dst = dst;
  a.keep = keep;
  a.n_keep = n_keep;
  return hip_status(lla::launch_kv_gather(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
