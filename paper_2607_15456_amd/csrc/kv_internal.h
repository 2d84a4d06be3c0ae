// Internal launch interface between the C ABI of the paged K/V cache
// (kv_api.cpp) and its kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lla {

// Rotary positions of rows [B][M][H][d] (strides in elements).
struct RotaryArgs {
  int dtype, B, M, H, d, rot, interleaved;
  const void* x;
  int64_t xb, xm, xh;
  const int32_t* pos;
  int pos_tokens, pos0;
  const double* freq;
  float magnitude, sign;  // sign -1: the transposed rotation
  void* y;
  int64_t yb, ym, yh;
};
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream);

// One layer's pools and the page table.
struct KvPages {
  int dtype, Hkv, d;
  int n_seqs, max_pages, n_pages;
  const int32_t* table;
  void* k;
  void* v;
};

struct KvWriteArgs {
  KvPages p;
  int B, M, rot, interleaved;
  const void* k;
  const void* v;
  int64_t kb, km, vb, vm;
  const double* freq;
  float magnitude;
  const int32_t* rows;
  const int32_t* start;
  const int32_t* pos;  // NULL: start
  const int32_t* n_new;
};
hipError_t launch_kv_write(const KvWriteArgs& a, hipStream_t stream);

struct KvDecodeArgs {
  KvPages p;
  int out_dtype, B, H;
  int n_ctx, sink, window;
  // workgroups per (entry, key head, query tile); pages that a slice takes of the
  // longest entry that n_ctx allows, and of any entry at least
  int slices, per, least;
  unsigned inverse;  // 2^32 / slices, rounded up
  const int32_t* length;
  const int32_t* rows;
  const void* q;
  float qscale;  // softmax scale * log2(e)
  void* out;
  float* lse;
  float* part;
};
hipError_t launch_kv_decode(const KvDecodeArgs& a, hipStream_t stream);
// Chooses slices, per, least and inverse; returns the workspace bytes that this takes.
size_t kv_decode_shape(KvDecodeArgs& a);
// The most that it takes for any B and n_ctx up to a's.
size_t kv_decode_workspace(const KvDecodeArgs& a);

struct TableArgs {
  int n, n_seqs, max_pages, n_pages;
  const int32_t* rows;
  const int32_t* more;  // reserve: add; fork: src
  int32_t* table;
  int32_t* length;
  int32_t* refs;
  int32_t* free_pages;
  int32_t* start;
  int32_t* pairs;
  int32_t* result;
};
hipError_t launch_pages_reserve(const TableArgs& a, hipStream_t stream);
hipError_t launch_pages_fork(const TableArgs& a, hipStream_t stream);
hipError_t launch_pages_free(const TableArgs& a, hipStream_t stream);

struct PageCopyArgs {
  int layers, n_pages, n_pairs;
  void* pool[2];
  int64_t bytes[2];
  const int32_t* pairs;
  const int32_t* count;
};
hipError_t launch_pages_copy(const PageCopyArgs& a, hipStream_t stream);
// Workgroups of a pair and layer for pages of these sizes.
int64_t page_copy_pieces(int64_t a_bytes, int64_t b_bytes);

struct KvGatherArgs {
  KvPages p;
  int B, max_keep, layers;
  const int32_t* src;
  const int32_t* dst;
  const int32_t* keep;
  const int32_t* n_keep;
};
hipError_t launch_kv_gather(const KvGatherArgs& a, hipStream_t stream);

int device_cu_count();

}  // namespace lla
