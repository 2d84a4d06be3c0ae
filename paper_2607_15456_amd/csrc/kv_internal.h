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

// How tiles are cut into slices of their pages: slices of a tile at most, pages of a slice
// at least, the workgroups that they are shared out to, the tiles that there is room for
// (more are of offsets that decrease, and left out), and their partial rows.
struct KvTileCut {
  int most, least, wgs, tiles;
  float* part;
};

// Attention of packed tokens (offset, start), and of entries that share a prompt
// (length, lead, shared), over the pages.
struct KvTileArgs {
  KvPages p;
  int out_dtype, B, total, H;
  int n_ctx, sink, window;
  const int32_t* rows;
  const int32_t* offset;
  const int32_t* start;
  const int32_t* length;
  const int32_t* lead;
  const int32_t* shared;
  const void* q;
  int64_t q_t;  // elements from one token's (entry's) queries to the next
  float qscale;
  void* out;
  float* lse;
  KvTileCut small, large;
  // rows up to which a packed entry, or a run of entries that share a prompt, is of small tiles
  int small_rows;
  // rows of a small tile, and at which a run is cut into tiles
  int small_cols, prefix_cols;
  // slices that an entry's own tokens are cut into, at most
  int own_slices;
  float* own_part;
};
// Choose how the work is cut; return the workspace bytes that this takes.
size_t kv_prefill_shape(KvTileArgs& a);
size_t kv_shared_shape(KvTileArgs& a);
// The most that it takes for any smaller call.
size_t kv_prefill_workspace(const KvTileArgs& a);
size_t kv_shared_workspace(const KvTileArgs& a);
hipError_t launch_kv_prefill(const KvTileArgs& a, hipStream_t stream);
hipError_t launch_kv_shared(const KvTileArgs& a, hipStream_t stream);

// Offsets, entries, positions and slots of packed tokens.
struct KvSlotsArgs {
  int B, total, n_seqs, max_pages, n_pages;
  const int32_t* table;
  const int32_t* rows;
  const int32_t* start;
  const int32_t* pos0;  // NULL: start
  const int32_t* n_new;
  int32_t* offset;
  int32_t* entry;
  int32_t* pos;
  int64_t* slot;
};
hipError_t launch_kv_slots(const KvSlotsArgs& a, hipStream_t stream);

// Groups of neighbouring entries with the same leading pages.
struct PagesSharedArgs {
  int B, least, n_seqs, max_pages, n_pages;
  const int32_t* table;
  const int32_t* length;
  const int32_t* rows;
  int32_t* lead;
  int32_t* shared;
};
hipError_t launch_pages_shared(const PagesSharedArgs& a, hipStream_t stream);

// Keys and values of packed tokens to their slots.
struct KvWriteSlotsArgs {
  KvPages p;  // (without a table)
  int total, rot, interleaved;
  const void* k;
  const void* v;
  int64_t kt, vt;
  const double* freq;
  float magnitude;
  const int32_t* pos;
  const int64_t* slot;
};
hipError_t launch_kv_write_slots(const KvWriteSlotsArgs& a, hipStream_t stream);

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
