/*
 * lla_kv.h -- C ABI of the paged K/V cache beside the latent cache of lla.h
 * (same library, liblla.so; AMD Instinct MI355X, gfx950).
 *
 * The latent cache is the paper's capacity path.  Its full-memory path (App. A;
 * tab:memory) attends over whole keys and values, as the teacher does.  These
 * entry points hold such a cache in pages that sequences share through a page
 * table: rotary positions for queries and keys, the write of new tokens, the
 * attention of one new token over the pages, and the pages' bookkeeping on the
 * device (room for new tokens, sharing, copy on write, freeing, keeping a part
 * of the tokens), so that a whole decode step can be captured into a graph.  Steps
 * whose entries bring different numbers of tokens are packed batches, with causal
 * attention over the pages; sequences that share a prompt read it once.
 *
 * lla.h's conventions hold: caller-owned device pointers, 16-byte aligned
 * (index arrays 4-byte); scalar arguments and pointers checked on the host
 * before anything is launched; no allocation, no synchronisation; work enqueued
 * on `stream` of the current device, which must be the pointers' device; dtype
 * is LLA_F32 or LLA_BF16 and sums are fp32; calls are stateless and reentrant,
 * and calls that touch the same pages, tables or workspace must be ordered by
 * the caller.  The contents of index arrays are checked on the device: an index
 * out of its range is never followed, with the effect that each call states.
 *
 * Pages
 * -----
 * A page holds LLA_PAGE_TOKENS = 64 consecutive positions of one sequence for
 * all H_kv key heads of one layer.  A pool of n_pages pages is
 *   keys    [n_pages][H_kv][64][d_head]   element (p, h, t, i) at ((p*H_kv + h)*64 + t)*d_head + i
 *   values  [n_pages][H_kv][d_head][64]   element (p, h, t, i) at ((p*H_kv + h)*d_head + i)*64 + t
 * (keys token-major, values feature-major, as the LLA-2D caches).  d_head is a
 * multiple of 32 in [32, 256].
 *
 * Tables (int32, on the device; one set serves every layer)
 * ----------------------------------------------------------
 *   table   [n_seqs][max_pages]  page of positions 64*i .. 64*i + 63 of a
 *                                sequence; -1 (or anything) past its last page
 *   length  [n_seqs]             its tokens
 *   refs    [n_pages]            how many table entries name a page
 *   free    [1 + n_pages]        free[0] pages are free: free[1 .. free[0]], a
 *                                stack whose last entry is taken first
 * with n_seqs >= 1, 1 <= max_pages <= 2^20, 1 <= n_pages <= 2^30 (all calls).
 * To begin: length and refs 0, free[0] = n_pages, free[1 ..] every page once.
 * A page with refs > 1 is shared; it may be read, and lla_pages_reserve gives a
 * sequence a copy of its own before it is written.
 */
#ifndef LLA_KV_H_
#define LLA_KV_H_

#include "lla.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LLA_KV_ABI_VERSION 3
#define LLA_KV_MAX_ROWS 1024 /* sequences of one reserve, fork or free; entries of a packed or shared batch */
#define LLA_KV_MAX_ROW 512   /* widest row of lla_rope_positions */

/* How rotary frequencies are scaled for contexts past the trained length. */
typedef enum lla_rope_scaling {
  LLA_ROPE_PLAIN = 0,  /* base^(-2i/d_rot) */
  LLA_ROPE_LINEAR = 1, /* position interpolation: every frequency over `factor` */
  LLA_ROPE_NTK = 2,    /* a larger base: base * factor^(d_rot/(d_rot-2)) */
  LLA_ROPE_YARN = 3    /* per wavelength: pairs that turn at least beta_fast times
                          within `original` positions keep their frequency, those
                          that turn at most beta_slow times are interpolated, a
                          linear ramp over the pair index between */
} lla_rope_scaling;

/* Status word of the table calls, result[0] (on the device). */
typedef enum lla_pages_status {
  LLA_PAGES_OK = 0,
  LLA_PAGES_FULL = 1, /* fewer free pages than the call needs */
  LLA_PAGES_BAD = 2   /* a row out of range or named twice (-1 is padding, as often as
                         wanted), a sequence that would outgrow max_pages, a fork onto
                         a sequence that is not empty */
} lla_pages_status;

/* LLA_KV_ABI_VERSION of the built library. */
int lla_kv_abi_version(void);

/*
 * The d_rot/2 angles per position, freq[i] (host memory), and the factor by
 * which turned features are multiplied (1, but 0.1 ln(factor) + 1 for YaRN with
 * factor > 1).  factor, original, beta_fast and beta_slow are read as `scaling`
 * needs them: factor >= 1 finite; original >= 1 and beta_fast > beta_slow > 0
 * for YaRN.  Host only.
 * Requires d_rot a multiple of 8 in [8, LLA_MAX_ROPE], base > 1 finite.
 * Errors: LLA_ERR_INVALID_ARG.
 */
lla_status lla_rope_frequencies(int d_rot, double base, int scaling, double factor, double original,
                                double beta_fast, double beta_slow, double* freq, double* magnitude);

/*
 * Rotary positions of rows x [B][M][H][d_head] into y of the same sizes:
 * features 0 .. d_rot-1 of row (b, m, h) are turned in d_rot/2 pairs, pair i by
 * the angle p * freq[i] and multiplied by `magnitude`; features from d_rot on
 * are copied.  Pair i is features (i, i + d_rot/2), or (2i, 2i + 1) when
 * `interleaved` is not 0.  The position p is
 *   pos0 + m             when pos is NULL,
 *   pos[b] + pos0 + m    when pos_tokens is 0 (pos: int32 [B]),
 *   pos[b*M + m] + pos0  otherwise            (pos: int32 [B][M]).
 * With `transpose` not 0 the angles are negated: magnitude * R^T, which takes
 * the gradient of y to the gradient of x.
 *
 *   freq    device double [d_rot/2] (lla_rope_frequencies)
 *   x_b, x_m, x_h and y_b, y_m, y_h  strides in elements of b, m and h, each a
 *           multiple of 16 bytes (a row's features are dense).  x may be read
 *           with stride 0; y's strides must nest (each at least as wide as what the
 *           smaller ones span); y may be x with the same strides (in place), and
 *           must not overlap it otherwise.
 * Angles are formed and reduced in 64 bits, sine and cosine and the products in
 * 32, rounded once to dtype.
 * Requires B, M >= 1; 1 <= H <= 65535; d_head a multiple of 8 in [8, LLA_KV_MAX_ROW]; d_rot a
 * multiple of 8 in [8, min(d_head, LLA_MAX_ROPE)]; B*M < 2^24, B*M*H < 2^31; magnitude finite.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_rope_positions(int dtype, int B, int M, int H, int d_head, int d_rot, int interleaved,
                              int transpose, const void* x, int64_t x_b, int64_t x_m, int64_t x_h,
                              const int32_t* pos, int pos_tokens, int pos0, const double* freq,
                              float magnitude, void* y, int64_t y_b, int64_t y_m, int64_t y_h,
                              void* stream);

/*
 * Write the keys and values of new tokens into their sequences' pages: token m
 * < n_new[b] of entry b goes to position start[b] + m of sequence rows[b], its
 * key turned there as by lla_rope_positions (d_rot = 0: not turned; freq is
 * then NULL).
 *
 *   k, v    [B][M][H_kv][d_head], heads and features dense, strides k_b, k_m,
 *           v_b, v_m in elements (multiples of 16 bytes): slices of a fused
 *           projection's rows can be passed as they are
 *   rows    int32 [B], or NULL: entry b is sequence b
 *   start   int32 [B] (as lla_pages_reserve gives it: -1 for a refused row)
 *   n_new   int32 [B], or NULL: M tokens each
 *   k_pages, v_pages  one layer's pools
 * Tokens of an entry with start[b] < 0, a row outside [0, n_seqs), a position
 * of 64*max_pages or more, or a page outside [0, n_pages) are not written;
 * n_new[b] counts as at most M and no less than 0.  Slots of other positions
 * are not touched.  Pages written must have one holder, and a position must
 * occur once in a call.
 * Requires B, M >= 1; 1 <= H_kv <= 65535; B*M*H_kv < 2^31, B*(M/64 + 2)*H_kv < 2^24 (whole
 * pages); d_rot as above, or 0.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_kv_write(int dtype, int B, int M, int H_kv, int d_head, int d_rot, int interleaved,
                        const void* k, int64_t k_b, int64_t k_m, const void* v, int64_t v_b,
                        int64_t v_m, const double* freq, float magnitude, int n_seqs, int max_pages,
                        int n_pages, const int32_t* table, const int32_t* rows, const int32_t* start,
                        const int32_t* n_new, void* k_pages, void* v_pages, void* stream);

/*
 * lla_kv_write for sequences whose places in the cache are not their positions, as
 * after lla_kv_gather has kept a part of them: token m goes to place start[b] + m as
 * there, and its key is turned to position pos[b] + m.
 *   pos     int32 [B], or NULL: start
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_kv_write_at(int dtype, int B, int M, int H_kv, int d_head, int d_rot, int interleaved,
                           const void* k, int64_t k_b, int64_t k_m, const void* v, int64_t v_b,
                           int64_t v_m, const double* freq, float magnitude, int n_seqs, int max_pages,
                           int n_pages, const int32_t* table, const int32_t* rows, const int32_t* start,
                           const int32_t* pos, const int32_t* n_new, void* k_pages, void* v_pages,
                           void* stream);

/* Workspace bytes that serve lla_kv_decode_attn for every batch of 1 .. B entries
 * and every bound of 1 .. n_ctx (other arguments the same) on the current device,
 * so that the largest sizes of a program are asked for once: 0 where none of these
 * calls splits a context over workgroups.  Host only.
 * Errors: LLA_ERR_INVALID_ARG. */
lla_status lla_kv_decode_workspace_bytes(int dtype, int B, int H, int H_kv, int d_head, int n_ctx,
                                         int sink, int window, size_t* bytes);

/*
 * Decode attention over the paged cache: entry b is sequence rows[b] with its
 * N = length[rows[b]] tokens, and query head h reads key head h / (H / H_kv):
 *   s_n = scale * q . k_n,   a = softmax(s),   out = sum_n a_n v_n
 * over n < N, and with window > 0 only over n < sink or n >= N - window.
 *
 *   q       [B][H][d_head]
 *   rows    int32 [B], or NULL: entry b is sequence b
 *   n_ctx   upper bound of the lengths, in [1, 64*max_pages]: how many workgroups
 *           may share an entry goes by it; what each takes, by the entry's length
 *   scale   > 0, scale * log2(e) finite in 32 bits (usually 1/sqrt(d_head))
 *   out     [B][H][d_head] of out_dtype
 *   lse     NULL, or float [B][H]: the natural logarithm of sum_n exp(s_n)
 *   workspace  device memory of ws_bytes >= lla_kv_decode_workspace_bytes(), no
 *           initial contents needed and none kept between calls; NULL with ws_bytes == 0
 *           where that is 0 (a call whose own sizes need less takes less)
 * An entry with N = 0 or rows[b] = -1 (padding of a batch) gets zeros and an
 * lse of -inf; another row outside [0, n_seqs), an N outside [0, n_ctx] or a page outside
 * [0, n_pages) among those read gets NaN.  Slots that are not attended may hold anything.
 * Scores times log2(e) have to be finite in 32 bits (or -inf: such a key weighs nothing).
 * An attended value that is not finite makes its feature's results not finite (NaN or
 * infinite), and no other feature's.  Sums hold weights of up to 2^8, so finite values
 * give finite results below 2^120 / N in magnitude.
 * Products of bf16 are exact; the softmax weights enter their product with the
 * values with their 24 bits, as a sum of three bf16.
 * Requires B >= 1, H a multiple of H_kv >= 1, H / H_kv <= 65535, sink >= 0, window >= 0,
 * sink = 0 without a window, B*H < 2^24.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_WORKSPACE, LLA_ERR_HIP.
 */
lla_status lla_kv_decode_attn(int dtype, int out_dtype, int B, int H, int H_kv, int d_head,
                              int n_seqs, int max_pages, int n_pages, int n_ctx, int sink,
                              int window, const int32_t* table, const int32_t* length,
                              const int32_t* rows, const void* q, const void* k_pages,
                              const void* v_pages, float scale, void* out, float* lse,
                              void* workspace, size_t ws_bytes, void* stream);

/*
 * The table calls below run on the device in stream order and take n <= LLA_KV_MAX_ROWS sequences in `rows`
 * (int32 [n]).  Each sets result (int32 [4]) to a lla_pages_status, the number
 * of copy pairs, the pages taken or given back, and the free pages left; with
 * any status but LLA_PAGES_OK it changes nothing else (lla_pages_reserve sets
 * start to -1 as well).  The outcome is that of taking the rows one after
 * another in the order of `rows`, and does not vary between runs.  Rows of -1 (of
 * lla_pages_fork: in dst) are padding, as in lla_kv_write and lla_kv_decode_attn: they
 * are passed over, whatever stands beside them, and get a start of -1, so that a
 * captured step of a fixed number of rows serves fewer sequences.
 */

/*
 * Room for add[i] >= 0 new tokens of sequence rows[i].  If the sequence ends inside a
 * page and that page has other holders (refs > 1 when the row's turn comes), a
 * page of its own takes its place, and (old page, new page) is the next entry
 * of pairs, for lla_pages_copy.  Pages for the new tokens follow, length grows
 * by add[i] and start[i] is the length before.
 *   add, start  int32 [n];  pairs  int32 [n][2]
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_pages_reserve(int n, const int32_t* rows, const int32_t* add, int n_seqs, int max_pages,
                             int n_pages, int32_t* table, int32_t* length, int32_t* refs,
                             int32_t* free_pages, int32_t* start, int32_t* pairs, int32_t* result,
                             void* stream);

/*
 * Sequence dst[i], which must be empty, becomes sequence src[i]: its pages are
 * shared (refs grow), its length is the same.  A source may occur many times and
 * may not be a destination.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_pages_fork(int n, const int32_t* src, const int32_t* dst, int n_seqs, int max_pages,
                          int n_pages, int32_t* table, int32_t* length, int32_t* refs,
                          const int32_t* free_pages, int32_t* result, void* stream);

/*
 * Empty the sequences `rows`: table entries become -1, lengths 0, and pages that
 * nobody holds any more go back to the free stack, the first that was met on
 * top, so that a reserve of the same sizes takes the same pages again.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_pages_free(int n, const int32_t* rows, int n_seqs, int max_pages, int n_pages,
                          int32_t* table, int32_t* length, int32_t* refs, int32_t* free_pages,
                          int32_t* result, void* stream);

/*
 * Copy whole pages pairs[i][0] -> pairs[i][1] in both pools, [layers][n_pages]
 * pages of a_bytes and b_bytes bytes (multiples of 16; b may be NULL with
 * b_bytes 0): keys and values, or latents of one rank each.  With count (a device
 * int32) only the first min(*count, n_pairs) pairs, e.g. result + 1 of
 * lla_pages_reserve.  A pair with a page out of range is passed over.  No page may be
 * written twice, or be read and written, by one call.
 * Requires 1 <= layers <= 65535, 1 <= n_pairs <= 2^20, page sizes of at most 2^40 bytes,
 * n_pairs times the pages' pieces of 8 KB below 2^24.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_pages_copy(int layers, int n_pages, void* a, int64_t a_bytes, void* b, int64_t b_bytes,
                          const int32_t* pairs, int n_pairs, const int32_t* count, void* stream);

/*
 * Keep a part of a sequence's tokens: for i < n_keep[j], position i of sequence
 * dst[j] becomes position keep[j][i] of sequence src[j] (keys as they are
 * stored, so turned at the position they were written for), in pools of
 * [layers][n_pages] pages.  From then on a length counts kept tokens and is no
 * position: the caller keeps the count of all tokens, turns queries to it
 * (lla_rope_positions) and gives it to lla_kv_write_at for the keys.  A start of
 * lla_pages_reserve would put new tokens before kept ones.
 *   src, dst  int32 [B];  keep  int32 [B][max_keep];  n_keep  int32 [B], or NULL: max_keep each
 * dst's pages must be its own and not src's (lla_pages_reserve after
 * lla_pages_fork and lla_pages_free keeps the sequence's number).  A position keep[j][i]
 * outside [0, 64*max_pages) or on a page out of range gives NaN; tokens of a
 * destination row or page out of range are not written.
 * Requires 1 <= layers <= 32767, 1 <= H_kv <= 65535, B >= 1, 1 <= max_keep <= 64*max_pages,
 * B*max_keep <= 2^30, B times the pages of max_keep tokens below 2^24.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_kv_gather(int dtype, int B, int max_keep, int layers, int H_kv, int d_head, int n_seqs,
                         int max_pages, int n_pages, const int32_t* table, const int32_t* src,
                         const int32_t* dst, const int32_t* keep, const int32_t* n_keep,
                         void* k_pages, void* v_pages, void* stream);

/*
 * Packed batches.  The tokens of B <= LLA_KV_MAX_ROWS entries, n_new[b] each, lie one
 * after another in `total` packed rows: entry b's are offset[b] .. offset[b+1] - 1, at
 * places start[b], start[b] + 1, .. of sequence rows[b] (NULL: sequence b), as
 * lla_pages_reserve gives them.  total is the rows that there is room for, so a
 * captured step serves fewer tokens; rows from offset[B] on belong to nobody.
 */

/*
 * Offsets, entries, positions and slots of packed tokens, from request lengths:
 *   offset[b] = min(total, sum of max(0, n_new[i]) over i < b), b = 0 .. B
 * and for token i of entry b, t = offset[b] + i:
 *   entry[t] = b,  pos[t] = pos0[b] + i (pos0 NULL: start),
 *   slot[t] = 64 * page + (start[b] + i) % 64, in the page of that place.
 * Where start[b] < 0 (a refused or padding row), pos and slot are -1; slot is -1, too,
 * where the row is outside [0, n_seqs), the place 64*max_pages or more, or the page
 * outside [0, n_pages), and pos where it is not in [0, 2^31).  Tokens from offset[B] on
 * get -1 in all three.
 *   rows, pos0  int32 [B] or NULL;  start, n_new  int32 [B]
 *   offset  int32 [B + 1];  entry, pos  int32 [total];  slot  int64 [total], 8-byte aligned
 * Requires 1 <= B <= LLA_KV_MAX_ROWS, 1 <= total < 2^24.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_kv_slots(int B, int total, int n_seqs, int max_pages, int n_pages, const int32_t* table,
                        const int32_t* rows, const int32_t* start, const int32_t* pos0,
                        const int32_t* n_new, int32_t* offset, int32_t* entry, int32_t* pos,
                        int64_t* slot, void* stream);

/*
 * Write packed keys and values to their slots: token t's go to place slot[t] % 64 of
 * page slot[t] / 64, its key turned to position pos[t] as by lla_rope_positions
 * (d_rot = 0: not turned; freq is then NULL and pos may be).
 *   k, v    [total][H_kv][d_head], heads and features dense, strides k_t, v_t in elements
 *           (multiples of 16 bytes)
 * Tokens with a slot outside [0, 64*n_pages) are not written, other slots are not
 * touched.  Pages written must have one holder, and a slot must occur once in a call.
 * Requires total >= 1, 1 <= H_kv <= 65535, (total/64 + 1)*H_kv < 2^24; d_rot as above, or 0.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_kv_write_slots(int dtype, int total, int H_kv, int d_head, int d_rot, int interleaved,
                              const void* k, int64_t k_t, const void* v, int64_t v_t,
                              const double* freq, float magnitude, int n_pages, const int64_t* slot,
                              const int32_t* pos, void* k_pages, void* v_pages, void* stream);

/* Workspace bytes that serve lla_kv_prefill_attn for every batch of up to B entries,
 * total tokens and a bound of n_ctx (other arguments the same) on the current device.
 * Host only.
 * Errors: LLA_ERR_INVALID_ARG. */
lla_status lla_kv_prefill_workspace_bytes(int dtype, int out_dtype, int B, int total, int H, int H_kv, int d_head,
                                          int n_ctx, int sink, int window, size_t* bytes);

/*
 * Causal attention of packed tokens over the paged cache: token i of entry b, at place
 * p = start[b] + i of sequence rows[b], attends the places n <= p, and with window > 0
 * of these only n < sink and n > p - window; query head h reads key head h / (H / H_kv).
 * Its own key and value must have been written.  Prompts, pieces of prompts, drafts and
 * single tokens may stand in one batch.
 *
 *   q       [total][H][d_head], heads and features dense, stride q_t in elements (a
 *           multiple of 16 bytes): a slice of a fused projection's rows can be passed
 *   offset  int32 [B + 1], not decreasing (lla_kv_slots); start  int32 [B]
 *   n_ctx   upper bound of the places, in [1, 64*max_pages]
 *   scale   as for lla_kv_decode_attn
 *   out     [total][H][d_head] of out_dtype
 *   lse     NULL, or float [total][H]: the natural logarithm of sum_n exp(s_n)
 *   workspace  device memory of ws_bytes >= lla_kv_prefill_workspace_bytes(), as for
 *           lla_kv_decode_attn
 * Tokens of an entry with rows[b] = -1 or start[b] < 0 get zeros and an lse of -inf;
 * tokens of another row outside [0, n_seqs), at a place of n_ctx or more, or that attend
 * a page outside [0, n_pages) get NaN.  Rows of out and lse that are no entry's are not
 * touched.  What slots after a token hold does not matter to it, in the values of other
 * tokens of its batch too: values that are not finite make results not finite (NaN
 * or infinite) of the tokens that attend them, in their own feature.
 * Offsets that decrease leave some of the tokens undone and do no other harm.
 * bf16: products are exact, and the softmax weights enter their product with the values
 * with their 24 bits, whatever out_dtype: results in bf16 are those in fp32, rounded once.
 * Requires 1 <= B <= LLA_KV_MAX_ROWS, 1 <= total < 2^24, H a multiple of H_kv >= 1,
 * total*H < 2^30, sink >= 0, window >= 0, sink = 0 without a window.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_WORKSPACE, LLA_ERR_HIP.
 */
lla_status lla_kv_prefill_attn(int dtype, int out_dtype, int B, int total, int H, int H_kv, int d_head, int n_seqs,
                               int max_pages, int n_pages, int n_ctx, int sink, int window,
                               const int32_t* table, const int32_t* rows, const int32_t* offset,
                               const int32_t* start, const void* q, int64_t q_t, const void* k_pages,
                               const void* v_pages, float scale, void* out, float* lse,
                               void* workspace, size_t ws_bytes, void* stream);

/*
 * Which neighbours among the entries rows[b] (NULL: sequence b) share leading pages:
 * entry b joins the group of b - 1 when both read the same pages at their first
 * c >= least places (c counts no place past either's length).  For all entries of a
 * group, lead[b] is its first entry and shared[b] the least c of its joins; an entry
 * alone has lead[b] = b and shared[b] = 0.  Families behind one prompt that all have are one
 * group of that prompt unless `least` is above its places.  Sequences that lla_pages_fork made share the
 * pages that they had, until lla_pages_reserve gives one a copy of its last.
 *   rows  int32 [B] or NULL (-1 or out of range: joins nobody);  length  int32 [n_seqs]
 *   lead, shared  int32 [B]
 * Requires 1 <= B <= LLA_KV_MAX_ROWS, least >= 1.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_HIP.
 */
lla_status lla_pages_shared(int B, int least, const int32_t* rows, int n_seqs, int max_pages, int n_pages,
                            const int32_t* table, const int32_t* length, int32_t* lead, int32_t* shared,
                            void* stream);

/* Workspace bytes that serve lla_kv_decode_attn_shared for every batch of up to B
 * entries and a bound of n_ctx (other arguments the same) on the current device.  Host
 * only.
 * Errors: LLA_ERR_INVALID_ARG. */
lla_status lla_kv_shared_workspace_bytes(int dtype, int B, int H, int H_kv, int d_head, int n_ctx, size_t* bytes);

/*
 * lla_kv_decode_attn for entries of which neighbours share a long prompt: the keys and
 * values of entry b's places below shared[b] are those of entry lead[b], and are read
 * through that entry's pages by the queries of neighbours with the same lead and shared
 * together: up to 16 rows (entries times H / H_kv; 32 where H / H_kv is more than 16) read a
 * page at once, in bf16 up to 256 (128 above a d_head of 128) where the batch has enough to
 * do; the places from shared[b] to its length through its own pages.  It pays where neighbours
 * would read some 450 MB more without it; below that lla_kv_decode_attn is faster.  (lla_pages_shared
 * finds both; a program that knows its prompts may give other numbers, down to a place
 * inside a page.)  Arguments and results are otherwise those of lla_kv_decode_attn without
 * a window.
 *   lead, shared  int32 [B]
 * An entry with shared[b] < 0 or above its length, or with shared[b] > 0 and a lead[b]
 * outside [0, B), whose row is out of range, or that has fewer places, gets NaN.
 * Requires 1 <= B <= LLA_KV_MAX_ROWS, and as lla_kv_decode_attn.
 * Errors: LLA_ERR_INVALID_ARG, LLA_ERR_WORKSPACE, LLA_ERR_HIP.
 */
lla_status lla_kv_decode_attn_shared(int dtype, int out_dtype, int B, int H, int H_kv, int d_head, int n_seqs,
                                     int max_pages, int n_pages, int n_ctx, const int32_t* table,
                                     const int32_t* length, const int32_t* rows, const int32_t* lead,
                                     const int32_t* shared, const void* q, const void* k_pages,
                                     const void* v_pages, float scale, void* out, float* lse,
                                     void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LLA_KV_H_ */
