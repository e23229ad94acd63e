/*
 * toolspec_ops.h - operators on DEVICE memory, next to the whole passes of toolspec.h: 4-bit
 * microscaled weights (quantisation and product), and one layer's step of the paged cache
 * (append with rotary embedding, attention of one new token) for programs that run decoder
 * blocks of their own over the library's caches or over pages they allocate themselves.
 *
 * Conventions
 *  - Pointers are DEVICE pointers unless a parameter says "host"; they must all belong to one
 *    GPU, which need not be the current one.  16-byte aligned buffers with rows a multiple of 16
 *    bytes apart take vector accesses; other alignments (down to the element) and row strides
 *    give the same results more slowly.  Buffers written must not overlap those read, except
 *    where a parameter says so.
 *  - Every call is enqueued on `stream` (a hipStream_t of that GPU; NULL is its default
 *    stream), returns without waiting, allocates nothing and may be captured into a HIP graph;
 *    whatever the kernels read (lengths, tables, offsets) is read when they run, so a captured
 *    step may be replayed with other contents.  Two calls that may overlap in time need
 *    different workspaces and outputs.
 *  - Return values and ts_last_error() as in toolspec.h.  Nothing is enqueued on an error.
 *  - Values read from device memory cannot be checked by the host: each call says what it does
 *    with a page, length or offset that makes no sense.  None is followed out of bounds.
 *  - dtype is TS_DTYPE_F32 or TS_DTYPE_BF16; strides count elements.
 */
#ifndef TOOLSPEC_OPS_H
#define TOOLSPEC_OPS_H

#include "toolspec.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef void* ts_stream; /* hipStream_t */

/* ---- 4-bit microscaled values -------------------------------------------------
 * A row is cut into blocks of 32 (the last may be shorter).  With a = the largest magnitude of
 * a block its scale is 2^e, e = floor(log2 a) - 2 limited to [-127, 127] (all zeros: -127); a
 * value x is held as the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 to |x| / 2^e (ties to the even
 * code, beyond 6: 6) with its sign: code 0..7 in that order, + 8 if negative.  A block with an
 * infinity or NaN has scale byte 255 and all its values are NaN.
 *   codes  : [rows][blocks][16] bytes, element 2 i of a block in the low half of byte i
 *   scales : [rows][blocks] bytes, e + 127;   blocks = ceil(cols / 32)
 * Positions of the last block behind the row's end get code 0.
 * Errors: INVALID_ARG (null, dtype, negative sizes, row_stride < cols, misaligned codes: 16
 * bytes; host pointers, pointers of different GPUs), DEVICE.  rows or cols 0: nothing to do. */
ts_status ts_mx_quantize(const void* x, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride,
                         uint8_t* codes, uint8_t* scales, ts_stream stream);
/* The values again, in fp32 or bf16 (both hold every one of them exactly; with scale bytes 253 and 254,
 * which ts_mx_quantize never writes, magnitudes from 2^128 on come back infinite, and their products
 * are infinite or NaN). */
ts_status ts_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols,
                           void* x, int32_t dtype, int64_t row_stride, ts_stream stream);

/* A weight matrix [n_out][n_in] laid out for the product, once: ts_mx_packed_bytes bytes,
 * 16-byte aligned, written by ts_mx_pack from codes and scales (which may be freed then).
 * Errors: as above; n_out in [1, 2^24], n_in in [1, 2^22]. */
ts_status ts_mx_packed_bytes(int32_t n_out, int32_t n_in, uint64_t* bytes);
ts_status ts_mx_pack(const uint8_t* codes, const uint8_t* scales, int32_t n_out, int32_t n_in, void* packed, ts_stream stream);

/* y[r][n] = sum_k x[r][k] W[n][k]: x [rows][n_in] and y [rows][n_out] of the same dtype.  The
 * products are exact (a weight has two significant bits; fp32 rows enter as three bf16 terms of
 * one sign that add up to them, up to the largest finite number; bits below 2^-133 are lost, so
 * magnitudes below 2^-110 have fewer than 24), the sums are fp32, y is rounded once.  The order of the sums depends on
 * the sizes only, never on the contents, the device's load or the other rows.
 * A row's result does not depend on the other rows' values.
 * Errors: INVALID_ARG as above (rows in [0, 2^19], strides at least the row,
 * x_stride at most 2^22). */
ts_status ts_mx_project(const void* packed, int32_t n_out, int32_t n_in, const void* x, int32_t dtype, int64_t rows,
                        int64_t x_stride, void* y, int64_t y_stride, ts_stream stream);

/* ---- one layer of a paged cache ------------------------------------------------
 * Pages of 16 positions: keys [n_pages][n_kv_heads][16][head_dim], values transposed within the
 * page, [n_pages][n_kv_heads][head_dim][16], both 16-byte aligned.  dtype BF16: head_dim 64 or
 * 128; F32: a power of two in [8, 128].  Position p of sequence s lies on page
 * table[s * table_stride + p / 16], p / 16 < table_width. */
typedef struct {
  void* k; void* v;
  int32_t n_pages, n_kv_heads, head_dim, dtype;
} ts_kv_pages;

/* One layer of a cache of toolspec.h (of the whole pool if it draws from one), its page table
 * (host_pages: ceil(capacity / 16) ints), and its committed length grown by n_pos positions that
 * the caller has written (every layer) by ts_kv_append on `stream`: waits for that stream, then
 * len += n_pos; an unapplied verify result is dropped, the pending token stays.  The library's own
 * passes run on the model's stream: they see what was appended before ts_kv_extend returned.
 * Passes of bf16 models read whole blocks of 64 positions in IEEE half: what the pages of their caches
 * hold has to be finite and at most 65504 in magnitude, also behind the length (pages come zeroed); a
 * pass that meets a NaN has no next token (see ts_verify).
 * Errors: INVALID_ARG (also a stream of another GPU), KV_CAPACITY (length + n_pos beyond the capacity), DEVICE. */
ts_status ts_kv_layer_pages(const ts_kv* kv, int32_t layer, ts_kv_pages* pages);
ts_status ts_kv_page_table(const ts_kv* kv, int32_t* host_pages, int32_t n_pages);
ts_status ts_kv_extend(ts_kv* kv, int32_t n_pos, ts_stream stream);

/* Appends new rows to the cache.  Rows [row_offsets[s], row_offsets[s + 1]) belong to sequence s
 * and get positions lengths[s], lengths[s] + 1, ... .  Keys are stored rotated (pair
 * (j, j + head_dim / 2) by position * rope_theta^(-2 j / head_dim), an angle that is good to 1e-7
 * radians at any position; rope_theta 0: not rotated),
 * values as they are, both in the cache's dtype; with q, the rotated queries go to q_out (which
 * may be q).  Rows outside every sequence, and rows whose position is negative, beyond the table
 * or on a page outside [0, n_pages), leave cache and q_out as they were.  Lengths are not
 * changed.  Two sequences must not have a page that both write in common.
 *   row_offsets : [n_seqs + 1], non-decreasing;  lengths : [n_seqs]
 *   q, k, v     : rows of n_q_heads resp. n_kv_heads heads of head_dim, in `dtype`, with their
 *                 own strides (slices of one projection's rows will do); q and q_out may be null
 * Errors: INVALID_ARG (also n_seqs in [1, 2^20], n_rows in [0, 2^23]), DEVICE. */
typedef struct {
  ts_kv_pages pages;
  const int32_t* table; int64_t table_stride; int32_t table_width;
  const int32_t* lengths; const int32_t* row_offsets;
  int32_t n_seqs, n_rows, n_q_heads, dtype;
  const void* q; int64_t q_stride;
  const void* k; int64_t k_stride;
  const void* v; int64_t v_stride;
  void* q_out; int64_t q_out_stride;
  float rope_theta;
} ts_kv_append_args;
ts_status ts_kv_append(const ts_kv_append_args* args, ts_stream stream);

/* Attention of one token per sequence over the cache: out[s][h] = sum_p w_p v_p, w = softmax of
 * scale * (q[s][h] . k_p) over the positions p < lengths[s], with window > 0 only the last
 * `window` of them; query head h reads KV head h / (n_q_heads / n_kv_heads).  A position on a
 * page outside [0, n_pages), beyond the table or not below max_len is not seen; contents of
 * positions that are not seen have no influence, whatever they are.  Where nothing is seen, or
 * every score is -infinity, out is 0 and lse -infinity; a score of +infinity or NaN makes its
 * head NaN, an infinite value its dimension infinite.
 * Scores, probabilities, sums and outputs are fp32 (over a bf16 cache fp32 queries and the
 * probabilities enter the products as three bf16 terms, 24 bits, those below 2^-133 lost); out is
 * rounded once, to q's dtype.
 *   max_len  : no length is above it (sizes the launch: the bound of the step, not the capacity)
 *   q, out   : [n_seqs] rows of n_q_heads * head_dim, in `dtype`
 *   lse      : natural logarithm of the sum of exp(scores), [n_seqs][n_q_heads] fp32; may be null
 *   workspace: ts_kv_attend_workspace bytes for the same sizes, 16-byte aligned, contents irrelevant
 *              (null where that is 0)
 * Errors: INVALID_ARG (also n_q_heads not a multiple of n_kv_heads, n_seqs in [1, 2^20], max_len in
 * [0, 2^30], window < 0, scale not finite, workspace too small, n_seqs * n_q_heads or the
 * workgroups beyond 2^24), DEVICE. */
typedef struct {
  ts_kv_pages pages;
  const int32_t* table; int64_t table_stride; int32_t table_width;
  const int32_t* lengths;
  int32_t n_seqs, max_len, window, n_q_heads, dtype;
  const void* q; int64_t q_stride;
  void* out; int64_t out_stride;
  float* lse;
  float scale;
  void* workspace; uint64_t workspace_bytes;
} ts_kv_attend_args;
ts_status ts_kv_attend(const ts_kv_attend_args* args, ts_stream stream);
/* Bytes of workspace a call with these sizes needs; never decreases with max_len at the same other
 * sizes, so the bytes for a longer max_len serve a shorter one. */
ts_status ts_kv_attend_workspace(int32_t n_seqs, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t max_len,
                                 int32_t window, uint64_t* bytes);

#ifdef __cplusplus
}
#endif
#endif /* TOOLSPEC_OPS_H */
