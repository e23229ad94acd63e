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
 * radians up to position 2^25, and to 5e-7 at any; rope_theta 0: not rotated),
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

/* ---- more rows, other rotations, 8-bit pages ---------------------------------------
 * Pages of dtype TS_DTYPE_E4M3 (for the calls below only; head_dim 64 or 128) hold one byte per value, laid out as other
 * pages are (keys [n_pages][n_kv_heads][16][head_dim], values [n_pages][n_kv_heads][head_dim][16]): OCP e4m3, four
 * significant bits, largest 448.  k_scales and v_scales, [n_pages][n_kv_heads][16] bytes each, 16-byte aligned, hold e + 127
 * for each position's row of a head, and a value stands for its e4m3 value times 2^e: e is the least that keeps the row's
 * largest magnitude at or below 448 * 2^e, and at least -127 (all zeros: -127); values are rounded to nearest, ties to
 * even.  A row with an infinity or NaN has scale byte 255 and all its values are NaN.  Values whose magnitude 2^e takes to 2^128 and
 * beyond (rows with magnitudes above 31/32 of 2^128, or scales that a program wrote itself) are infinite; in products and as bf16 bits
 * below 2^-133 are lost.  For pages of other types the two are null. */
enum { TS_DTYPE_E4M3 = 3 };
typedef struct {
  ts_kv_pages pages;
  uint8_t* k_scales; uint8_t* v_scales;
} ts_kv_pages_any;

/* ts_kv_append for decoder blocks that norm the heads of queries and keys, turn them otherwise, or keep 8-bit pages.  Rows, offsets,
 * lengths, tables and places as there (q_out may be q).  A head of a query or key is, in fp32 and in this order
 *   normed  : x / sqrt(mean of x^2 + norm_eps) * gain, where there is a gain: q_norm, k_norm, [head_dim] of norm_dtype, each
 *             may be null
 *   rotated : its first rope_dim values (even, at most head_dim; 0: none) in pairs - (j, j + rope_dim / 2), or (2 j, 2 j + 1)
 *             with rope_pairs != 0 - by the angle position * f_j, and multiplied by rope_magnitude; the other values stay.
 *             f_j = rope_freqs[j], rope_dim / 2 floats in radians per position (a table scaled for long contexts, say), or
 *             rope_theta^(-2 j / rope_dim) where that is null (rope_theta 0: not rotated).  The angle is as good as that of ts_kv_append
 *             (a table's entries are taken as exact).
 * and then rounded once, to its place.  The position of the angle is that of the row, or positions[row] where that is not null
 * (a draft tree's rows lie one behind the other and are turned by their depths); the row's place is not changed by it.
 * A head whose squares overflow fp32 is normed to zeros; with norm_eps 0 one whose squares all vanish in fp32 becomes infinite, or NaN where it is
 * zero; NaN stays NaN.  Where nothing of this is asked for, ts_kv_append does the same in less time.
 * Errors: INVALID_ARG (as ts_kv_append; scales missing or misaligned, rope_dim, norm_eps negative or not finite, rope_magnitude not finite,
 * misaligned gains, frequencies or positions), DEVICE. */
typedef struct {
  ts_kv_pages_any cache;
  const int32_t* table; int64_t table_stride; int32_t table_width;
  const int32_t* lengths; const int32_t* row_offsets; const int32_t* positions;
  int32_t n_seqs, n_rows, n_q_heads, dtype;
  const void* q; int64_t q_stride;
  const void* k; int64_t k_stride;
  const void* v; int64_t v_stride;
  void* q_out; int64_t q_out_stride;
  const void* q_norm; const void* k_norm;
  int32_t norm_dtype; float norm_eps;
  const float* rope_freqs;
  float rope_theta, rope_magnitude;
  int32_t rope_dim, rope_pairs;
} ts_kv_append_norm_rope_args;
ts_status ts_kv_append_norm_rope(const ts_kv_append_norm_rope_args* args, ts_stream stream);

/* Positions of a cache given back as rows: row row_offsets[s] + i of k_out and v_out is position starts[s] + i of sequence s,
 * as it is stored (keys rotated), n_kv_heads heads of head_dim, in `dtype` (8-bit values and bf16 widen exactly to fp32, 8-bit
 * values to bf16 as said above; fp32 rounds to bf16 once).  starts null: from position 0 on; k_out or
 * v_out may be null.  Rows outside every sequence, and rows whose position is negative, beyond the table or on a page outside [0, n_pages),
 * stay as they were, or become zeros where zero_rest is not 0.
 * Errors: INVALID_ARG (as above; n_rows in [0, 2^23]), DEVICE. */
typedef struct {
  ts_kv_pages_any cache;
  const int32_t* table; int64_t table_stride; int32_t table_width;
  const int32_t* starts; const int32_t* row_offsets;
  int32_t n_seqs, n_rows, dtype, zero_rest;
  void* k_out; int64_t k_stride;
  void* v_out; int64_t v_stride;
} ts_kv_read_args;
ts_status ts_kv_read(const ts_kv_read_args* args, ts_stream stream);

/* Attention of chunks of rows over the cache: rows [row_offsets[s], row_offsets[s + 1]) belong to sequence s and have the
 * positions lengths[s], lengths[s] + 1, ... whose keys and values ts_kv_append has written with the same lengths and offsets
 * (row_offsets null: sequence s has row s alone).  A row sees the positions up to its own, with window > 0 only the last
 * `window` of them; or, where ancestors is not null, the positions before lengths[s], row 0 of its chunk, and those rows j >= 1 of its
 * chunk whose bit j - 1 of ancestors[row] is set (a draft tree of a root and up to 64 nodes; no row beyond 64 is seen; a row's own
 * bit is set like any other; window has to be 0).  out, lse, scale, heads, pages out of range, max_len (here: no position of
 * a row is at or above it), contents of what is not seen, and rows that see nothing: as ts_kv_attend; rows outside every sequence
 * stay as they were in out and lse.  A seen infinite value makes its dimension infinite, or NaN where its probability is zero.
 * Scores, sums and outputs are fp32; queries and probabilities of fp32 rows enter the products over bf16 and 8-bit pages with 24 bits.
 * Probabilities of bf16 rows have 24 bits too where the chunks have up to 16 rows x heads per KV head on average; where they have more they are
 * rounded to bf16, once, for the product with the values (not for their sum): as much as the rounding of the output.  The average is that of the
 * call, n_rows * n_q_heads / (n_seqs * n_kv_heads): a row's bits go by the sizes of the call that it is in, and a program that wants 24 bits for chunks of
 * many rows gives them in fp32.  The order of
 * the sums depends on the sizes (n_seqs, n_rows, heads, max_len, window) and a chunk's own rows, never on contents.
 * The same averages choose how the work is cut: sequences of one or a few rows and chunks of many, or one long sequence and many short ones, take less
 * time in calls of their own than in one together.  One token per sequence over fp32 and bf16 pages takes as long or less by ts_kv_attend.
 *   q, out    : [n_rows] rows of n_q_heads * head_dim, in `dtype`
 *   lse       : [n_rows][n_q_heads] fp32, or null
 *   ancestors : [n_rows] 64-bit sets, or null
 *   workspace : ts_kv_attend_rows_workspace bytes for the same sizes, 16-byte aligned, contents irrelevant (null where that is 0)
 * Errors: INVALID_ARG (as ts_kv_attend; window with ancestors, n_rows in [0, 2^23], n_rows below n_seqs where row_offsets is null,
 * n_rows * n_q_heads or the workgroups beyond 2^24), DEVICE. */
typedef struct {
  ts_kv_pages_any cache;
  const int32_t* table; int64_t table_stride; int32_t table_width;
  const int32_t* lengths; const int32_t* row_offsets; const uint64_t* ancestors;
  int32_t n_seqs, n_rows, max_len, window, n_q_heads, dtype;
  const void* q; int64_t q_stride;
  void* out; int64_t out_stride;
  float* lse;
  float scale;
  void* workspace; uint64_t workspace_bytes;
} ts_kv_attend_rows_args;
ts_status ts_kv_attend_rows(const ts_kv_attend_rows_args* args, ts_stream stream);
/* Bytes of workspace a call with these sizes needs, whatever the pages' type; never decreases with max_len at the same other sizes. */
ts_status ts_kv_attend_rows_workspace(int32_t n_seqs, int32_t n_rows, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                      int32_t max_len, int32_t window, uint64_t* bytes);

#ifdef __cplusplus
}
#endif
#endif /* TOOLSPEC_OPS_H */
