/*
 * m2r2_kv8.h — operators of the paged cache held in 8 bits: appending keys and
 * values with the position rotation applied on the way, and attention over
 * what was appended.  The decode path (m2r2.h) calls them where the
 * configuration's kvdtype is M2R2_FP8; a program with projections of its own
 * calls them directly.
 *
 * The cache of one layer.  k_pages and v_pages are
 * [num_blocks][n_kv_heads][block_size][head_dim] bytes, e4m3 codes (OCP: 4
 * exponent bits, 3 mantissa bits, no infinities, 0x7f and 0xff NaN); k_scales
 * and v_scales are [num_blocks][n_kv_heads] floats, powers of two in [2^-120,
 * 2^112].  A cached value is code * scale.  A power of two costs no precision
 * in a floating format, multiplies exactly, and lets a block's scale grow
 * without a second rounding of its codes (but of those that become subnormal).
 *
 * Conventions are those of m2r2.h: the caller owns every buffer, nothing is
 * allocated, calls only enqueue on `stream` and may be captured into a HIP
 * graph, arguments are checked before anything is enqueued, m2r2_last_error()
 * describes a failure.  All pointers belong to the current device.  Device
 * arrays (row starts, lengths, block tables) are read by the kernels and
 * cannot be checked by the host: what they hold out of range is left out, with
 * a bit set in *err_d, and reaches no memory.
 */
#ifndef M2R2_KV8_H_
#define M2R2_KV8_H_

#include "m2r2.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  void* k_pages;                 /* 16-byte aligned */
  void* v_pages;
  float* k_scales;
  float* v_scales;
  const int32_t* block_table_d;  /* [n_seqs][max_blocks_per_seq]: physical block of each logical block */
  int32_t num_blocks;
  int32_t block_size;            /* a multiple of 16, at most 256 */
  int32_t max_blocks_per_seq;
  int32_t n_kv_heads;
  int32_t head_dim;              /* 64, 96 or 128 */
} m2r2_kv8;

/* Bits set in *err_d (the same as m2r2_device_errors'). */
#define M2R2_KV8_ERR_BLOCK 2     /* a position outside the block table, or a table entry outside the pool */
#define M2R2_KV8_ERR_ROPE 8      /* a position beyond the rotation table */
#define M2R2_KV8_ERR_ROWS 32     /* row_start_d descends, or leaves [0, n_rows] */

/* Rows of a ragged batch: sequence s has rows row_start_d[s] ..
 * row_start_d[s+1]-1 of the call's n_rows.  Rows that belong to no sequence
 * (behind the last one of a padded batch) are neither read nor written.
 * Element (row, head, dim) of an array lies at row * row_stride + head *
 * head_stride + dim elements; every (row, head) starts on 16 bytes.  Arrays
 * without rows, and per-sequence arrays without sequences, may be NULL. */
typedef struct {
  int32_t n_seqs, n_rows;
  const int32_t* row_start_d;    /* [n_seqs + 1], ascending from row_start_d[0] >= 0 to at most n_rows */
  const int32_t* positions_d;    /* [n_seqs]: position of the sequence's first row */
  int32_t dtype;                 /* m2r2_dtype of k, v, q, q_out */
  const void* k;                 /* [n_rows][n_kv_heads][head_dim], before the rotation */
  const void* v;
  int64_t k_row, k_head, v_row, v_head;
  /* rotate-half table [rope_len][head_dim / 2][2]: (cos, sin); NULL: no rotation */
  const float* rope_d;
  int32_t rope_len;
  /* optional (n_heads 0 and NULL otherwise): the rows' queries, rotated into
   * q_out, which may be q itself (with the same strides).  With rope_d NULL they are copied. */
  int32_t n_heads;               /* query heads, a multiple of n_kv_heads */
  const void* q;
  void* q_out;
  int64_t q_row, q_head, qo_row, qo_head;
  int32_t* err_d;                /* optional: error bits are or-ed into it */
} m2r2_kv8_rows;

/* Append rows to the cache.  For every block that receives rows of a
 * sequence, every head, keys and values apart: the exponent e is the least
 * integer in [-120, 112] with 448 * 2^e >= max |y| over the block's new finite
 * entries y (the rotated key in float32, or the value).  If slots before the
 * first new one of that block exist, they hold earlier rows: e is then at
 * least the stored exponent, and if it grows their codes are rounded to the
 * new scale.  New codes are y / 2^e rounded to nearest, ties to even, |y|
 * above 448 * 2^112 saturated, NaN and infinities stored as NaN.  Slots behind the
 * last new row keep their bytes.  The rotation's products are exact and
 * rounded once, to float32.
 *
 * Two sequences must not append to the same physical block in one call (two
 * that share a prefix share only whole blocks): what such a block then holds
 * is one's rows, the other's, or a mixture.  The same holds for a table that
 * names a block twice among those that one sequence appends to.  The arrays
 * must not overlap each other (but q_out q) or the cache; in q_out neither rows
 * nor heads overlap, in the others both strides may be 0. */
M2R2_API m2r2_status m2r2_kv8_append(const m2r2_kv8* kv, const m2r2_kv8_rows* rows, hipStream_t stream);

typedef struct {
  int32_t n_seqs, n_rows;
  const int32_t* row_start_d;    /* as above */
  const int32_t* lens_d;         /* [n_seqs]: valid cache positions (those of this step's rows included) */
  /* [n_rows]: the row sees the first min(visible, len) positions; NULL: causal,
   * row i of a sequence's n sees len - (n - 1 - i) (none if that is negative) */
  const int32_t* visible_d;
  int32_t dtype;                 /* m2r2_dtype of q, own_k, own_v, out */
  int32_t n_heads;               /* query heads, a multiple of n_kv_heads: head h reads head h / (n_heads / n_kv_heads) */
  const void* q;
  int64_t q_row, q_head;
  /* Optional: keys and values that are not in the cache (a fast row's own,
   * exact).  own_d[row] is an index into own_k / own_v [n_own][n_kv_heads][head_dim],
   * or negative for none.  NULL own_d: none. */
  const int32_t* own_d;
  const void* own_k;
  const void* own_v;
  int32_t n_own;
  int64_t ok_row, ok_head, ov_row, ov_head;
  float scale;                   /* of the scores, > 0; 0: 1 / sqrt(head_dim) */
  void* out;                     /* [n_rows][n_heads][head_dim] */
  int64_t out_row, out_head;
  int32_t* err_d;
} m2r2_kv8_query;

/* Bytes of scratch that m2r2_kv8_attention needs for calls of up to n_seqs
 * sequences and n_rows rows. */
M2R2_API m2r2_status m2r2_kv8_workspace_size(const m2r2_kv8* kv, int32_t n_seqs, int32_t n_rows, int32_t n_heads,
                                             size_t* bytes_out);

/* out = softmax(scale * q K^T) V over the positions that each row sees and
 * its own key and value, if it has one.  A row that sees nothing is zero.  What
 * a row does not see does not reach it, NaN included.  Scores, the softmax and
 * all sums are float32.  `out` overlaps none of the other arrays and the cache.
 *
 * `workspace`: device memory of at least m2r2_kv8_workspace_size() bytes, 256-byte
 * aligned, zeroed by the caller before its first use; every call leaves it
 * ready for the next, of any shape that it is large enough for.  Calls that
 * may run at the same time need a workspace each. */
M2R2_API m2r2_status m2r2_kv8_attention(const m2r2_kv8* kv, const m2r2_kv8_query* query, void* workspace,
                                        size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* M2R2_KV8_H_ */
