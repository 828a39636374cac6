/*
 * sdnn_decode.h -- C ABI of the operators of a decoder's step that stand between the
 * sparse products of sdnn.h: rotary positions, a paged cache of keys and values with a
 * small summary for each block, the choice of blocks by that summary, attention over the
 * chosen blocks, and products of 4-bit weights with the activations of few tokens.
 *
 * Conventions, beyond those of sdnn.h (status codes, no exception crosses the boundary,
 * device pointers, streams as void*, asynchronous calls that allocate nothing and may be
 * captured in a HIP graph unless stated otherwise):
 *   - Rows of heads (queries, keys, values, outputs) are given by a pointer and two strides
 *     in elements: value d of head h of token t is data[t * token_stride + h * head_stride
 *     + d]; the values of one head are contiguous.  Any strides and any alignment of whole
 *     elements are accepted; 16-byte aligned rows are the fast case.
 *   - pos[t] is the position of token t in its sequence, seq[t] the sequence's row in the
 *     block table, both on the device.  A token with pos[t] < 0 or seq[t] outside
 *     [0, sequences) is a filler: nothing is stored for it, nothing is chosen for it, and
 *     its rows of outputs are zero.
 *   - table[s * max_blocks + b] is the page that holds block b (positions b * block ...
 *     b * block + block - 1) of sequence s.  A page outside [0, pages) and a block at or
 *     past max_blocks hold nothing: nothing is stored there and attention passes over them.
 *   - Values must be finite, but memory of a page that no token was stored to may hold
 *     anything: it is never read into a result.
 *   - Kernels are chosen by a call's sizes, the rows of its table among them; seq is not looked at.  A call
 *     of 16 tokens and more for each row of the table is taken for prompts, whose neighbouring tokens
 *     share what they read; else each token is handled for itself.  So prompts and single tokens
 *     belong in calls of their own, and a prompt's call should get its own sequences' rows alone
 *     (sdnn_block_attend of 2048 tokens over 16 of 128 blocks: 0.2 ms, with a table of 256 rows 0.9;
 *     with one token each of 64 other sequences 1.4, in two calls 0.26).
 *   - A call whose launch would have 2^32 threads or more gets SDNN_ERR_DIM: split its tokens over
 *     several.  None is refused for it up to these products: sdnn_rope: tokens 2^25;
 *     sdnn_cache_append: tokens * (kv_heads + 1) 2^23; sdnn_block_select: tokens * kv_heads 2^21;
 *     sdnn_block_attend: tokens * kv_heads * ceil(heads / kv_heads / 16) 2^23.
 */
#ifndef SDNN_DECODE_H_
#define SDNN_DECODE_H_

#include "sdnn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of activations, keys, values and scales. */
typedef enum { SDNN_F32 = 0, SDNN_F16 = 1, SDNN_BF16 = 2 } sdnn_dtype;

/* Which values of a head are rotated together. */
typedef enum {
  SDNN_ROPE_HALF = 0,       /* values i and i + pairs */
  SDNN_ROPE_INTERLEAVED = 1 /* values 2 i and 2 i + 1 */
} sdnn_rope_layout;

/* A rotation: pair i (0 <= i < pairs) of the first 2 * pairs values of a head at position p
 * turns by the angle p * freq[i] (radians) and is multiplied by amplitude:
 *     (x0, x1) -> (x0 c - x1 s, x1 c + x0 s),  c = amplitude cos, s = amplitude sin.
 * The angle is a product in 64 bits and its cosine and sine are accurate to 64 bits before
 * they are rounded to 32, so that long positions lose nothing; the rotation itself is in 32
 * bits with each operation rounded.  The values from 2 * pairs on are copied.
 *   freq: device, pairs doubles.  Scaling for long contexts is in these (and amplitude). */
typedef struct {
  const double* freq;
  int32_t pairs;
  int32_t layout; /* sdnn_rope_layout */
  double amplitude;
} sdnn_rotation;

/* The cache.  Pages of `block` tokens (32, 64 or 128), kv_heads heads of head_dim values
 * (a multiple of 8, at most 256), all device memory of the caller:
 *   k_pages:     [pages][kv_heads][block][head_dim]
 *   v_pages:     [pages][kv_heads][head_dim][block]  (values lie along the tokens, the order
 *                in which attention's second product takes them)
 *   means:       [pages][kv_heads][head_dim] int8 and
 *   mean_scales: [pages][kv_heads] float: the mean key of a full block is
 *                mean_scales * means.
 * Calls that do not use an array take NULL for it.  The arrays are 16-byte aligned. */
typedef struct {
  void* k_pages;
  void* v_pages;
  int8_t* means;
  float* mean_scales;
  int64_t pages;
  int32_t kv_heads;
  int32_t head_dim;
  int32_t block;
  int32_t dtype; /* sdnn_dtype of k_pages and v_pages, and of the rows of every call on it */
} sdnn_block_cache;

/* The tokens of a call: see the conventions above. */
typedef struct {
  const int32_t* pos;   /* tokens */
  const int32_t* seq;   /* tokens */
  const int32_t* table; /* sequences * max_blocks */
  int32_t tokens;
  int32_t sequences;
  int32_t max_blocks;
  int32_t reserved; /* 0 */
} sdnn_tokens;

/* Rows of heads. */
typedef struct {
  void* data;
  int64_t token_stride;
  int64_t head_stride;
  int32_t heads;
  int32_t reserved; /* 0 */
} sdnn_heads;

/* Rotary positions: y = rotation of x, or with inverse = 1 by the negative angles (which
 * undoes it, and is also the gradient of the rotation).  x and y have the same heads; they
 * are the same rows (in place) or do not overlap.  pos may be negative here: it is a
 * position like any other.  head_dim at most 256, 2 * pairs at most head_dim.
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM, SDNN_ERR_HIP. */
sdnn_status sdnn_rope(const sdnn_heads* x, const sdnn_heads* y, sdnn_dtype dtype, int32_t tokens,
                      int32_t head_dim, const int32_t* pos, const sdnn_rotation* rotation,
                      int32_t inverse, void* stream);

/* Stores the keys and values of the call's tokens at their positions, the keys rotated
 * (rotation NULL: as they are), and writes the mean of every block that a token of the call
 * fills (its last position is stored).  With q, also rotates the queries into q_out, in the
 * same launch (rows of fillers become zero).
 *   The mean: with x_i the block's keys as stored, i = 0 ... block - 1, halves are added
 *   until one is left (x_i + x_(i + block/2), then i + block/4, ...) in 32 bits, giving S;
 *   a = max |S|; means = rint(S * (127 * (1 / a))), mean_scales = a / (127 * block), each
 *   operation rounded to 32 bits; zeros if a = 0.
 * The tokens of one sequence in a call are consecutive and ascend by one position.  A token
 * at a position that is stored already replaces what is there.
 *   k, v: kv_heads heads; q, q_out: any number of the same heads, both or neither; q_out is
 *   q (in place) or overlaps no other rows.  means and mean_scales both or neither.
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM, SDNN_ERR_HIP. */
sdnn_status sdnn_cache_append(const sdnn_block_cache* cache, const sdnn_tokens* tokens,
                              const sdnn_heads* k, const sdnn_heads* v,
                              const sdnn_rotation* rotation, const sdnn_heads* q,
                              const sdnn_heads* q_out, void* stream);

/* Chooses blocks for each token and cached head.  Of the n = pos / block + 1 blocks that a
 * token sees, the first `sink` and the last `local` (its own among them) are always taken,
 * and of the others the ones with the largest score, ties to the lower block, until `blocks`
 * are taken or none is left.  The score of block b for a head's group of queries q_h
 * (h = the heads / kv_heads queries that share the cached head):
 *     a_h = max |q_h|,  m_h = rint(q_h * (127 * (1 / a_h)))   (zeros if a_h = 0)
 *     score = mean_scales_b * max_h ( a_h * (m_h . means_b) )
 * The dot product is of whole numbers and exact, the operations before and after it are rounded to
 * 32 bits one by one: a choice depends on nothing but q and the summaries.  A block without a valid page
 * scores below all others.
 *   chosen: device, [tokens][kv_heads][blocks] int32: the blocks in ascending order, then -1.
 *   At least one page, 1 <= blocks <= 1024, sink >= 0, local >= 1, sink + local <= blocks, max_blocks <= 32768,
 *   heads a multiple of kv_heads, at most 64 to a cached head.
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM, SDNN_ERR_HIP. */
sdnn_status sdnn_block_select(const sdnn_block_cache* cache, const sdnn_tokens* tokens,
                              const sdnn_heads* q, int32_t blocks, int32_t sink, int32_t local,
                              int32_t* chosen, void* stream);

/* Attention of each token's queries over the cached positions up to its own in the blocks
 * chosen for it (chosen as sdnn_block_select leaves it; NULL: in every block it sees):
 *     s_j = scale * q . k_j,  m = max s_j,  l = sum exp(s_j - m),
 *     o = (1 / l) sum exp(s_j - m) v_j,  lse = m + log l.
 * A token that sees nothing gets o = 0, lse = -infinity.  Negative entries of chosen count for
 * nothing wherever they stand; the others ascend, none repeats, and those past the token's own
 * block or the table count for nothing.
 *   o: like q.  lse: device, [tokens][heads] float, or NULL.
 *   blocks: row length of chosen (ignored when it is NULL).
 *   workspace: device, 16-byte aligned, at least sdnn_block_attend_floats floats, scratch of
 *   this call only; may be NULL where that is 0.  Where few tokens leave compute units idle
 *   the blocks of a token are spread over workgroups, whose parts are joined from it.
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM (also a workspace too small), SDNN_ERR_HIP. */
sdnn_status sdnn_block_attend(const sdnn_block_cache* cache, const sdnn_tokens* tokens,
                              const sdnn_heads* q, const sdnn_heads* o, const int32_t* chosen,
                              int32_t blocks, float scale, float* lse, float* workspace,
                              int64_t workspace_floats, void* stream);

/* Floats of workspace that sdnn_block_attend needs for `tokens` tokens of `heads` queries
 * over `blocks` blocks each (max_blocks where chosen is NULL).  Host only. */
int64_t sdnn_block_attend_floats(const sdnn_block_cache* cache, int32_t tokens, int32_t heads,
                                 int32_t blocks);

/* A matrix of 4-bit weights, laid out for sdnn_qmat_apply.  Row m, column k holds
 * scales[m][k / group] * (n - z), with n the 4-bit number (0 ... 15) and z = 8, or
 * zeros[m][k / group]. */
typedef struct sdnn_qmat_s* sdnn_qmat;

/* Lays out M x K weights on the current device (preparation; allocates and synchronises
 * `stream`).  All arrays are device memory, read during the call only:
 *   packed: [M][(K + 1) / 2] bytes, two numbers each, the lower column in the low half.
 *   scales: [M][ceil(K / group)] of scale_dtype.
 *   zeros:  [M][ceil(K / group)] bytes, or NULL.
 *   group:  32, 64 or a multiple of 128.  M, K >= 1, K <= 2^20, M <= 2^24.
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM, SDNN_ERR_ALLOC, SDNN_ERR_HIP. */
sdnn_status sdnn_qmat_create(const uint8_t* packed, const void* scales, sdnn_dtype scale_dtype,
                             const uint8_t* zeros, int32_t M, int32_t K, int32_t group,
                             void* stream, sdnn_qmat* out);

/* y = epi(W x + bias) for the N <= 2^18 columns of x.  Value k of column n is
 * x[k * x_feature + n * x_column] and value m of column n y[m * y_feature + n * y_column]:
 * a K x N matrix as sdnn_spmm takes it has strides (N, 1), rows of tokens (1, K).
 *   y's memory, from its first value to its last, holds none of x or bias; of tokens' rows that lie as
 *   far apart (x_feature = y_feature = 1, x_column = y_column) the rows themselves do not meet.
 *   bias: device, M floats, or NULL.  The products are exact and are summed in 32 bits; x
 *   must be finite.  Made for few columns: the weights are read once for every 16 of them (8 in
 *   32 bits).
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM, SDNN_ERR_DEVICE, SDNN_ERR_HIP. */
sdnn_status sdnn_qmat_apply(sdnn_qmat w, const void* x, int64_t x_feature, int64_t x_column, void* y,
                            int64_t y_feature, int64_t y_column, int32_t N, sdnn_dtype dtype,
                            const float* bias, sdnn_epilogue epi, void* stream);

/* Frees the matrix and its device memory.  NULL is a no-op. */
void sdnn_qmat_destroy(sdnn_qmat w);

#ifdef __cplusplus
}
#endif

#endif /* SDNN_DECODE_H_ */
