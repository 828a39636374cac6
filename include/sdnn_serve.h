/*
 * sdnn_serve.h -- C ABI of the operators that a serving decoder's step needs beside those of
 * sdnn_decode.h: norms of queries and keys with the rotation in the same pass, a cache in 8
 * bits (written, read back, attended to), attention of a batch that shares a long prefix, and
 * the choice of the next token.
 *
 * The conventions are those of sdnn_decode.h: rows of heads, positions and sequences of
 * tokens, fillers, the block table, missing pages; status codes; asynchronous calls that
 * allocate nothing and may be captured in a HIP graph; SDNN_ERR_DIM for a call whose launch
 * would have 2^32 threads or more (none is refused for it where tokens * heads, of the kind with
 * most, is at most 2^21; rows of sdnn_sample likewise).
 * A workspace is scratch of one call: calls that may run at the same time (two streams, two
 * captured graphs) need one each.
 */
#ifndef SDNN_SERVE_H_
#define SDNN_SERVE_H_

#include "sdnn_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A norm of each head by its root mean square: with S = sum x_d^2 (in 64 bits),
 *     r = 1 / sqrt(S / head_dim + eps)   (in 64 bits, then rounded to 32),
 *     a_d = (x_d r) w_d                  (each product rounded to 32 bits).
 *   q_weight, k_weight: device, floats: head_dim of them for all heads, or with the stride
 *   head_dim in place of 0 a row of its own for each head; NULL: all 1.
 *   eps: finite, not negative. */
typedef struct {
  const float* q_weight;
  const float* k_weight;
  int32_t q_head_stride; /* floats from one head's weights to the next: 0 or head_dim */
  int32_t k_head_stride;
  double eps;
} sdnn_head_norm;

/* q_out = rotation(norm(q)), and where k is not NULL k_out = rotation(norm(k)) with the keys'
 * weights, in one pass: the norm's 32-bit results are rotated in 32 bits as in sdnn_rope and
 * rounded to dtype once.  rotation NULL: the norm alone.  With k NULL so is k_out.
 *   Outputs are their inputs' rows (in place) or overlap no others.  pos (device, tokens) may
 *   be NULL without rotation; it may be negative, a position like any other.
 *   head_dim even, at most 256; 2 * pairs at most head_dim.
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM, SDNN_ERR_HIP. */
sdnn_status sdnn_norm_rope(const sdnn_heads* q, const sdnn_heads* q_out, const sdnn_heads* k,
                           const sdnn_heads* k_out, sdnn_dtype dtype, int32_t tokens,
                           int32_t head_dim, const int32_t* pos, const sdnn_head_norm* norm,
                           const sdnn_rotation* rotation, void* stream);

/* A cache in 8 bits: a token's key (value) of a head is scale * n, its numbers n from -127 to
 * 127, its scale a float.  Pages of `block` tokens (32, 64 or 128), kv_heads heads of head_dim
 * values (a multiple of 16, at most 256), all device memory of the caller:
 *   k_codes:  [pages][kv_heads][block][head_dim] int8
 *   v_codes:  [pages][kv_heads][head_dim][block] int8
 *   k_scales, v_scales: [pages][kv_heads][block] float
 *   means, mean_scales: as in sdnn_block_cache, or both NULL.
 * A row x (32-bit values) becomes, with a = max |x_d|,
 *     f = 127 * (1 / a),  n_d = rint(x_d f),  scale = a * (1 / 127)
 * each operation rounded to 32 bits (1 / 127 too); all zeros where a < 2^-100.  Of a row with a
 * value that is infinite or not a number (a key also after its norm) the scale is NaN, and its
 * numbers mean nothing: it is read back as NaN, outputs of tokens that see it are NaN, sums over
 * such keys too, and the mean of a block with such a key counts as 0.  The arrays are 16-byte
 * aligned. */
typedef struct {
  int8_t* k_codes;
  int8_t* v_codes;
  float* k_scales;
  float* v_scales;
  int8_t* means;
  float* mean_scales;
  int64_t pages;
  int32_t kv_heads;
  int32_t head_dim;
  int32_t block;
  int32_t reserved; /* 0 */
} sdnn_q8_cache;

/* Stores the keys and values of the call's tokens at their positions in 8 bits.  Keys are
 * normed (norm NULL: not) and rotated (rotation NULL: not) in 32 bits first, and quantised from
 * there; values are quantised as they are.  With q, also q_out = rotation(norm(q)) (rows of
 * fillers become zero).  Rows are of type dtype.
 *   With means (and mean_scales), the mean of every block that a token of the call fills (its
 *   last position is stored) is written as by sdnn_cache_append, of the keys as stored, each
 *   the product scale * n rounded to 32 bits; this takes a second launch.
 * The tokens of one sequence in a call are consecutive and ascend by one position.  A token
 * at a position that is stored already replaces what is there.
 *   k, v: kv_heads heads; q, q_out: any number of the same heads, both or neither; q_out is q
 *   (in place) or overlaps no other rows.
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM, SDNN_ERR_HIP. */
sdnn_status sdnn_q8_append(const sdnn_q8_cache* cache, const sdnn_tokens* tokens,
                           sdnn_dtype dtype, const sdnn_heads* k, const sdnn_heads* v,
                           const sdnn_head_norm* norm, const sdnn_rotation* rotation,
                           const sdnn_heads* q, const sdnn_heads* q_out, void* stream);

/* Reads the tokens' keys and values back: k and v (either may be NULL) receive scale * n
 * rounded to 32 bits, then to dtype; zeros for fillers and missing pages.  Any positions in
 * any order, also the same one twice.
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM, SDNN_ERR_HIP. */
sdnn_status sdnn_q8_read(const sdnn_q8_cache* cache, const sdnn_tokens* tokens, sdnn_dtype dtype,
                         const sdnn_heads* k, const sdnn_heads* v, void* stream);

/* sdnn_block_attend over a cache in 8 bits, and with a shared prefix.  Keys and values are
 * scale * n exactly; q and o are of type dtype.
 *   shared: the blocks 0 ... shared - 1 are looked up in the table's first row for every
 *   sequence, and are read once for all of them (0: none; at most max_blocks, and then
 *   chosen is NULL).  Which tokens see how much of them is up to their positions, as ever.
 *   workspace: at least sdnn_q8_attend_floats floats.
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM (also a workspace too small), SDNN_ERR_HIP. */
sdnn_status sdnn_q8_attend(const sdnn_q8_cache* cache, const sdnn_tokens* tokens,
                           sdnn_dtype dtype, const sdnn_heads* q, const sdnn_heads* o,
                           const int32_t* chosen, int32_t blocks, int32_t shared, float scale,
                           float* lse, float* workspace, int64_t workspace_floats, void* stream);

/* Floats of workspace that sdnn_q8_attend needs for `tokens` tokens of `heads` queries over
 * `blocks` blocks each (max_blocks where chosen is NULL), `shared` of them in common.  Host
 * only. */
int64_t sdnn_q8_attend_floats(const sdnn_q8_cache* cache, int32_t tokens, int32_t heads,
                              int32_t blocks, int32_t shared);

/* sdnn_block_attend (of all blocks) with a shared prefix: as `shared` above, at least 1.
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM (also a workspace too small), SDNN_ERR_HIP. */
sdnn_status sdnn_block_attend_shared(const sdnn_block_cache* cache, const sdnn_tokens* tokens,
                                     const sdnn_heads* q, const sdnn_heads* o, int32_t shared,
                                     float scale, float* lse, float* workspace,
                                     int64_t workspace_floats, void* stream);

/* Floats of workspace that sdnn_block_attend_shared needs.  Host only. */
int64_t sdnn_block_attend_shared_floats(const sdnn_block_cache* cache, int32_t tokens,
                                        int32_t heads, int32_t blocks, int32_t shared);

/* What a row's token is drawn by; each is a device array of a value for every row, or NULL. */
typedef struct {
  const float* temperature; /* NULL: 1; 0 or less (and NaN): the largest logit is taken */
  const int32_t* top_k;     /* NULL, 0 or less: all */
  const float* top_p;       /* NULL, 1 or more (and NaN): all */
  const float* min_p;       /* NULL, 0 or less (and NaN): all */
} sdnn_sampling;

/* Draws a token for each row of logits.  With l_i the row's logits (NaN counts as -infinity),
 * m their maximum and t the temperature, a token's weight is w_i = exp((l_i - m) / t)
 * (1 where l_i = m, also where that is infinite).  Of the tokens in descending order of their
 * logits, equal ones in the order of their indexes,
 *     top_k keeps the first top_k,
 *     top_p of these all whose weights before them sum to less than top_p times the sum of
 *           the weights that top_k keeps (the first always),
 *     min_p of these all with w_i >= min_p (the first always).
 * token = the lowest index i at which the weights kept, summed up to and with i in the order of
 * indexes, exceed u times their sum M; logprob = log(w_token / M).  A row without a logit above
 * -infinity gets token -1 and logprob -infinity.
 *   A weight's exponent is computed in 64 bits, its power of two in 32, to 2^-22 of itself, and
 *   held as a whole number of 2^-44, cut off: so sums are the same in any order, a token of weight
 *   below 2^-44 is never drawn, and a border of the weights within 2^-21 M of u M (or that near to
 *   top_p's limit) may count as on either side of it.
 *   logits: device, row r at logits + r * row_stride (elements, at least vocab), of dtype.
 *   u: device, rows floats in [0, 1) (others count as the nearest of these).
 *   token: device, rows int32.  logprob: device, rows floats, or NULL.
 *   workspace: device, 16-byte aligned, at least sdnn_sample_floats floats; may be NULL where
 *   that is 0.
 *   1 <= vocab <= 2^19 (524288).
 * Errors: SDNN_ERR_NULL, SDNN_ERR_DIM (also a workspace too small), SDNN_ERR_HIP. */
sdnn_status sdnn_sample(const void* logits, int64_t row_stride, sdnn_dtype dtype, int32_t rows,
                        int32_t vocab, const float* u, const sdnn_sampling* settings,
                        int32_t* token, float* logprob, float* workspace,
                        int64_t workspace_floats, void* stream);

/* Floats of workspace that sdnn_sample needs.  Host only. */
int64_t sdnn_sample_floats(int32_t rows, int32_t vocab);

#ifdef __cplusplus
}
#endif

#endif /* SDNN_SERVE_H_ */
