// Argument checks that the host sides of sdnn_decode.h and sdnn_serve.h share.
#ifndef SDNN_DECODE_CHECK_H_
#define SDNN_DECODE_CHECK_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sdnn_decode_internal.h"

namespace sdnn {

inline bool bad_dtype(int dtype) { return dtype != SDNN_F32 && dtype != SDNN_F16 && dtype != SDNN_BF16; }
inline bool bad_align(const void* p) { return (uintptr_t)p % 16 != 0; }
// Strides in elements: not negative, and small enough that a row number times one fits 64 bits.
inline bool bad_stride(int64_t s) { return s < 0 || s >= (int64_t)1 << 36; }

inline sdnn_status check_cache(const sdnn_block_cache* c) {
  if (!c) return SDNN_ERR_NULL;
  if (bad_dtype(c->dtype) || c->pages < 0 || c->pages > INT32_MAX) return SDNN_ERR_DIM;
  if (c->kv_heads < 1 || c->kv_heads > 65536) return SDNN_ERR_DIM;
  if (c->head_dim < 8 || c->head_dim > kMaxHeadDim || c->head_dim % 8) return SDNN_ERR_DIM;
  if (c->block != 32 && c->block != 64 && c->block != 128) return SDNN_ERR_DIM;
  if (bad_align(c->k_pages) || bad_align(c->v_pages) || bad_align(c->means) || bad_align(c->mean_scales))
    return SDNN_ERR_DIM;
  return SDNN_OK;
}

inline sdnn_status check_tokens(const sdnn_tokens* t) {
  if (!t) return SDNN_ERR_NULL;
  if (t->tokens < 0 || t->sequences < 0 || t->max_blocks < 0) return SDNN_ERR_DIM;
  if (t->tokens > 0 && (!t->pos || !t->seq)) return SDNN_ERR_NULL;
  if (t->tokens > 0 && t->sequences > 0 && t->max_blocks > 0 && !t->table) return SDNN_ERR_NULL;
  return SDNN_OK;
}

// Rows of `heads` heads (0: any positive number) of head_dim values for `tokens` tokens.
inline sdnn_status check_rows(const sdnn_heads* r, int32_t heads, int32_t tokens, int dtype) {
  if (!r) return SDNN_ERR_NULL;
  if (r->heads < 1 || r->heads > 65536 || (heads && r->heads != heads)) return SDNN_ERR_DIM;
  if (bad_stride(r->token_stride) || bad_stride(r->head_stride)) return SDNN_ERR_DIM;
  if (tokens > 0 && !r->data) return SDNN_ERR_NULL;
  return (uintptr_t)r->data % dtype_bytes(dtype) ? SDNN_ERR_DIM : SDNN_OK;
}

inline sdnn_status check_rotation(const sdnn_rotation* r, int32_t head_dim) {
  if (r->pairs < 0 || 2 * (int64_t)r->pairs > head_dim) return SDNN_ERR_DIM;
  if (r->layout != SDNN_ROPE_HALF && r->layout != SDNN_ROPE_INTERLEAVED) return SDNN_ERR_DIM;
  return r->pairs > 0 && !r->freq ? SDNN_ERR_NULL : SDNN_OK;
}

inline bool overlap(const void* a, int64_t abytes, const void* b, int64_t bbytes) {
  if (!a || !b || abytes <= 0 || bbytes <= 0) return false;
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a0 < b0 + (uintptr_t)bbytes && b0 < a0 + (uintptr_t)abytes;
}

// The same of two sets of rows of a_row and b_row bytes, `rows` of each, stride bytes apart: columns of one buffer may lie
// side by side.
inline bool overlap_rows(const void* a, int64_t a_row, const void* b, int64_t b_row, int64_t rows, int64_t stride) {
  if (!overlap(a, (rows - 1) * stride + a_row, b, (rows - 1) * stride + b_row)) return false;
  if (rows < 2 || stride == 0) return true;
  const int64_t between = (int64_t)((uintptr_t)b - (uintptr_t)a) % stride, off = between < 0 ? between + stride : between;
  return off < a_row || off + b_row > stride;
}

inline bool same_rows(const sdnn_heads& a, const sdnn_heads& b) {
  return a.data == b.data && a.token_stride == b.token_stride && a.head_stride == b.head_stride;
}
// Outputs have to lie apart from each other: a stride of zero would write one row for several.
inline bool distinct_rows(const sdnn_heads& a, int32_t tokens, int32_t head_dim) {
  return (tokens < 2 || a.token_stride != 0) && (a.heads < 2 || a.head_stride >= head_dim);
}

// (A call of more threads than a launch has is refused before it.)
inline sdnn_status result(hipError_t e) {
  return e == hipSuccess ? SDNN_OK : e == hipErrorInvalidConfiguration ? SDNN_ERR_DIM : SDNN_ERR_HIP;
}

// The scratch of an attention call that needs `need` floats.
inline sdnn_status check_workspace(const float* workspace, int64_t floats, int64_t need, const sdnn_tokens& t,
                                   const sdnn_heads& q, const sdnn_heads& o, const float* lse) {
  if (need > 0 && !workspace) return SDNN_ERR_NULL;
  if (need > 0 && (floats < need || bad_align(workspace))) return SDNN_ERR_DIM;
  const bool meets = overlap(workspace, need * 4, lse, (int64_t)t.tokens * q.heads * 4) || workspace == q.data ||
                     workspace == o.data;
  return need > 0 && meets ? SDNN_ERR_DIM : SDNN_OK;
}

#define SDNN_CHECK(call)                  \
  do {                                    \
    const sdnn_status st_ = (call);       \
    if (st_ != SDNN_OK) return st_;       \
  } while (0)

}  // namespace sdnn

#endif  // SDNN_DECODE_CHECK_H_
