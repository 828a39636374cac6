// Host side of sdnn_serve.h: argument checks.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "sdnn_decode_check.h"
#include "sdnn_serve_shape.h"

using namespace sdnn;

namespace {

sdnn_status check_q8(const sdnn_q8_cache* c) {
  if (!c) return SDNN_ERR_NULL;
  if (c->pages < 0 || c->pages > INT32_MAX) return SDNN_ERR_DIM;
  if (c->kv_heads < 1 || c->kv_heads > 65536) return SDNN_ERR_DIM;
  if (c->head_dim < 16 || c->head_dim > kMaxHeadDim || c->head_dim % 16) return SDNN_ERR_DIM;
  if (c->block != 32 && c->block != 64 && c->block != 128) return SDNN_ERR_DIM;
  if (bad_align(c->k_codes) || bad_align(c->v_codes) || bad_align(c->k_scales) || bad_align(c->v_scales) ||
      bad_align(c->means) || bad_align(c->mean_scales))
    return SDNN_ERR_DIM;
  return !c->means != !c->mean_scales ? SDNN_ERR_NULL : SDNN_OK;
}

bool has_pages(const sdnn_q8_cache& c) {
  return c.pages == 0 || (c.k_codes && c.v_codes && c.k_scales && c.v_scales);
}

sdnn_status check_norm(const sdnn_head_norm* n, int32_t head_dim) {
  if (!(n->eps >= 0.0 && n->eps < (double)INFINITY)) return SDNN_ERR_DIM;
  if ((n->q_head_stride != 0 && n->q_head_stride != head_dim) || (n->k_head_stride != 0 && n->k_head_stride != head_dim))
    return SDNN_ERR_DIM;
  return (uintptr_t)n->q_weight % 4 || (uintptr_t)n->k_weight % 4 ? SDNN_ERR_DIM : SDNN_OK;
}

// Rows that are written: those of x, or apart.
sdnn_status check_out(const sdnn_heads* x, const sdnn_heads* y, int32_t tokens, int32_t head_dim, int dtype) {
  SDNN_CHECK(check_rows(y, x->heads, tokens, dtype));
  if (!distinct_rows(*y, tokens, head_dim)) return SDNN_ERR_DIM;
  return x->data == y->data && !same_rows(*x, *y) ? SDNN_ERR_DIM : SDNN_OK;
}

}  // namespace

extern "C" {

sdnn_status sdnn_norm_rope(const sdnn_heads* q, const sdnn_heads* q_out, const sdnn_heads* k,
                           const sdnn_heads* k_out, sdnn_dtype dtype, int32_t tokens,
                           int32_t head_dim, const int32_t* pos, const sdnn_head_norm* norm,
                           const sdnn_rotation* rotation, void* stream) {
  if (!norm || !k != !k_out) return SDNN_ERR_NULL;
  if (bad_dtype(dtype) || tokens < 0 || head_dim < 2 || head_dim > kMaxHeadDim || head_dim % 2) return SDNN_ERR_DIM;
  SDNN_CHECK(check_norm(norm, head_dim));
  SDNN_CHECK(check_rows(q, 0, tokens, dtype));
  SDNN_CHECK(check_out(q, q_out, tokens, head_dim, dtype));
  if (k) {
    SDNN_CHECK(check_rows(k, 0, tokens, dtype));
    SDNN_CHECK(check_out(k, k_out, tokens, head_dim, dtype));
    // (rows of one that workgroups write while others read those of the other)
    if (tokens > 0 && (k_out->data == q_out->data || q_out->data == k->data || k_out->data == q->data)) return SDNN_ERR_DIM;
  }
  if (rotation) SDNN_CHECK(check_rotation(rotation, head_dim));
  if (tokens == 0) return SDNN_OK;
  if (rotation && rotation->pairs > 0 && !pos) return SDNN_ERR_NULL;
  return result(launch_norm(*q, *q_out, k, k_out, dtype, tokens, head_dim, pos, *norm, rotation, (hipStream_t)stream));
}

sdnn_status sdnn_q8_append(const sdnn_q8_cache* cache, const sdnn_tokens* tokens,
                           sdnn_dtype dtype, const sdnn_heads* k, const sdnn_heads* v,
                           const sdnn_head_norm* norm, const sdnn_rotation* rotation,
                           const sdnn_heads* q, const sdnn_heads* q_out, void* stream) {
  SDNN_CHECK(check_q8(cache));
  SDNN_CHECK(check_tokens(tokens));
  if (bad_dtype(dtype)) return SDNN_ERR_DIM;
  SDNN_CHECK(check_rows(k, cache->kv_heads, tokens->tokens, dtype));
  SDNN_CHECK(check_rows(v, cache->kv_heads, tokens->tokens, dtype));
  if (norm) SDNN_CHECK(check_norm(norm, cache->head_dim));
  if (rotation) SDNN_CHECK(check_rotation(rotation, cache->head_dim));
  if (!q != !q_out) return SDNN_ERR_NULL;
  if (q) {
    SDNN_CHECK(check_rows(q, 0, tokens->tokens, dtype));
    SDNN_CHECK(check_out(q, q_out, tokens->tokens, cache->head_dim, dtype));
    if (tokens->tokens > 0 && (q_out->data == k->data || q_out->data == v->data)) return SDNN_ERR_DIM;
  }
  if (tokens->tokens == 0) return SDNN_OK;
  if (!has_pages(*cache)) return SDNN_ERR_NULL;
  return result(launch_q8_append(*cache, *tokens, dtype, *k, *v, norm, rotation, q, q_out, (hipStream_t)stream));
}

sdnn_status sdnn_q8_read(const sdnn_q8_cache* cache, const sdnn_tokens* tokens, sdnn_dtype dtype,
                         const sdnn_heads* k, const sdnn_heads* v, void* stream) {
  SDNN_CHECK(check_q8(cache));
  SDNN_CHECK(check_tokens(tokens));
  if (bad_dtype(dtype)) return SDNN_ERR_DIM;
  for (const sdnn_heads* r : {k, v}) {
    if (!r) continue;
    SDNN_CHECK(check_rows(r, cache->kv_heads, tokens->tokens, dtype));
    if (!distinct_rows(*r, tokens->tokens, cache->head_dim)) return SDNN_ERR_DIM;
  }
  if (tokens->tokens == 0 || (!k && !v)) return SDNN_OK;
  if (k && v && k->data == v->data) return SDNN_ERR_DIM;
  if (!has_pages(*cache)) return SDNN_ERR_NULL;
  return result(launch_q8_read(*cache, *tokens, dtype, k, v, (hipStream_t)stream));
}

int64_t sdnn_q8_attend_floats(const sdnn_q8_cache* cache, int32_t tokens, int32_t heads,
                              int32_t blocks, int32_t shared) {
  if (check_q8(cache) != SDNN_OK || tokens <= 0 || heads <= 0 || blocks <= 0 || heads % cache->kv_heads || shared < 0 ||
      shared > blocks)
    return 0;
  const sdnn_block_cache c = as_blocks(*cache);
  return shared > 0 ? shared_floats(c, tokens, heads, blocks, shared) : attend_floats(c, tokens, heads, blocks);
}

sdnn_status sdnn_q8_attend(const sdnn_q8_cache* cache, const sdnn_tokens* tokens,
                           sdnn_dtype dtype, const sdnn_heads* q, const sdnn_heads* o,
                           const int32_t* chosen, int32_t blocks, int32_t shared, float scale,
                           float* lse, float* workspace, int64_t workspace_floats, void* stream) {
  SDNN_CHECK(check_q8(cache));
  SDNN_CHECK(check_tokens(tokens));
  if (bad_dtype(dtype)) return SDNN_ERR_DIM;
  SDNN_CHECK(check_rows(q, 0, tokens->tokens, dtype));
  SDNN_CHECK(check_rows(o, q->heads, tokens->tokens, dtype));
  if (q->heads % cache->kv_heads || q->heads / cache->kv_heads > kMaxGroup) return SDNN_ERR_DIM;
  if (!distinct_rows(*o, tokens->tokens, cache->head_dim)) return SDNN_ERR_DIM;
  if (!(scale > -1e30f && scale < 1e30f)) return SDNN_ERR_DIM;
  if (chosen && (blocks < 1 || blocks > kMaxBlocks)) return SDNN_ERR_DIM;
  if (shared < 0 || shared > tokens->max_blocks || shared > kMaxShared || (shared > 0 && chosen)) return SDNN_ERR_DIM;
  if (shared > 0 && tokens->sequences == 0) shared = 0;  // all tokens are fillers
  if (!chosen) blocks = tokens->max_blocks;
  if (tokens->tokens == 0) return SDNN_OK;
  if (!has_pages(*cache)) return SDNN_ERR_NULL;
  const int64_t need = sdnn_q8_attend_floats(cache, tokens->tokens, q->heads, blocks, shared);
  SDNN_CHECK(check_workspace(workspace, workspace_floats, need, *tokens, *q, *o, lse));
  return result(launch_q8_attend(*cache, *tokens, dtype, *q, *o, chosen, blocks, shared, scale, lse, workspace,
                                 (hipStream_t)stream));
}

int64_t sdnn_block_attend_shared_floats(const sdnn_block_cache* cache, int32_t tokens,
                                        int32_t heads, int32_t blocks, int32_t shared) {
  if (check_cache(cache) != SDNN_OK || tokens <= 0 || heads <= 0 || blocks <= 0 || heads % cache->kv_heads || shared < 1 ||
      shared > blocks)
    return 0;
  return shared_floats(*cache, tokens, heads, blocks, shared);
}

sdnn_status sdnn_block_attend_shared(const sdnn_block_cache* cache, const sdnn_tokens* tokens,
                                     const sdnn_heads* q, const sdnn_heads* o, int32_t shared,
                                     float scale, float* lse, float* workspace,
                                     int64_t workspace_floats, void* stream) {
  SDNN_CHECK(check_cache(cache));
  SDNN_CHECK(check_tokens(tokens));
  SDNN_CHECK(check_rows(q, 0, tokens->tokens, cache->dtype));
  SDNN_CHECK(check_rows(o, q->heads, tokens->tokens, cache->dtype));
  if (q->heads % cache->kv_heads || q->heads / cache->kv_heads > kMaxGroup) return SDNN_ERR_DIM;
  if (!distinct_rows(*o, tokens->tokens, cache->head_dim)) return SDNN_ERR_DIM;
  if (!(scale > -1e30f && scale < 1e30f)) return SDNN_ERR_DIM;
  if (shared < 1 || shared > tokens->max_blocks || shared > kMaxShared) return SDNN_ERR_DIM;
  if (tokens->tokens == 0) return SDNN_OK;
  if (cache->pages > 0 && (!cache->k_pages || !cache->v_pages)) return SDNN_ERR_NULL;
  const int64_t need =
      sdnn_block_attend_shared_floats(cache, tokens->tokens, q->heads, tokens->max_blocks, shared);
  SDNN_CHECK(check_workspace(workspace, workspace_floats, need, *tokens, *q, *o, lse));
  // one row of the table has nothing to share
  if (tokens->sequences <= 1)
    return result(launch_attend(*cache, *tokens, *q, *o, nullptr, tokens->max_blocks, scale, lse, workspace,
                                (hipStream_t)stream));
  return result(launch_attend_shared(*cache, *tokens, *q, *o, shared, scale, lse, workspace, (hipStream_t)stream));
}

int64_t sdnn_sample_floats(int32_t rows, int32_t vocab) {
  return rows > 0 && vocab > 0 && vocab <= kMaxVocab ? sample_floats(rows, vocab) : 0;
}

sdnn_status sdnn_sample(const void* logits, int64_t row_stride, sdnn_dtype dtype, int32_t rows,
                        int32_t vocab, const float* u, const sdnn_sampling* settings,
                        int32_t* token, float* logprob, float* workspace,
                        int64_t workspace_floats, void* stream) {
  if (!settings) return SDNN_ERR_NULL;
  if (bad_dtype(dtype) || rows < 0 || vocab < 1 || vocab > kMaxVocab) return SDNN_ERR_DIM;
  if (bad_stride(row_stride) || (rows > 1 && row_stride < vocab)) return SDNN_ERR_DIM;
  if (rows == 0) return SDNN_OK;
  if (!logits || !u || !token) return SDNN_ERR_NULL;
  if ((uintptr_t)logits % dtype_bytes(dtype)) return SDNN_ERR_DIM;
  const int64_t need = sdnn_sample_floats(rows, vocab);
  if (need > 0 && !workspace) return SDNN_ERR_NULL;
  if (need > 0 && (workspace_floats < need || bad_align(workspace))) return SDNN_ERR_DIM;
  return result(launch_sample(logits, row_stride, dtype, rows, vocab, u, *settings, token, logprob, workspace,
                              (hipStream_t)stream));
}

}  // extern "C"
