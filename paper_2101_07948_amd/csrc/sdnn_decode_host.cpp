// Host side of sdnn_decode.h: argument checks and the lifetime of 4-bit matrices.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <new>

#include "sdnn_decode_internal.h"
#include "sdnn_decode_shape.h"

using namespace sdnn;

namespace {

bool bad_dtype(int dtype) { return dtype != SDNN_F32 && dtype != SDNN_F16 && dtype != SDNN_BF16; }
bool bad_align(const void* p) { return (uintptr_t)p % 16 != 0; }
// Strides in elements: not negative, and small enough that a row number times one fits 64 bits.
bool bad_stride(int64_t s) { return s < 0 || s >= (int64_t)1 << 36; }

sdnn_status check_cache(const sdnn_block_cache* c) {
  if (!c) return SDNN_ERR_NULL;
  if (bad_dtype(c->dtype) || c->pages < 0 || c->pages > INT32_MAX) return SDNN_ERR_DIM;
  if (c->kv_heads < 1 || c->kv_heads > 65536) return SDNN_ERR_DIM;
  if (c->head_dim < 8 || c->head_dim > kMaxHeadDim || c->head_dim % 8) return SDNN_ERR_DIM;
  if (c->block != 32 && c->block != 64 && c->block != 128) return SDNN_ERR_DIM;
  if (bad_align(c->k_pages) || bad_align(c->v_pages) || bad_align(c->means) || bad_align(c->mean_scales))
    return SDNN_ERR_DIM;
  return SDNN_OK;
}

sdnn_status check_tokens(const sdnn_tokens* t) {
  if (!t) return SDNN_ERR_NULL;
  if (t->tokens < 0 || t->sequences < 0 || t->max_blocks < 0) return SDNN_ERR_DIM;
  if (t->tokens > 0 && (!t->pos || !t->seq)) return SDNN_ERR_NULL;
  if (t->tokens > 0 && t->sequences > 0 && t->max_blocks > 0 && !t->table) return SDNN_ERR_NULL;
  return SDNN_OK;
}

// Rows of `heads` heads (0: any positive number) of head_dim values for `tokens` tokens.
sdnn_status check_rows(const sdnn_heads* r, int32_t heads, int32_t tokens, int dtype) {
  if (!r) return SDNN_ERR_NULL;
  if (r->heads < 1 || r->heads > 65536 || (heads && r->heads != heads)) return SDNN_ERR_DIM;
  if (bad_stride(r->token_stride) || bad_stride(r->head_stride)) return SDNN_ERR_DIM;
  if (tokens > 0 && !r->data) return SDNN_ERR_NULL;
  return (uintptr_t)r->data % dtype_bytes(dtype) ? SDNN_ERR_DIM : SDNN_OK;
}

sdnn_status check_rotation(const sdnn_rotation* r, int32_t head_dim) {
  if (r->pairs < 0 || 2 * (int64_t)r->pairs > head_dim) return SDNN_ERR_DIM;
  if (r->layout != SDNN_ROPE_HALF && r->layout != SDNN_ROPE_INTERLEAVED) return SDNN_ERR_DIM;
  return r->pairs > 0 && !r->freq ? SDNN_ERR_NULL : SDNN_OK;
}

bool overlap(const void* a, int64_t abytes, const void* b, int64_t bbytes) {
  if (!a || !b || abytes <= 0 || bbytes <= 0) return false;
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a0 < b0 + (uintptr_t)bbytes && b0 < a0 + (uintptr_t)abytes;
}

// The same of two sets of rows of a_row and b_row bytes, `rows` of each, stride bytes apart: columns of one buffer may lie
// side by side.
bool overlap_rows(const void* a, int64_t a_row, const void* b, int64_t b_row, int64_t rows, int64_t stride) {
  if (!overlap(a, (rows - 1) * stride + a_row, b, (rows - 1) * stride + b_row)) return false;
  if (rows < 2 || stride == 0) return true;
  const int64_t between = (int64_t)((uintptr_t)b - (uintptr_t)a) % stride, off = between < 0 ? between + stride : between;
  return off < a_row || off + b_row > stride;
}

bool same_rows(const sdnn_heads& a, const sdnn_heads& b) {
  return a.data == b.data && a.token_stride == b.token_stride && a.head_stride == b.head_stride;
}
// Outputs have to lie apart from each other: a stride of zero would write one row for several.
bool distinct_rows(const sdnn_heads& a, int32_t tokens, int32_t head_dim) {
  return (tokens < 2 || a.token_stride != 0) && (a.heads < 2 || a.head_stride >= head_dim);
}

// (A call of more threads than a launch has is refused before it.)
sdnn_status result(hipError_t e) {
  return e == hipSuccess ? SDNN_OK : e == hipErrorInvalidConfiguration ? SDNN_ERR_DIM : SDNN_ERR_HIP;
}

#define SDNN_CHECK(call)                  \
  do {                                    \
    const sdnn_status st_ = (call);       \
    if (st_ != SDNN_OK) return st_;       \
  } while (0)

}  // namespace

extern "C" {

sdnn_status sdnn_rope(const sdnn_heads* x, const sdnn_heads* y, sdnn_dtype dtype, int32_t tokens,
                      int32_t head_dim, const int32_t* pos, const sdnn_rotation* rotation,
                      int32_t inverse, void* stream) {
  if (!rotation) return SDNN_ERR_NULL;
  if (bad_dtype(dtype) || tokens < 0 || head_dim < 1 || head_dim > kMaxHeadDim) return SDNN_ERR_DIM;
  if (inverse != 0 && inverse != 1) return SDNN_ERR_DIM;
  SDNN_CHECK(check_rows(x, 0, tokens, dtype));
  SDNN_CHECK(check_rows(y, x->heads, tokens, dtype));
  SDNN_CHECK(check_rotation(rotation, head_dim));
  if (!distinct_rows(*y, tokens, head_dim)) return SDNN_ERR_DIM;
  if (x->data == y->data && !same_rows(*x, *y)) return SDNN_ERR_DIM;
  if (tokens == 0) return SDNN_OK;
  if (!pos) return SDNN_ERR_NULL;
  return result(launch_rope(*x, *y, dtype, tokens, head_dim, pos, *rotation, inverse != 0, (hipStream_t)stream));
}

sdnn_status sdnn_cache_append(const sdnn_block_cache* cache, const sdnn_tokens* tokens,
                              const sdnn_heads* k, const sdnn_heads* v,
                              const sdnn_rotation* rotation, const sdnn_heads* q,
                              const sdnn_heads* q_out, void* stream) {
  SDNN_CHECK(check_cache(cache));
  SDNN_CHECK(check_tokens(tokens));
  SDNN_CHECK(check_rows(k, cache->kv_heads, tokens->tokens, cache->dtype));
  SDNN_CHECK(check_rows(v, cache->kv_heads, tokens->tokens, cache->dtype));
  if (rotation) SDNN_CHECK(check_rotation(rotation, cache->head_dim));
  if (!q != !q_out) return SDNN_ERR_NULL;
  if (q) {
    SDNN_CHECK(check_rows(q, 0, tokens->tokens, cache->dtype));
    SDNN_CHECK(check_rows(q_out, q->heads, tokens->tokens, cache->dtype));
    if (!distinct_rows(*q_out, tokens->tokens, cache->head_dim)) return SDNN_ERR_DIM;
    if (q->data == q_out->data && !same_rows(*q, *q_out)) return SDNN_ERR_DIM;
  }
  if (!cache->means != !cache->mean_scales) return SDNN_ERR_NULL;
  if (tokens->tokens == 0) return SDNN_OK;
  if (cache->pages > 0 && (!cache->k_pages || !cache->v_pages)) return SDNN_ERR_NULL;
  return result(launch_append(*cache, *tokens, *k, *v, rotation, q, q_out, (hipStream_t)stream));
}

sdnn_status sdnn_block_select(const sdnn_block_cache* cache, const sdnn_tokens* tokens,
                              const sdnn_heads* q, int32_t blocks, int32_t sink, int32_t local,
                              int32_t* chosen, void* stream) {
  SDNN_CHECK(check_cache(cache));
  SDNN_CHECK(check_tokens(tokens));
  SDNN_CHECK(check_rows(q, 0, tokens->tokens, cache->dtype));
  if (q->heads % cache->kv_heads || q->heads / cache->kv_heads > kMaxGroup) return SDNN_ERR_DIM;
  if (blocks < 1 || blocks > kMaxChosen || sink < 0 || local < 1 || (int64_t)sink + local > blocks)
    return SDNN_ERR_DIM;
  if (tokens->max_blocks > kMaxBlocks) return SDNN_ERR_DIM;
  if (tokens->tokens == 0) return SDNN_OK;
  if (!chosen) return SDNN_ERR_NULL;
  if (cache->pages > 0 && (!cache->means || !cache->mean_scales)) return SDNN_ERR_NULL;
  if (cache->pages == 0) return SDNN_ERR_DIM;  // the kernel reads the summary of page 0 in a missing page's place
  return result(launch_select(*cache, *tokens, *q, blocks, sink, local, chosen, (hipStream_t)stream));
}

int64_t sdnn_block_attend_floats(const sdnn_block_cache* cache, int32_t tokens, int32_t heads,
                                 int32_t blocks) {
  if (check_cache(cache) != SDNN_OK || tokens <= 0 || heads <= 0 || blocks <= 0 || heads % cache->kv_heads)
    return 0;
  return attend_floats(*cache, tokens, heads, blocks);
}

sdnn_status sdnn_block_attend(const sdnn_block_cache* cache, const sdnn_tokens* tokens,
                              const sdnn_heads* q, const sdnn_heads* o, const int32_t* chosen,
                              int32_t blocks, float scale, float* lse, float* workspace,
                              int64_t workspace_floats, void* stream) {
  SDNN_CHECK(check_cache(cache));
  SDNN_CHECK(check_tokens(tokens));
  SDNN_CHECK(check_rows(q, 0, tokens->tokens, cache->dtype));
  SDNN_CHECK(check_rows(o, q->heads, tokens->tokens, cache->dtype));
  if (q->heads % cache->kv_heads || q->heads / cache->kv_heads > kMaxGroup) return SDNN_ERR_DIM;
  if (!distinct_rows(*o, tokens->tokens, cache->head_dim)) return SDNN_ERR_DIM;
  if (!(scale > -1e30f && scale < 1e30f)) return SDNN_ERR_DIM;
  if (chosen && (blocks < 1 || blocks > kMaxBlocks)) return SDNN_ERR_DIM;
  if (!chosen) blocks = tokens->max_blocks;
  if (tokens->tokens == 0) return SDNN_OK;
  if (cache->pages > 0 && (!cache->k_pages || !cache->v_pages)) return SDNN_ERR_NULL;
  const int64_t need = sdnn_block_attend_floats(cache, tokens->tokens, q->heads, blocks);
  if (need > 0 && !workspace) return SDNN_ERR_NULL;
  if (need > 0 && (workspace_floats < need || bad_align(workspace))) return SDNN_ERR_DIM;
  if (need > 0 && (overlap(workspace, need * 4, lse, (int64_t)tokens->tokens * q->heads * 4) ||
                   workspace == q->data || workspace == o->data))
    return SDNN_ERR_DIM;
  return result(launch_attend(*cache, *tokens, *q, *o, chosen, blocks, scale, lse, workspace,
                              (hipStream_t)stream));
}

sdnn_status sdnn_qmat_create(const uint8_t* packed, const void* scales, sdnn_dtype scale_dtype,
                             const uint8_t* zeros, int32_t M, int32_t K, int32_t group,
                             void* stream, sdnn_qmat* out) {
  if (!out) return SDNN_ERR_NULL;
  *out = nullptr;
  if (!packed || !scales) return SDNN_ERR_NULL;
  if (bad_dtype(scale_dtype) || M < 1 || K < 1 || K > (1 << 20) || M > (1 << 24)) return SDNN_ERR_DIM;
  if (group != 32 && group != 64 && (group < kQChunk || group % kQChunk)) return SDNN_ERR_DIM;
  sdnn_qmat_s* w = new (std::nothrow) sdnn_qmat_s();
  if (!w) return SDNN_ERR_ALLOC;
  w->M = M, w->K = K, w->group = group, w->scale_dtype = scale_dtype, w->zeros = zeros != nullptr;
  w->chunks = (K + kQChunk - 1) / kQChunk;
  w->tiles = (M + kQTileRows - 1) / kQTileRows;
  const int64_t bytes = qmat_weight_bytes(*w);
  if (hipGetDevice(&w->device) != hipSuccess) {
    delete w;
    return SDNN_ERR_HIP;
  }
  if (hipMalloc(&w->d_mem, (size_t)(bytes + qmat_meta_bytes(*w))) != hipSuccess) {
    (void)hipGetLastError();
    delete w;
    return SDNN_ERR_ALLOC;
  }
  w->weights = static_cast<const uint8_t*>(w->d_mem);
  w->meta = w->weights + bytes;
  hipError_t e = launch_qmat_pack(*w, packed, scales, zeros, (hipStream_t)stream);
  if (e == hipSuccess) e = hipStreamSynchronize((hipStream_t)stream);
  if (e != hipSuccess) {
    (void)hipFree(w->d_mem);
    delete w;
    return SDNN_ERR_HIP;
  }
  *out = w;
  return SDNN_OK;
}

sdnn_status sdnn_qmat_apply(sdnn_qmat w, const void* x, int64_t x_feature, int64_t x_column, void* y,
                            int64_t y_feature, int64_t y_column, int32_t N, sdnn_dtype dtype,
                            const float* bias, sdnn_epilogue epi, void* stream) {
  if (!w) return SDNN_ERR_NULL;
  if (bad_dtype(dtype) || N < 0 || N > (1 << 18)) return SDNN_ERR_DIM;
  if (epi != SDNN_EPI_NONE && epi != SDNN_EPI_RELU && epi != SDNN_EPI_GELU) return SDNN_ERR_DIM;
  if (bad_stride(x_feature) || bad_stride(x_column) || bad_stride(y_feature) || bad_stride(y_column))
    return SDNN_ERR_DIM;
  if ((w->M > 1 && y_feature == 0) || (N > 1 && y_column == 0)) return SDNN_ERR_DIM;
  if (N == 0) return SDNN_OK;
  if (!x || !y) return SDNN_ERR_NULL;
  const int e = dtype_bytes(dtype);
  if ((uintptr_t)x % e || (uintptr_t)y % e) return SDNN_ERR_DIM;
  const int64_t xbytes = ((w->K - 1) * x_feature + (N - 1) * x_column + 1) * e;
  const int64_t ybytes = ((w->M - 1) * y_feature + (N - 1) * y_column + 1) * e;
  const bool meet = x_feature == 1 && y_feature == 1 && x_column == y_column
                        ? overlap_rows(x, (int64_t)w->K * e, y, (int64_t)w->M * e, N, x_column * e)
                        : overlap(x, xbytes, y, ybytes);
  if (meet || overlap(bias, (int64_t)w->M * 4, y, ybytes)) return SDNN_ERR_DIM;
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess) return SDNN_ERR_HIP;
  if (device != w->device) return SDNN_ERR_DEVICE;
  return result(launch_qmat(*w, x, x_feature, x_column, y, y_feature, y_column, N, dtype, bias, (int)epi,
                            (hipStream_t)stream));
}

void sdnn_qmat_destroy(sdnn_qmat w) {
  if (!w) return;
  int device = -1;
  (void)hipGetDevice(&device);
  if (device != w->device) (void)hipSetDevice(w->device);
  (void)hipFree(w->d_mem);
  if (device != w->device && device >= 0) (void)hipSetDevice(device);
  delete w;
}

}  // extern "C"
