// What the host side of sdnn_serve.h and its kernels share.
#ifndef SDNN_SERVE_INTERNAL_H_
#define SDNN_SERVE_INTERNAL_H_

#include "../../include/sdnn_serve.h"
#include "sdnn_decode_internal.h"

namespace sdnn {

constexpr int kMaxVocab = 1 << 19;
constexpr int kMaxShared = 1 << 20;  // blocks of a shared prefix

hipError_t launch_norm(const sdnn_heads& q, const sdnn_heads& q_out, const sdnn_heads* k, const sdnn_heads* k_out, int dtype,
                       int32_t tokens, int32_t head_dim, const int32_t* pos, const sdnn_head_norm& norm,
                       const sdnn_rotation* rotation, hipStream_t stream);
hipError_t launch_q8_append(const sdnn_q8_cache& c, const sdnn_tokens& t, int dtype, const sdnn_heads& k, const sdnn_heads& v,
                            const sdnn_head_norm* norm, const sdnn_rotation* rotation, const sdnn_heads* q,
                            const sdnn_heads* q_out, hipStream_t stream);
hipError_t launch_q8_read(const sdnn_q8_cache& c, const sdnn_tokens& t, int dtype, const sdnn_heads* k, const sdnn_heads* v,
                          hipStream_t stream);
hipError_t launch_q8_attend(const sdnn_q8_cache& c, const sdnn_tokens& t, int dtype, const sdnn_heads& q, const sdnn_heads& o,
                            const int32_t* chosen, int32_t blocks, int32_t shared, float scale, float* lse, float* workspace,
                            hipStream_t stream);
hipError_t launch_sample(const void* logits, int64_t row_stride, int dtype, int32_t rows, int32_t vocab, const float* u,
                         const sdnn_sampling& settings, int32_t* token, float* logprob, float* workspace, hipStream_t stream);

}  // namespace sdnn

#endif  // SDNN_SERVE_INTERNAL_H_
