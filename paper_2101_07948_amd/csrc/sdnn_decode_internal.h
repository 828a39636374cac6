// What the host side of sdnn_decode.h and its kernels share.
#ifndef SDNN_DECODE_INTERNAL_H_
#define SDNN_DECODE_INTERNAL_H_

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/sdnn_decode.h"

struct sdnn_qmat_s {
  int32_t M, K, group;
  int32_t scale_dtype;
  int32_t zeros;    // zero points given
  int32_t device;
  int32_t chunks;   // of kQChunk columns
  int32_t tiles;    // of 16 rows
  void* d_mem;      // the weights, then the scales (see sdnn_qmat.hip)
  const uint8_t* weights;
  const uint8_t* meta;
};

namespace sdnn {

constexpr int kMaxHeadDim = 256;
constexpr int kMaxBlocks = 32768;       // of a sequence, for sdnn_block_select
constexpr int kMaxChosen = 1024;
constexpr int kMaxGroup = 64;           // queries to a cached head
constexpr int kQChunk = 128;            // columns of a 4-bit weight tile
constexpr int kQTileRows = 16;

inline int dtype_bytes(int dtype) { return dtype == SDNN_F32 ? 4 : 2; }

hipError_t launch_rope(const sdnn_heads& x, const sdnn_heads& y, int dtype, int32_t tokens, int32_t head_dim,
                       const int32_t* pos, const sdnn_rotation& r, bool inverse, hipStream_t stream);
hipError_t launch_append(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& k,
                         const sdnn_heads& v, const sdnn_rotation* r, const sdnn_heads* q,
                         const sdnn_heads* q_out, hipStream_t stream);
hipError_t launch_select(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q,
                         int32_t blocks, int32_t sink, int32_t local, int32_t* chosen, hipStream_t stream);
hipError_t launch_attend(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q,
                         const sdnn_heads& o, const int32_t* chosen, int32_t blocks, float scale,
                         float* lse, float* workspace, hipStream_t stream);
hipError_t launch_attend_shared(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q,
                                const sdnn_heads& o, int32_t shared, float scale, float* lse, float* workspace,
                                hipStream_t stream);
hipError_t launch_qmat_pack(const sdnn_qmat_s& w, const uint8_t* packed, const void* scales,
                            const uint8_t* zeros, hipStream_t stream);
hipError_t launch_qmat(const sdnn_qmat_s& w, const void* x, int64_t x_feature, int64_t x_column, void* y,
                       int64_t y_feature, int64_t y_column, int32_t N, int dtype, const float* bias,
                       int epi, hipStream_t stream);

}  // namespace sdnn

#endif  // SDNN_DECODE_INTERNAL_H_
