// Launch shapes of the operators of sdnn_decode.h: arithmetic on sizes, without a GPU.
#ifndef SDNN_DECODE_SHAPE_H_
#define SDNN_DECODE_SHAPE_H_

#include <stddef.h>
#include <stdint.h>

#include "sdnn_decode_internal.h"

namespace sdnn {

constexpr int kWindow = 64;       // tokens of an append workgroup, the most
constexpr int kTileBytes = 32768; // the most of a window's keys
constexpr int kCus = 256;
constexpr int kSumRows = 8;       // keys of a block that a thread adds

// Bytes of LDS of a window's rotated keys [token][head_dim], and of its values, whose rows are a piece longer.
__host__ __device__ constexpr int key_bytes(int window, int head_dim, int size) { return (window * head_dim * size + 15) & ~15; }
__host__ __device__ constexpr int value_bytes(int window, int head_dim, int size) {
  return window * (head_dim * size + 16);
}

struct AppendShape {
  int32_t window;   // tokens of a workgroup
  int32_t before;   // bytes of LDS before the rows of a block's keys that lie before the window
  int32_t passes;   // of a mean, each with a part of those rows
  size_t lds;
  int64_t windows;
};

inline AppendShape append_shape(const sdnn_block_cache& c, const sdnn_tokens& t) {
  AppendShape s = {};
  const int size = dtype_bytes(c.dtype);
  // one token to a workgroup; in prompts, and where single tokens fill the device several times, windows
  // whose values are written in runs
  s.window = 1;
  if ((int64_t)t.tokens * c.kv_heads > 4096 || t.tokens >= (int64_t)16 * t.sequences)
    s.window = kWindow * c.head_dim * size <= kTileBytes ? kWindow : kWindow / 2;
  // Prompts that leave compute units without one take shorter windows: a window's steps follow one another, and so do
  // its means, while what a shorter one rotates again of a block it shares is little.  (Kernel, us: windows of 64, 32
  // and 16: 941 tokens of 3 heads of 128, blocks of 32: 26, 15, 15; 714 of 1 head, blocks of 64: 22, 20, 17; 186 of
  // 12 heads of 192, blocks of 128: 18, 12, 9; 1000 of 8 heads of 128 in 32 bits, blocks of 128: 29, 31, 31.)
  while (s.window > kWindow / 4 && (int64_t)t.tokens * c.kv_heads < (int64_t)kCus * s.window) s.window /= 2;
  // LDS: the keys, then the values or the sums of a mean, then a block's keys from before the window
  const size_t sums = (size_t)c.block / kSumRows * c.head_dim * sizeof(float);
  const size_t keys = key_bytes(s.window, c.head_dim, size), values = value_bytes(s.window, c.head_dim, size);
  s.lds = keys + (values > sums ? values : sums);
  s.before = (int32_t)((s.lds + 15) & ~(size_t)15);
  s.passes = 1;
  // Windows are shifted by the first token's place in its block, so that a call of no more tokens than a window holds
  // has a second one too: every token but the first may have tokens of its block before its window.
  if (c.means && t.tokens > 1) {
    // (the rows may take the place that the values had, past the sums)
    s.before = (int32_t)(keys + ((sums + 15) & ~(size_t)15));
    while (s.before + key_bytes(c.block / s.passes, c.head_dim, size) > 128 * 1024) s.passes *= 2;
    const size_t with = s.before + key_bytes(c.block / s.passes, c.head_dim, size);
    if (with > s.lds) s.lds = with;
  }
  s.windows = ((int64_t)t.tokens + s.window - 1) / s.window + (s.window > 1);  // one more where they are shifted
  return s;
}

// ---------------------------------------------------------------- 4-bit weights

inline int32_t groups_of(const sdnn_qmat_s& w) { return (int32_t)(((int64_t)w.K + w.group - 1) / w.group); }
// Of a tile's scales: entries along K, and scales of each entry and row.
inline int32_t metas_of(const sdnn_qmat_s& w) { return w.group >= kQChunk ? groups_of(w) : w.chunks; }
inline int32_t inner_of(const sdnn_qmat_s& w) { return w.group >= kQChunk ? 1 : kQChunk / w.group; }
inline int64_t scales_of(const sdnn_qmat_s& w) { return (int64_t)w.tiles * metas_of(w) * inner_of(w) * kQTileRows; }
// Bytes of the laid-out weights and of their scales and zero points.
inline int64_t qmat_weight_bytes(const sdnn_qmat_s& w) { return (int64_t)w.tiles * w.chunks * 1024; }
inline int64_t qmat_meta_bytes(const sdnn_qmat_s& w) {
  return scales_of(w) * (dtype_bytes(w.scale_dtype) + (w.zeros ? 1 : 0));
}

}  // namespace sdnn

#endif  // SDNN_DECODE_SHAPE_H_
