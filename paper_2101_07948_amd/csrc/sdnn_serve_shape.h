// Launch shapes of the operators of sdnn_serve.h: arithmetic on sizes, without a GPU.
#ifndef SDNN_SERVE_SHAPE_H_
#define SDNN_SERVE_SHAPE_H_

#include "sdnn_decode_shape.h"
#include "sdnn_serve_internal.h"

namespace sdnn {

// ---------------------------------------------------------------- rows of heads

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kQ8Window = 64;  // tokens of a workgroup that turns values

// Pairs to a unit: a lane holds 2 of these values of a row, in two accesses (pairs half a head apart) or one (neighbours), of
// 16 bytes where the row's parts divide by them.
inline int row_pairs(int dtype, int layout, int pairs, int head_dim) {
  int v = 16 / dtype_bytes(dtype) / (layout == SDNN_ROPE_INTERLEAVED ? 2 : 1);
  while (v > 1 && (pairs % v || (head_dim - 2 * pairs) % (2 * v))) v /= 2;
  return v;
}

// A row takes `lanes` lanes of a wave, a task of a wave is 64 / lanes heads of one kind of a token, and `waves` waves share a
// token's tasks: one where tokens fill the device, else as many as there are tasks.
struct RowShape {
  int32_t lanes, waves, tasks;
  int64_t groups;
};
inline int row_tasks(int heads, int lanes) { return (heads * lanes + 63) / 64; }
inline int row_lanes(int units) {
  int l = 1;
  while (l < units && l < 64) l *= 2;
  return l;
}
inline RowShape row_shape(int32_t tokens, int units, const int (&heads)[3]) {
  RowShape s = {};
  s.lanes = row_lanes(units);
  for (const int h : heads) s.tasks += row_tasks(h, s.lanes);
  s.waves = 1;
  while (s.waves < s.tasks && (int64_t)tokens * s.waves < 4096) ++s.waves;
  s.groups = ((int64_t)tokens * s.waves + kRowWaves - 1) / kRowWaves;
  return s;
}

// Whether values are turned by windows of tokens (prompts) or written and read one by one.
inline bool by_windows(const sdnn_tokens& t) { return t.tokens >= 8 && t.tokens >= (int64_t)4 * t.sequences; }
inline int64_t window_groups(const sdnn_tokens& t, int32_t heads) {
  return ((int64_t)t.tokens + kQ8Window - 1) / kQ8Window * heads;
}

// Tokens of a workgroup that looks for full blocks and writes their means.
inline int mean_range(const sdnn_tokens& t, int32_t heads) { return (int64_t)t.tokens * heads > 4096 ? 64 : 1; }
inline int64_t mean_groups(const sdnn_tokens& t, int32_t heads) {
  const int range = mean_range(t, heads);
  return ((int64_t)t.tokens + range - 1) / range * heads;
}

// ---------------------------------------------------------------- attention

// The cache as one of 16-bit values, for the rules that go by sizes.
inline sdnn_block_cache as_blocks(const sdnn_q8_cache& c) {
  sdnn_block_cache b = {};
  b.pages = c.pages, b.kv_heads = c.kv_heads, b.head_dim = c.head_dim, b.block = c.block, b.dtype = SDNN_BF16;
  return b;
}

// ---------------------------------------------------------------- sampling

constexpr int kSampleThreads = 1024;
constexpr int kSampleBins = 8192;

inline int64_t sample_floats(int32_t, int32_t) { return 0; }

}  // namespace sdnn

#endif  // SDNN_SERVE_SHAPE_H_
