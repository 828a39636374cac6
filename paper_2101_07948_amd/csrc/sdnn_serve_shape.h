// Launch shapes of the operators of sdnn_serve.h: arithmetic on sizes, without a GPU.
#ifndef SDNN_SERVE_SHAPE_H_
#define SDNN_SERVE_SHAPE_H_

#include "sdnn_decode_shape.h"
#include "sdnn_serve_internal.h"

namespace sdnn {

// ---------------------------------------------------------------- rows of heads

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kRowRun = 8;     // most tokens of a workgroup that has rows of heads
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

// Rows that are normed, rotated and stored: a workgroup has a run of tokens and `shares` workgroups share a run's tasks.  Long
// runs share cosines and sines among more heads and keep loads under way, where they leave workgroups enough for the device.
struct RunShape {
  int32_t lanes, tasks, run, shares;
  int64_t groups;
};
inline RunShape run_shape(int32_t tokens, int units, const int (&heads)[3]) {
  RunShape s = {};
  s.lanes = row_lanes(units);
  for (const int h : heads) s.tasks += row_tasks(h, s.lanes);
  s.run = 1, s.shares = 1;
  while (s.run < kRowRun && tokens >= 640 * s.run) s.run *= 2;
  while (s.run == 1 && s.shares * kRowWaves < s.tasks && tokens * s.shares < 2048) ++s.shares;
  s.groups = ((int64_t)tokens + s.run - 1) / s.run * s.shares;
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

constexpr int kSampleThreads = 1024;  // of a workgroup that has a row
constexpr int kSamplePass = 256;      // of one that passes over a part of one
constexpr int kSampleBins = 2048;
constexpr int kSampleList = 2048;    // tokens that are put in order in LDS
constexpr int kMostSampleParts = 64;

// What a row asks for; limits that leave everything are 0 (top_k, min_p) or 1 (top_p).
struct Limits {
  float temperature, top_p, min_p, u;
  int32_t top_k;
  int32_t first;  // only the first token is left
};

// What a row's weights are made by.
struct Weights {
  float top;     // the largest logit; 0 where that is infinite
  double scale;  // log2 e / temperature
};

// What the bins of a row's weights tell of its limits:
//   kWhole: they leave every token that has a weight;
//   kShort: what they leave is among the `tokens` tokens up to and with bin `edge`, which a list holds;
//   kEdges: the last token that top_k leaves is among the `tokens` of bin `edge` (-1: no top_k, or it leaves all), after `rank`
//           others of it; the last one that top_p leaves is among the `tokens_p` of bins `edge_p` to `end_p` (-1: no top_p);
//   kOther: none of these.
// mass, mass_p: before bins edge and edge_p; total: of all bins.
enum CutKind : int32_t { kWhole, kShort, kEdges, kOther };
struct Cut {
  CutKind kind;
  int32_t edge, edge_p, end_p;
  uint32_t tokens, tokens_p, rank;
  uint64_t mass, mass_p, total;
};

// The logits of tokens that go to lists: from at[0] on and below at[1], from at[2] on and below at[3].
struct Ranges {
  float at[4];
};

// The tokens that are left: those with a logit above `logit`, and of those that have it the ones up to `index`.
struct Kept {
  float logit;
  int32_t index;
};

// Of a row that several workgroups share.
struct alignas(16) SampleSpace {
  Limits limits;
  Weights weights;
  Cut cut;
  Ranges ranges;
  Kept kept;
  uint64_t first;                     // token, of the row
  uint64_t firsts[kMostSampleParts];  // and of each part
  uint64_t masses[kMostSampleParts];
  uint64_t mass[kSampleBins];
  uint64_t list[kSampleList], list_p[kSampleList];
  uint32_t count[kSampleBins];
  int32_t listed, listed_p;
};

// Workgroups that share a row, each with about 4096 tokens (more where a row has kMostSampleParts of them or all rows 4096);
// 0: a row to a workgroup, in one launch.  Seven launches take 24 us
// before their first pass counts, and then share a row's passes out, which one workgroup makes at about 4 tokens a
// nanosecond.  One row in 32 bits, in one launch and shared out: of 32000 tokens top_k and top_p 20 us and 29, top_p alone 32 and
// 37, no limit 17 and 25; of 50021 25 and 28, 41 and 35, 23 and 25; of 65000 30 and 28, 51 and 34, 26 and 26; of 131001 in 16
// bits top_k and top_p 48 and 28.  128 of
// these with all kinds of limits 87 and 117, 256 of them 126 and 123.  (Parts of 2048, 4096, 8192 and 16384 tokens: one row 27,
// 28, 32 and 40 us, 32 rows 65, 59, 62 and 80.  Four launches, in which the last of a row's workgroups goes on with what all have
// left in memory: one row 24 us, but 128 rows 145 to 173: each workgroup's release writes its XCD's L2 back.)
inline int sample_parts(int32_t rows, int32_t vocab) {
  if (vocab <= 57344 || rows > vocab / 900) return 0;
  return std::min((vocab + 4095) / 4096, std::min(kMostSampleParts, 4096 / rows));
}
inline int64_t sample_floats(int32_t rows, int32_t vocab) {
  return sample_parts(rows, vocab) ? (int64_t)rows * (int64_t)(sizeof(SampleSpace) / 4) : 0;
}

}  // namespace sdnn

#endif  // SDNN_SERVE_SHAPE_H_
