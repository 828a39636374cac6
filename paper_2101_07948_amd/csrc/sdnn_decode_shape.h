// Launch shapes of the operators of sdnn_decode.h: arithmetic on sizes, without a GPU.
#ifndef SDNN_DECODE_SHAPE_H_
#define SDNN_DECODE_SHAPE_H_

#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "sdnn_decode_internal.h"

namespace sdnn {

// A launch has fewer than 2^32 threads.
inline bool launchable(int64_t workgroups, int threads) { return workgroups <= 0xffffffffll / threads; }

// ---------------------------------------------------------------- rotation, append

constexpr int kRopeThreads = 256;  // of both kernels
// Tokens of a workgroup (8192 tokens of 32 heads of 128: 1, 2, 4 and 8 tokens to a workgroup 29.3, 29.1, 28.9 and 39.1 us;
// few tokens fill the device only one by one).
inline int rope_tile(int32_t tokens) { return tokens >= 2048 ? 4 : 1; }
inline int64_t rope_groups(int32_t tokens) { return ((int64_t)tokens + rope_tile(tokens) - 1) / rope_tile(tokens); }

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

// ---------------------------------------------------------------- choice of blocks

constexpr int kWaveKeys = 16;  // keys of a lane where a wave chooses alone: up to 1024 blocks

struct SelectShape {
  int32_t tile;       // tokens of a workgroup
  int32_t per_token;  // rows of a token
  int32_t threads;
  int64_t groups;
};

inline SelectShape select_shape(const sdnn_block_cache& c, const sdnn_tokens& t, int32_t heads) {
  SelectShape s = {};
  const int group = heads / c.kv_heads;
  // A workgroup has several tokens where most of them are of one sequence and a wave can select alone: so
  // many that their rows fill two matrix operands (2048 tokens of 4 queries to a head over 512 blocks: one operand
  // 44 us, two 38, four 51, whose LDS leaves fewer workgroups to a compute unit), their keys at most 64 KiB of
  // LDS, and that the device is full.
  // Otherwise it has one token, and so many waves that each has some blocks.
  int rows = 1;
  while (rows < group && rows < 16) rows *= 2;
  const bool tiles = t.tokens >= (int64_t)16 * t.sequences && t.max_blocks <= 64 * kWaveKeys &&
                     (int64_t)(t.tokens / (16 / rows)) * c.kv_heads >= 512 && group <= 16;
  s.tile = 1;
  if (tiles) {
    s.tile = 16 / rows;
    while (s.tile * rows < 32 && s.tile * 2 * t.max_blocks <= 16384 &&
           (int64_t)(t.tokens / (s.tile * 2)) * c.kv_heads >= 1024)
      s.tile *= 2;
  }
  s.per_token = tiles ? rows : (group + 15) & ~15;
  s.threads = 64;
  while (s.threads < 1024 && s.threads < t.max_blocks) s.threads *= 2;
  if (tiles) s.threads = 256;
  s.groups = ((int64_t)t.tokens + s.tile - 1) / s.tile * c.kv_heads;
  return s;
}

// ---------------------------------------------------------------- attention

constexpr int kWaves = 4;      // of a workgroup of attend_kernel
constexpr int kTileWaves = 8;  // and of attend_tiles
constexpr int kRows = 16;      // queries of a tile: the columns of one matrix instruction
constexpr int kFewParts = 8;   // that attend_join_few joins
constexpr int kMostParts = 64; // of a query (the lanes of attend_join)

// Waves of a SIMD that the registers of attend_kernel leave room for, and so its workgroups at work at once on a compute
// unit, for heads of up to 16 * tiles values.  (For the compiler a bound: without one it takes registers of both kinds
// and leaves room for one wave less.  3 waves fit for heads of 128 in 16 bits too, but read worse: 64 tokens of 8 heads
// over 32 blocks of 64 tokens, 537 MB, 107 us with 3 and 95 with 2.)
constexpr int attend_waves(int tiles) { return tiles <= 4 ? 4 : tiles <= 6 ? 3 : tiles <= 12 ? 2 : 1; }

// How attend_tiles takes a call: tokens of a wave's tile (a token's queries take a power of two of its 16 rows), and
// shares of the blocks; tokens 0: attend_kernel does.
struct Tiles {
  int tokens, splits;
};
inline int tile_of(const sdnn_block_cache& c, int32_t heads) {
  int rows = 1;
  while (rows < heads / c.kv_heads && rows < kRows) rows *= 2;
  return kRows / rows;
}
inline int64_t tile_groups(const sdnn_block_cache& c, int32_t tokens, int32_t heads) {
  const int each = tile_of(c, heads) * kTileWaves;
  return ((int64_t)tokens + each - 1) / each * c.kv_heads * ((heads / c.kv_heads + kRows - 1) / kRows);
}
constexpr int64_t kTileRoom = 512;  // workgroups at work at once
// The most shares that a call of so many tokens is split into.
inline int tile_splits(const sdnn_block_cache& c, int32_t tokens, int32_t heads) {
  const int64_t groups = tile_groups(c, tokens, heads);
  int s = 1;
  while (s < kFewParts && tokens >= 16 && groups * 2 * s <= kTileRoom) s *= 2;
  return s;
}

// attend_tiles serves a call where many tokens of a sequence are neighbours, as far as the sizes tell, and it is estimated
// to be faster.  (Sequences are counted by the table's rows.  What that costs where it is wrong, 2048 tokens of a sequence over
// 16 of 128 blocks: 0.2 ms; with a table of 256 rows, token by token, 0.9; with single tokens of 64 other sequences,
// whose lists a workgroup walks one after the other, 1.4, and over all blocks 9.4 where two calls take 0.8.)
// attend_kernel reads every token's blocks from L2, at about 8 TB/s (16384 heads of 16 blocks of 32 KiB:
// 994 us; 8760 of 3 of 128 KiB: 683).  attend_tiles takes its workgroups' unions of blocks, 512 workgroups at a
// time, two to a compute unit, at about 3.7 us for 32 KiB, or 2.2 where they have a unit each (38 and 133 of them: 142 and
// 288 us; the matrix instructions of 32 bits take four times as long).  How large a union is depends on the lists:
// between three of them, where neighbours choose alike, and what lists that have nothing in common cover (107 tokens of
// 4 of 468 blocks of 4 KiB, 12 heads: 280 blocks, 74 us; one by one 20), whose geometric mean is taken.  Where few
// workgroups leave compute units idle the blocks are shared out, and the parts joined at the rate of a copy (512 tokens
// at the end of 8512, 8 heads of 128: 1 share 288 us, 4 shares 123 and 8 to join; 900 tokens of a sequence's first 900,
// whose longest lists have 15 blocks: 41, and 2 shares 33 and 11 to join).
inline Tiles tiles_of(const sdnn_block_cache& c, int32_t tokens, int32_t sequences, int32_t max_blocks, int32_t heads,
                      int32_t chosen) {
  if (max_blocks > 1 << 20 || tokens < (int64_t)16 * sequences) return {0, 1};
  const int tile = tile_of(c, heads), head_tiles = (heads / c.kv_heads + kRows - 1) / kRows;
  const double page = 2.0 * c.block * c.head_dim * dtype_bytes(c.dtype);
  const int each = chosen > 0 && chosen < max_blocks ? chosen : max_blocks;
  const double few = chosen > 0 && chosen < max_blocks / 3 ? 3.0 * chosen : max_blocks;
  const double many = max_blocks * (1.0 - std::pow(1.0 - (double)each / max_blocks, std::min(tokens, tile * kTileWaves)));
  const double all = few < many ? std::sqrt(few * many) : few;
  const double groups = (double)tile_groups(c, tokens, heads);
  const double one_by_one = (double)tokens * c.kv_heads * head_tiles * each * page / 8e6;
  const double parts = 8.0 * tokens * heads * (c.head_dim + 2) / 4e6;
  const auto tiled_in = [&](int shares) {
    const double at_once = std::min(std::max(groups * shares / 256, 1.0), 2.0), rounds = std::max(groups * shares / kTileRoom, 1.0);
    const double block = page / 32768 * (0.7 + 1.5 * at_once * (c.dtype == SDNN_F32 ? 4 : 1));
    return rounds * all / shares * block + (shares > 1 ? shares * parts + 5 : 0.0);
  };
  int best = 1;
  for (int s = 2; s <= tile_splits(c, tokens, heads); s *= 2)
    if (tiled_in(s) < tiled_in(best)) best = s;
  const double tiled = tiled_in(best);
  return tiled < one_by_one ? Tiles{tile, best} : Tiles{0, 1};
}

// Shares of a token's blocks: so many that about 1024 workgroups (4 for each compute unit) are at work, so that those of
// long sequences have company to the end; but where a wave would have fewer than 4 steps, no more than are at work at
// once, since another round of workgroups costs more than it shares out (732 tokens of a head of 192 over 4 blocks of
// 128: 2 shares 53 us and the join, 1 share 31; 22 tokens of 2 heads over lists of 64 blocks that are nearly empty: 24
// shares 24 us, 11 shares 8).  A wave has a step of its own at least, and there are at most 64 shares (the lanes of
// attend_join).  Where all blocks are 192 KiB or less, 48 to a wave, they are not shared out: the join, a launch of its
// own, would take longer (1 to 16 tokens of 1 to 32 heads of 128 in 16 bits over blocks of 32 KiB, a call, not shared out
// and shared out: 4 blocks 8.0 to 8.6 us and 10.3 to 10.8, 6 blocks 9.7 to 10.1 and 10.4 to 11.8; 8, shared out, 10.3 to
// 12.3).
inline int attend_splits(const sdnn_block_cache& c, int32_t tokens, int32_t heads, int32_t blocks) {
  const int64_t units = (int64_t)tokens * c.kv_heads * ((heads / c.kv_heads + kRows - 1) / kRows);
  if (units == 0) return 1;
  const int step = c.dtype == SDNN_F32 ? 16 : 32;
  const int64_t steps = (int64_t)blocks * (c.block / step), most = (steps + kWaves - 1) / kWaves;
  if (blocks * 2ll * c.block * c.head_dim * dtype_bytes(c.dtype) <= 192 * 1024) return 1;
  int64_t wanted = (1024 + units - 1) / units;
  if (steps < 4 * kWaves * wanted) wanted = 256 * attend_waves((c.head_dim + 15) / 16) / units;
  const int64_t s = wanted < most ? wanted : most;
  return (int)(s < 1 ? 1 : s > kMostParts ? kMostParts : s);
}

inline int64_t attend_floats(const sdnn_block_cache& c, int32_t tokens, int32_t heads, int32_t blocks) {
  const int s = std::max(attend_splits(c, tokens, heads, blocks), tile_splits(c, tokens, heads));
  return s > 1 ? (int64_t)s * tokens * heads * (c.head_dim + 2) : 0;
}

struct AttendShape {
  int32_t tile_tokens;  // 0: attend_kernel; else attend_tiles, tokens of a wave's tile
  int32_t splits;
  int64_t groups;
  int32_t threads;
  int64_t join_groups;  // of 256 threads; 0: no parts
};

// Workgroups of the join of `parts` parts of `rows` queries (0: no parts).
inline int64_t join_groups(int32_t parts, int64_t rows, int32_t head_dim) {
  return parts <= 1 ? 0 : parts <= kFewParts ? (rows * (head_dim / 4) + 255) / 256 : rows;
}

// (chosen: blocks of a token's list; 0: all of them)
inline AttendShape attend_shape(const sdnn_block_cache& c, const sdnn_tokens& t, int32_t heads, int32_t chosen,
                                int32_t most_splits = kMostParts) {
  AttendShape s = {};
  const Tiles tiles = tiles_of(c, t.tokens, t.sequences, t.max_blocks, heads, chosen);
  s.tile_tokens = tiles.tokens;
  s.splits = tiles.tokens ? tiles.splits : attend_splits(c, t.tokens, heads, chosen > 0 ? chosen : t.max_blocks);
  s.splits = std::min(s.splits, most_splits);
  s.threads = 64 * (tiles.tokens ? kTileWaves : kWaves);
  const int head_tiles = (heads / c.kv_heads + kRows - 1) / kRows;
  s.groups = s.splits * (tiles.tokens ? tile_groups(c, t.tokens, heads) : (int64_t)t.tokens * head_tiles * c.kv_heads);
  s.join_groups = join_groups(s.splits, (int64_t)t.tokens * heads, c.head_dim);
  return s;
}

// Attention with a shared prefix (sdnn_block_attend_shared): `prefix` is a launch of attend_tiles whose rows are all tokens'
// queries, in shares of its blocks; `own` the launch over the blocks after it (splits 0: there are none).
struct SharedShape {
  AttendShape prefix, own;
  int32_t parts;
  int64_t join_groups;
  bool fits;
};

// Shares of the prefix: so many that two workgroups are at work on each compute unit, of two blocks at least.
inline int prefix_splits(int64_t groups, int32_t shared) {
  int s = 1;
  while (s < 32 && groups * 2 * s <= kTileRoom && s * 4 <= shared) s *= 2;
  return s;
}

inline SharedShape shared_shape(const sdnn_block_cache& c, int32_t tokens, int32_t sequences, int32_t max_blocks, int32_t heads,
                                int32_t shared) {
  SharedShape s = {};
  const int64_t groups = tile_groups(c, tokens, heads);
  s.prefix.tile_tokens = tile_of(c, heads);
  s.prefix.splits = prefix_splits(groups, shared);
  s.prefix.groups = s.prefix.splits * groups;
  s.prefix.threads = 64 * kTileWaves;
  if (max_blocks > shared) {
    sdnn_tokens t = {};
    t.tokens = tokens, t.sequences = sequences, t.max_blocks = max_blocks - shared;
    s.own = attend_shape(c, t, heads, 0, kMostParts - s.prefix.splits);
  }
  s.parts = s.prefix.splits + s.own.splits;
  s.join_groups = join_groups(s.parts, (int64_t)tokens * heads, c.head_dim);
  s.fits = launchable(s.prefix.groups, s.prefix.threads) && launchable(s.own.groups, 64 * kTileWaves) &&
           launchable(s.join_groups, 256);
  return s;
}

// (The table's rows are not known here: the most that any number of them needs.)
inline int64_t shared_floats(const sdnn_block_cache& c, int32_t tokens, int32_t heads, int32_t blocks, int32_t shared) {
  const int own = std::max(attend_splits(c, tokens, heads, blocks - shared), tile_splits(c, tokens, heads));
  const int64_t parts = prefix_splits(tile_groups(c, tokens, heads), shared) + (blocks > shared ? own : 0);
  return std::max(parts > 1 ? parts * tokens * heads * (c.head_dim + 2) : 0, attend_floats(c, tokens, heads, blocks));
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
