// The choice of blocks by the score of their summaries.
#include "sdnn_decode_device.h"
#include "sdnn_decode_shape.h"

namespace sdnn {
namespace {

struct SelectArgs {
  const void* q;
  int64_t q_token, q_head;
  const int8_t* means;
  const float* scales;
  int64_t pages;
  const int32_t* pos;
  const int32_t* seq;
  const int32_t* table;
  int32_t* chosen;
  int32_t tokens, sequences, max_blocks;
  int32_t kv_heads, group, head_dim, block_shift;
  int32_t blocks, sink, local;
  int32_t tile, per_token;  // tokens of a workgroup, rows of a token (up to 16: a power of two)
  int32_t keys, stride;     // where the keys begin in LDS; of a token
  int32_t dtype, q_aligned;
};

// A number whose order as an unsigned integer is the order of the floats (-0 counts as 0); below 2^32 - 1, so
// that the next number exists.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return min(u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u), 0xfffffffeu);
}

// Sums of two counts over the workgroup's threads before this one, and over all of them.  `parts`: a word for
// each wave.
__device__ __forceinline__ uint2 before(uint2 n, uint2* parts, uint2* all) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
  uint2 s = n;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t x = __shfl_up(s.x, d), y = __shfl_up(s.y, d);
    if (lane >= d) s.x += x, s.y += y;
  }
  if (lane == 63) parts[wave] = s;
  __syncthreads();
  uint2 r = make_uint2(s.x - n.x, s.y - n.y);
  *all = make_uint2(0, 0);
  for (int w = 0; w < waves; ++w) {
    if (w < wave) r.x += parts[w].x, r.y += parts[w].y;
    all->x += parts[w].x, all->y += parts[w].y;
  }
  return r;
}

// x of the lane N further on among 16.
template <int N, typename X>
__device__ __forceinline__ X rotated(X x) {
  return __builtin_bit_cast(X, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x120 + N, 0xf, 0xf, false));
}

// The largest of a wave's 64 keys.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max(x, rotated<8>(x));
  x = max(x, rotated<4>(x));
  x = max(x, rotated<2>(x));
  x = max(x, rotated<1>(x));
  const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max(p[0], p[1]);
  const auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return __builtin_amdgcn_readfirstlane(max(q[0], q[1]));
}

// The largest number that at least `want` of a wave's 64 keys reach (0 if fewer are above 0), bit by bit
// from the top, or a smaller one that exactly `want` reach.  Most often it has the exponent of the largest key or one
// of the next below: these are tried first.
__device__ __forceinline__ uint32_t wave_kth(uint32_t key, uint32_t want) {
  constexpr uint32_t kExponent = 1u << 23;
  uint32_t t = wave_max(key) & ~(kExponent - 1), bit = kExponent >> 1;
  for (int i = 0;; ++i) {
    const uint32_t n = __popcll(__ballot(key >= t));
    if (n == want) return t;
    if (n > want) break;
    if (i == 4 || t == 0) {
      t = 0, bit = 1u << 31;
      break;
    }
    t -= kExponent;
  }
  for (; bit; bit >>= 1) {
    const uint32_t n = __popcll(__ballot(key >= (t | bit)));
    if (n >= want) t |= bit;
    if (n == want) break;
  }
  return t;
}

// Writes the blocks of the `want` largest of a wave's keys in lane order, ties to the lower lane.  Lanes without
// a key have 0 and are the last.
__device__ __forceinline__ void write_largest(uint32_t key, int32_t block, uint32_t want, int32_t* chosen) {
  const uint32_t t = wave_kth(key, want);
  const uint64_t lower = (1ull << (threadIdx.x % 64)) - 1;
  const uint64_t above = __ballot(key > t), same = __ballot(key == t);
  const uint32_t left = want - __popcll(above);  // of the keys equal to t
  const bool taken = key > t || (key == t && __popcll(same & lower) < left);
  const uint64_t all = __ballot(taken);
  if (taken) chosen[__popcll(all & lower)] = block;
}

// A key and its block that may be among the largest.
struct Candidate {
  uint32_t key;
  int32_t block;
};

// Of one token's `count` keys in LDS a wave writes the blocks of the `want` largest in order (want < count).
// The want-th largest of the lanes' own maxima is reached by at least `want` keys, and by few more: those are
// put together, one to a lane, and searched again.  Where more than 64 reach it (or more are wanted), all keys
// are searched.  KEYS: of a lane, 64 KEYS >= count.
template <int KEYS>
__device__ __forceinline__ void wave_choose(const uint32_t* keys, int count, uint32_t want, int32_t first, int32_t* chosen,
                                            Candidate* few) {
  const int lane = threadIdx.x % 64;
  const uint64_t lower = (1ull << lane) - 1;
  uint32_t key[KEYS], top = 0;
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    key[i] = i * 64 + lane < count ? keys[i * 64 + lane] : 0;
    top = max(top, key[i]);
  }
  uint32_t t = want <= 64 ? wave_kth(top, want) : 0, n = 0;
#pragma unroll
  for (int i = 0; i < KEYS; ++i) n += __popcll(__ballot(key[i] >= t));
  if (t > 0 && n <= 64) {
    uint32_t at = 0;
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
      const uint64_t in = __ballot(key[i] >= t);
      if (key[i] >= t) few[at + __popcll(in & lower)] = {key[i], first + i * 64 + lane};
      at += __popcll(in);
    }
    __threadfence_block();  // the wave's own writes
    const Candidate c = lane < (int)n ? few[lane] : Candidate{0, 0};
    write_largest(c.key, c.block, want, chosen);
    return;
  }
  t = 0;
  for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
    n = 0;
#pragma unroll
    for (int i = 0; i < KEYS; ++i) n += __popcll(__ballot(key[i] >= (t | bit)));
    if (n >= want) t |= bit;
    if (n == want) break;
  }
  uint32_t left = want, at = 0, equal = 0;
#pragma unroll
  for (int i = 0; i < KEYS; ++i) left -= __popcll(__ballot(key[i] > t));
#pragma unroll
  for (int i = 0; i < KEYS; ++i) {
    const bool same = i * 64 + lane < count && key[i] == t;
    const uint64_t sames = __ballot(same);
    const bool taken = key[i] > t || (same && equal + __popcll(sames & lower) < left);
    const uint64_t all = __ballot(taken);
    if (taken) chosen[at + __popcll(all & lower)] = first + i * 64 + lane;
    at += __popcll(all), equal += __popcll(sames);
  }
}

constexpr int kMaxWaves = 16;
constexpr int kUnit = 32;
constexpr int kMaxTile = 32;

struct GroupLds {
  uint32_t top[64];       // of the keys whose number is l modulo 64
  uint32_t counts[16][4];
  uint32_t few_of[kMaxWaves];
  uint2 parts[kMaxWaves];
};

// The same by all waves of a workgroup, each with a run of the keys.  `g` is zero but for few_of.
__device__ __forceinline__ void group_choose(const uint32_t* keys, int count, uint32_t want, int32_t first,
                                             int32_t* chosen, Candidate* few, GroupLds& g) {
  const int threads = blockDim.x, waves = threads / 64, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const uint64_t lower = (1ull << lane) - 1;
  const int run = ((count + threads - 1) / threads) * 64;  // keys of a wave
  const int i0 = min(wave * run, count), i1 = min(i0 + run, count);
  uint32_t top = 0;
  for (int i = i0 + lane; i < i1; i += 64) top = max(top, keys[i]);
  atomicMax(&g.top[lane], top);
  __syncthreads();
  const uint32_t t = want <= 64 ? wave_kth(g.top[lane], want) : 0;
  uint32_t n = 0;
  for (int i = i0; i < i1; i += 64) n += __popcll(__ballot(i + lane < i1 && keys[i + lane] >= t));
  if (lane == 0) g.few_of[wave] = n;
  __syncthreads();
  uint32_t at = 0, total = 0;
  for (int w = 0; w < waves; ++w) {
    at += w < wave ? g.few_of[w] : 0;
    total += g.few_of[w];
  }
  if (t > 0 && total <= 64) {
    for (int i = i0; i < i1; i += 64) {
      const uint32_t k = i + lane < i1 ? keys[i + lane] : 0;
      const uint64_t in = __ballot(k >= t);
      if (k >= t) few[at + __popcll(in & lower)] = {k, first + i + lane};
      at += __popcll(in);
    }
    __syncthreads();
    if (wave > 0) return;
    const Candidate c = lane < (int)total ? few[lane] : Candidate{0, 0};
    write_largest(c.key, c.block, want, chosen);
    return;
  }
  // all keys, two bits a round
  uint32_t s = 0;
  bool exact = false;
  for (int round = 0; round < 16 && !exact; ++round) {
    const int shift = 30 - 2 * round;
    uint32_t m[3] = {0, 0, 0};
    for (int i = i0; i < i1; i += 64) {
      const uint32_t k = i + lane < i1 ? keys[i + lane] : 0;
#pragma unroll
      for (int j = 0; j < 3; ++j) m[j] += __popcll(__ballot(k >= (s | (uint32_t)(j + 1) << shift)));
    }
    if (lane < 3) atomicAdd(&g.counts[round][lane], lane == 0 ? m[0] : lane == 1 ? m[1] : m[2]);
    __syncthreads();
    const uint32_t s0 = s;
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      const uint32_t all = g.counts[round][j];
      if (all >= want) s = s0 | (uint32_t)(j + 1) << shift, exact = all == want;
    }
  }
  uint2 mine = make_uint2(0, 0);  // keys above s, and equal to it
  const int each = (count + threads - 1) / threads;
  const int b0 = min((int)threadIdx.x * each, count), b1 = min(b0 + each, count);
  for (int i = b0; i < b1; ++i) mine.x += keys[i] > s, mine.y += keys[i] == s;
  uint2 all;
  const uint2 prior = before(mine, g.parts, &all);
  const uint32_t left = want - all.x;
  uint32_t equal = prior.y, to = prior.x + min(prior.y, left);
  for (int i = b0; i < b1; ++i)
    if (keys[i] > s || (keys[i] == s && equal++ < left)) chosen[to++] = first + i;
}

// The summaries of UNIT blocks on their way to a wave's part of LDS: rows of PIECES times 16 bytes, whose pieces are
// permuted by the row (piece x at x ^ swap) so that the 16 rows that a wave reads one piece of lie in different banks.
// (Read from the summaries straight into operands, neighbouring lanes have different rows: four times the cache
// lines an access, which took 5 of 16 us for 2048 blocks of 128 values to a token and 10 of 38 us for prompts.)
template <int STEPS, int UNIT>
struct Summaries {
  static constexpr int PIECES = STEPS * 4, ROWS = 64 / PIECES;  // of an access
  static constexpr int kBytes = UNIT * PIECES * 16;
  static __device__ __forceinline__ int swap(int row) { return row * PIECES / 16 & (PIECES - 1); }
  int32_t page;  // of block `lane` of the unit; -1: missing
  float scale;
  // (Bytes past a head's end meet zeros of the queries: any will do.  `wide`: whole 16-byte pieces.)
  __device__ __forceinline__ void fetch(const SelectArgs& a, int h, int32_t entry, bool wide, unsigned char* to) {
    const int lane = threadIdx.x % 64;
    page = entry < a.pages ? entry : -1;
    const int32_t p = max(page, 0);  // (in a missing page's place: page 0)
    const int8_t* from[UNIT / ROWS];
#pragma unroll
    for (int i = 0; i < UNIT / ROWS; ++i)
      from[i] = a.means + ((int64_t)__shfl(p, i * ROWS + lane / PIECES) * a.kv_heads + h) * a.head_dim;
    if (wide) {
#pragma unroll
      for (int i = 0; i < UNIT / ROWS; ++i) {
        const int piece = (lane % PIECES) ^ swap(i * ROWS + lane / PIECES);
        copy_to_lds(from[i] + min(piece * 16, a.head_dim - 16), to + i * 1024);
      }
    } else {
#pragma unroll
      for (int i = 0; i < UNIT / ROWS; ++i) {
        const int piece = (lane % PIECES) ^ swap(i * ROWS + lane / PIECES);
        const int2 lo = *reinterpret_cast<const int2*>(from[i] + min(piece * 16, a.head_dim - 8));
        const int2 hi = *reinterpret_cast<const int2*>(from[i] + min(piece * 16 + 8, a.head_dim - 8));
        *reinterpret_cast<i32x4*>(to + i * 1024 + lane * 16) = i32x4{lo.x, lo.y, hi.x, hi.y};
      }
    }
    scale = a.scales[(int64_t)p * a.kv_heads + h];
  }
  static __device__ __forceinline__ i32x4 piece(const unsigned char* unit, int row, int x) {
    return *reinterpret_cast<const i32x4*>(unit + (row * PIECES + (x ^ swap(row))) * 16);
  }
};

// A query's 8-bit row in LDS: 16 bytes longer, so that the rows of one piece lie in different banks.
constexpr int row_bytes(int steps) { return steps * 64 + 16; }

// Four values of a query.
__device__ __forceinline__ void load_values(const void* q, int64_t at, int dtype, bool aligned, float (&x)[4]) {
  if (dtype == SDNN_F32) {
    load_n<4>(static_cast<const float*>(q) + at, aligned, x);
    return;
  }
  uint16_t v[4];
  load_n<4>(static_cast<const uint16_t*>(q) + at, aligned, v);
#pragma unroll
  for (int k = 0; k < 4; ++k)
    x[k] = dtype == SDNN_F16 ? (float)__builtin_bit_cast(_Float16, v[k]) : __uint_as_float((uint32_t)v[k] << 16);
}

// A workgroup chooses the blocks of one cached head for `tile` tokens.  Scores: the dot products of 16 queries
// (the rows: 2^SHIFT of them to a token, or several tiles of 16, SHIFT = 5) and 16 summaries are one matrix
// instruction for 64 values of a head, bytes in, whole numbers out; a lane's four results are rows 4 g ...
// 4 g + 3 of its own block, so that a group of up to four queries takes its maximum within a lane.  A wave has
// UNIT blocks under way at a time, the first of them before the queries are there.  The scores go to LDS as
// ordered integers.  Then, of one token, all waves search the threshold together; of several, each wave takes
// whole tokens, whose keys stay in its registers.
//   4 tokens of 8 cached heads over 2048 blocks of 128 values: 11 to 12 us (queries 4, scores 4, choice 3): the 256 KiB of a
// workgroup's summaries go through one compute unit.  2048 tokens of 8 heads over 512 blocks: 38 us (queries 11,
// scores 17, choice 10), instructions, half of them of the vector unit, and the waits between them.
template <int STEPS, int SHIFT, int UNIT>
__global__ __launch_bounds__((SHIFT < 4 ? 256 : 1024), 4) void select_kernel(SelectArgs a) {
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ GroupLds group;
  __shared__ int32_t seqs[kMaxTile], seen[kMaxTile];  // of the tile's tokens; blocks that they see
  constexpr int ROW = row_bytes(STEPS);
  const int rows = a.tile * a.per_token;                      // a multiple of 16
  int8_t* m8 = reinterpret_cast<int8_t*>(lds);                // [rows][ROW]
  float* top = reinterpret_cast<float*>(m8 + rows * ROW);     // [rows]: largest value of each query
  float* dead = top + rows;                                   // [rows]: 0, or -infinity where there is no query
  uint32_t* keys = reinterpret_cast<uint32_t*>(lds + a.keys); // [tile][stride]
  Candidate* few = reinterpret_cast<Candidate*>(lds);         // [waves][64], in the queries' place afterwards
  const int threads = blockDim.x, lane = threadIdx.x % 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = threads / 64;
  const int h = blockIdx.x % a.kv_heads, t0 = blockIdx.x / a.kv_heads * a.tile;
  const int D = a.head_dim, r = lane & 15, g = lane >> 4;
  const int forced = a.sink + a.local;
  const uint32_t take = a.blocks - forced;    // of the blocks that are scored
  const bool wide = D % 16 == 0;
  const auto sees = [&](int32_t p, int32_t seq) {
    return p < 0 || (uint32_t)seq >= (uint32_t)a.sequences ? 0 : min((p >> a.block_shift) + 1, a.max_blocks);
  };

  // of the first token's sequence: what every wave needs to begin with its first blocks
  const int32_t first_seq = a.seq[t0];
  const int first_last = min(t0 + a.tile, a.tokens) - 1;  // (positions ascend within a sequence)
  int ahead = max(sees(a.pos[t0], first_seq), a.seq[first_last] == first_seq ? sees(a.pos[first_last], first_seq) : 0);
  ahead = take > 0 && ahead > a.blocks ? ahead - forced : 0;
  typedef Summaries<STEPS, UNIT> Unit;
  Unit sum;
  unsigned char* unit = lds + a.keys + a.tile * a.stride * 4 + wave * Unit::kBytes;
  if (wave * UNIT < ahead) {
    const int b = wave * UNIT + lane;
    sum.fetch(a, h, lane < UNIT && b < ahead ? a.table[(int64_t)first_seq * a.max_blocks + a.sink + b] : -1, wide, unit);
  }

  if (threadIdx.x < 64) group.top[threadIdx.x] = 0, group.counts[threadIdx.x / 4][threadIdx.x % 4] = 0;
  if ((int)threadIdx.x < a.tile) {
    const int t = t0 + threadIdx.x;
    int32_t p = -1, seq = -1;
    if (t < a.tokens) p = a.pos[t], seq = a.seq[t];
    seqs[threadIdx.x] = seq;
    seen[threadIdx.x] = sees(p, seq);
  }
  // queries in 8 bits, four rows of 16 lanes to a wave
  for (int row0 = wave * 4; row0 < rows; row0 += waves * 4) {
    const int row = row0 + g, i = row / a.per_token, gq = row % a.per_token;
    const bool live = gq < a.group && t0 + i < a.tokens;
    const int64_t q = (t0 + i) * a.q_token + (int64_t)(h * a.group + gq) * a.q_head;
    float x[STEPS][4], m = 0.0f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int d = s * 64 + r * 4;
#pragma unroll
      for (int k = 0; k < 4; ++k) x[s][k] = 0.0f;
      if (live && d < D) load_values(a.q, q + d, a.dtype, a.q_aligned, x[s]);
#pragma unroll
      for (int k = 0; k < 4; ++k) m = fmaxf(m, fabsf(x[s][k]));
    }
    m = fmaxf(m, rotated<8>(m));
    m = fmaxf(m, rotated<4>(m));
    m = fmaxf(m, rotated<2>(m));
    m = fmaxf(m, rotated<1>(m));
    const float f = m > 0.0f ? 127.0f * (1.0f / m) : 0.0f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      uint32_t w = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        w |= ((uint32_t)(int)fminf(fmaxf(rintf(x[s][k] * f), -127.0f), 127.0f) & 255u) << (8 * k);
      *reinterpret_cast<uint32_t*>(m8 + row * ROW + s * 64 + r * 4) = w;
    }
    if (r == 0) top[row] = m, dead[row] = live ? 0.0f : -INFINITY;
  }
  __syncthreads();
  // without a choice: everything the token sees; else the blocks that are always taken
  bool some = false;
  for (int i = 0; i < a.tile; ++i) some |= seen[i] > a.blocks && take > 0;
  for (int i = wave; i < a.tile; i += waves) {
    const int n = seen[i];
    if (t0 + i >= a.tokens) break;
    int32_t* chosen = a.chosen + ((int64_t)(t0 + i) * a.kv_heads + h) * a.blocks;
    if (n <= a.blocks) {
      for (int j = lane; j < a.blocks; j += 64) chosen[j] = j < n ? j : -1;
    } else {
      for (int j = lane; j < forced; j += 64) chosen[j < a.sink ? j : a.blocks - forced + j] = j < a.sink ? j : n - forced + j;
    }
  }
  if (!some) return;

  for (int i0 = 0; i0 < a.tile;) {  // tokens i0 ... i1 - 1 are of one sequence
    const int32_t seq = seqs[i0];
    int i1 = i0, most = 0;
    for (; i1 < a.tile && seqs[i1] == seq; ++i1) most = max(most, seen[i1]);
    const int count = most > a.blocks ? most - forced : 0;
    const int32_t* table = a.table + (int64_t)seq * a.max_blocks + a.sink;
    for (int b0 = wave * UNIT; b0 < count; b0 += waves * UNIT) {
      if (!(i0 == 0 && b0 < waves * UNIT && ahead >= count))
        sum.fetch(a, h, lane < UNIT && b0 + lane < count ? table[b0 + lane] : -1, wide, unit);
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // the wave's own copies
      const uint64_t gone = __ballot(sum.page < 0);
      float most_yet[UNIT / 16];  // (SHIFT 5) of block 16 k + r, over the rows so far
      for (int row0 = 0; row0 < rows; row0 += 16) {
        i32x4 qv[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) qv[s] = *reinterpret_cast<const i32x4*>(m8 + (row0 + r) * ROW + s * 64 + g * 16);
        const f32x4 tq = *reinterpret_cast<const f32x4*>(top + row0 + 4 * g);
        const f32x4 none = *reinterpret_cast<const f32x4*>(dead + row0 + 4 * g);
        // A lane's results become, after the maximum over the rows of a token, scores of tokens first, first + 1, ...
        // (of 8 or more rows to a token, lanes of 2 or 4 groups have the same ones, and share the
        // blocks).  Those of blocks past the last one are written too: a token has place for whole 64.
        const int first = SHIFT == 5 ? 0 : (row0 + 4 * g) >> SHIFT;
        uint32_t* key = keys + first * a.stride + b0 + r;
        uint32_t y[UNIT / 16];
#pragma unroll
        for (int k = 0; k < UNIT / 16; ++k) {
          i32x4 dot = {0, 0, 0, 0};
#pragma unroll
          for (int s = 0; s < STEPS; ++s)
            dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(qv[s], Unit::piece(unit, 16 * k + r, 4 * s + g), dot, 0, 0, 0);
          const float scale = __shfl(sum.scale, 16 * k + r);
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = fmaf((float)dot[i], tq[i], none[i]);  // (a product rounded once, or -infinity)
          const auto number = [&](float x) { return gone >> (16 * k + r) & 1 ? 0u : ordered(x * scale); };
          if (SHIFT >= 2) {
            float m = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
            if (SHIFT >= 3) m = max_over_16(m);
            if (SHIFT >= 4) m = max_over_32(m);
            if (SHIFT == 5) m = most_yet[k] = row0 ? fmaxf(most_yet[k], m) : m;
            y[k] = number(m);
          } else {
#pragma unroll
            for (int i = 0; i < 4; i += 1 << SHIFT)
              if (first + (i >> SHIFT) >= i0 && first + (i >> SHIFT) < i1)
                key[(i >> SHIFT) * a.stride + 16 * k] = number(SHIFT ? fmaxf(x[i], x[i + (SHIFT ? 1 : 0)]) : x[i]);
          }
        }
        if (SHIFT < 2 || first < i0 || first >= i1) continue;
        if (SHIFT == 2) {
#pragma unroll
          for (int k = 0; k < UNIT / 16; ++k) key[16 * k] = y[k];
          continue;
        }
        if (SHIFT == 5 && row0 + 16 < rows) continue;
#pragma unroll
        for (int k = 0; k + 1 < UNIT / 16; k += 2) {
          const uint32_t even = y[k], odd = y[k + 1];
          if (SHIFT == 3 || g >> 1 == k / 2) key[16 * (k + (g & 1))] = g & 1 ? odd : even;
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // everything read: the unit's place is free
    }
    i0 = i1;
  }
  __syncthreads();

  if (SHIFT >= 4 && a.tile == 1) {
    group_choose(keys, seen[0] - forced, take, a.sink,
                 a.chosen + ((int64_t)t0 * a.kv_heads + h) * a.blocks + a.sink, few, group);
    return;
  }
  for (int i = wave; i < a.tile; i += waves) {
    if (seen[i] <= a.blocks) continue;
    const int count = seen[i] - forced;
    int32_t* chosen = a.chosen + ((int64_t)(t0 + i) * a.kv_heads + h) * a.blocks + a.sink;
    const uint32_t* key = keys + i * a.stride;
    if (count <= 256)
      wave_choose<4>(key, count, take, a.sink, chosen, few + 64 * wave);
    else if (count <= 512)
      wave_choose<8>(key, count, take, a.sink, chosen, few + 64 * wave);
    else
      wave_choose<kWaveKeys>(key, count, take, a.sink, chosen, few + 64 * wave);
  }
}

template <int STEPS, int SHIFT>
hipError_t start(SelectArgs a, int threads, hipStream_t stream) {
  constexpr int UNIT = kUnit;
  const auto kernel = select_kernel<STEPS, SHIFT, UNIT>;
  a.keys = a.tile * a.per_token * (row_bytes(STEPS) + 8);
  const int few = (a.tile == 1 ? 1 : threads / 64) * 64 * (int)sizeof(Candidate);
  if (a.keys < few) a.keys = few;
  size_t lds = a.keys + (size_t)a.tile * a.stride * sizeof(uint32_t);
  while (threads > 64 && lds + threads / 64 * Summaries<STEPS, UNIT>::kBytes > 156 * 1024) threads /= 2;
  lds += threads / 64 * Summaries<STEPS, UNIT>::kBytes;
  if (lds > 60000) {  // with the kernel's own arrays past what a launch gives by default
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const unsigned grid = (unsigned)((a.tokens + a.tile - 1) / a.tile) * a.kv_heads;
  kernel<<<grid, threads, lds, stream>>>(a);
  return hipGetLastError();
}

template <int STEPS>
hipError_t start_rows(const SelectArgs& a, int threads, hipStream_t stream) {
  switch (a.per_token) {
    case 1: return start<STEPS, 0>(a, threads, stream);
    case 2: return start<STEPS, 1>(a, threads, stream);
    case 4: return start<STEPS, 2>(a, threads, stream);
    case 8: return start<STEPS, 3>(a, threads, stream);
    case 16: return start<STEPS, 4>(a, threads, stream);
    default: return start<STEPS, 5>(a, threads, stream);
  }
}

}  // namespace

hipError_t launch_select(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q,
                         int32_t blocks, int32_t sink, int32_t local, int32_t* chosen, hipStream_t stream) {
  SelectArgs a = {};
  a.q = q.data, a.q_token = q.token_stride, a.q_head = q.head_stride;
  a.means = c.means, a.scales = c.mean_scales, a.pages = c.pages;
  a.pos = t.pos, a.seq = t.seq, a.table = t.table, a.chosen = chosen;
  a.tokens = t.tokens, a.sequences = t.sequences, a.max_blocks = t.max_blocks;
  a.kv_heads = c.kv_heads, a.group = q.heads / c.kv_heads, a.head_dim = c.head_dim;
  a.block_shift = __builtin_ctz(c.block);
  a.blocks = blocks, a.sink = sink, a.local = local;
  const SelectShape shape = select_shape(c, t, q.heads);
  if (!launchable(shape.groups, shape.threads)) return hipErrorInvalidConfiguration;
  a.tile = shape.tile, a.per_token = shape.per_token;
  a.q_aligned = (uintptr_t)q.data % (4 * dtype_bytes(c.dtype)) == 0 && q.token_stride % 4 == 0 && q.head_stride % 4 == 0;
  a.stride = (t.max_blocks + 63) & ~63;
  a.dtype = c.dtype;
  if (a.head_dim <= 64) return start_rows<1>(a, shape.threads, stream);
  if (a.head_dim <= 128) return start_rows<2>(a, shape.threads, stream);
  return start_rows<4>(a, shape.threads, stream);
}

}  // namespace sdnn
