// The choice of blocks by the score of their summaries.
#include "sdnn_decode_device.h"

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
  int32_t tile, per_token;  // tokens of a workgroup, rows of a token (tile > 1: 1, 2, 4 or 8)
};

// A number whose order as an unsigned integer is the order of the floats (-0 counts as 0).
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.0f);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

// 16 bytes of a summary from byte k on, zeros past its end (D is a multiple of 8).
__device__ __forceinline__ i32x4 load_mean(const int8_t* row, int k, int D, bool wide) {
  i32x4 v = {0, 0, 0, 0};
  if (wide) {
    if (k < D) v = *reinterpret_cast<const i32x4*>(row + k);
  } else {
    if (k < D) {
      const int2 lo = *reinterpret_cast<const int2*>(row + k);
      v[0] = lo.x, v[1] = lo.y;
    }
    if (k + 8 < D) {
      const int2 hi = *reinterpret_cast<const int2*>(row + k + 8);
      v[2] = hi.x, v[3] = hi.y;
    }
  }
  return v;
}

// Sums of two counts over the workgroup's threads before this one.  `parts`: a word for each wave.
__device__ __forceinline__ uint2 before(uint2 n, uint2* parts) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint2 s = n;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t x = __shfl_up(s.x, d), y = __shfl_up(s.y, d);
    if (lane >= d) s.x += x, s.y += y;
  }
  __syncthreads();
  if (lane == 63) parts[wave] = s;
  __syncthreads();
  uint2 r = make_uint2(s.x - n.x, s.y - n.y);
  for (int w = 0; w < wave; ++w) r.x += parts[w].x, r.y += parts[w].y;
  return r;
}

constexpr int kMaxWaves = 16;
constexpr int kWaveKeys = 16;  // keys of a lane where a wave selects alone: up to 1024 blocks

// What is taken: all keys above `above`, and of those equal to it the first `equal`.
struct Threshold {
  uint32_t above, equal;
};

// The `want` largest of a wave's keys (want >= 1, fewer than count), bit by bit from the top: `t` is the
// largest prefix with at least `want` keys at or over it.  Most searches end early, at a prefix that exactly
// `want` reach.
__device__ __forceinline__ Threshold wave_threshold(const uint32_t (&key)[kWaveKeys], int count, uint32_t want) {
  uint32_t t = 0;
  for (uint32_t bit = 1u << 31; bit; bit >>= 1) {
    const uint32_t c = t | bit;
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < kWaveKeys; ++i)
      if (i * 64 < count) n += __popcll(__ballot(key[i] >= c));  // (past the end a key is 0, and c is not)
    if (n == want) return {c - 1, 0};
    if (n > want) t = c;
  }
  uint32_t more = 0;
#pragma unroll
  for (int i = 0; i < kWaveKeys; ++i)
    if (i * 64 < count) more += __popcll(__ballot(key[i] > t));
  return {t, want - more};
}

// The same over the keys of a workgroup in LDS, two bits at a time.  counts: [17][4], zero.
__device__ __forceinline__ Threshold group_threshold(const uint32_t* key, int count, uint32_t want, uint32_t (*counts)[4]) {
  const int threads = blockDim.x, lane = threadIdx.x % 64;
  const int first = threadIdx.x - lane;
  uint32_t t = 0;
  for (int round = 0; round < 16; ++round) {
    const int shift = 30 - 2 * round;
    uint32_t n[3] = {0, 0, 0};
    for (int i = first; i < count; i += threads) {
      const uint32_t k = i + lane < count ? key[i + lane] : 0;
#pragma unroll
      for (int j = 0; j < 3; ++j) n[j] += __popcll(__ballot(k >= (t | (uint32_t)(j + 1) << shift)));
    }
    if (lane < 3 && n[0]) atomicAdd(&counts[round][lane], lane == 0 ? n[0] : lane == 1 ? n[1] : n[2]);
    __syncthreads();
    uint32_t next = t;
#pragma unroll
    for (int j = 0; j < 3; ++j) {
      const uint32_t c = t | (uint32_t)(j + 1) << shift, m = counts[round][j];
      if (m == want) return {c - 1, 0};
      if (m > want) next = c;
    }
    t = next;
  }
  uint32_t more = 0;
  for (int i = first; i < count; i += threads)
    more += __popcll(__ballot((i + lane < count ? key[i + lane] : 0) > t));
  if (lane == 0 && more) atomicAdd(&counts[16][0], more);
  __syncthreads();
  return {t, want - counts[16][0]};
}

// A workgroup chooses the blocks of one cached head for `tile` tokens.  Scores: the dot products of 16 queries
// (the rows: a power of two of them to a token) and 16 summaries are one matrix instruction for 64 values of
// a head, bytes in, whole numbers out; a lane's four results are rows 4 g ... 4 g + 3 of its own block, so that
// a group of up to four queries takes its maximum within a lane.  A wave has 64 blocks under way at a time.
// The scores go to LDS as ordered integers.  Then, of one token, all waves search the threshold together; of
// several, each wave takes whole tokens, whose keys stay in its registers.
template <typename T, int STEPS>
__global__ __launch_bounds__(1024) void select_kernel(SelectArgs a) {
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ uint32_t counts[17][4];
  __shared__ uint2 parts[kMaxWaves];
  __shared__ int32_t seqs[16], seen[16];      // of the tile's tokens; blocks that they see
  constexpr int ROW = STEPS * 64;
  const int rows = a.tile * a.per_token;      // a multiple of 16
  int8_t* m8 = reinterpret_cast<int8_t*>(lds);                // [rows][ROW]
  float* top = reinterpret_cast<float*>(m8 + rows * ROW);     // [rows]; -1: no query
  uint32_t* keys = reinterpret_cast<uint32_t*>(top + rows);   // [tile][max_blocks]
  const int threads = blockDim.x, lane = threadIdx.x % 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = threads / 64;
  const int h = blockIdx.x % a.kv_heads, t0 = blockIdx.x / a.kv_heads * a.tile;
  const int D = a.head_dim, r = lane & 15, g = lane >> 4;
  const int forced = a.sink + a.local;
  const uint32_t take = a.blocks - forced;    // of the blocks that are scored

  if (threadIdx.x < 17 * 4) counts[threadIdx.x / 4][threadIdx.x % 4] = 0;
  if ((int)threadIdx.x < a.tile) {
    const int t = t0 + threadIdx.x;
    int32_t p = -1, seq = -1;
    if (t < a.tokens) p = a.pos[t], seq = a.seq[t];
    seqs[threadIdx.x] = seq;
    seen[threadIdx.x] =
        p < 0 || (uint32_t)seq >= (uint32_t)a.sequences ? 0 : min((p >> a.block_shift) + 1, a.max_blocks);
  }
  __syncthreads();
  // without a choice: everything the token sees; else the blocks that are always taken
  bool some = false;
  for (int i = 0; i < a.tile; ++i) {
    const int n = seen[i];
    some |= n > a.blocks && take > 0;
    if (t0 + i >= a.tokens) continue;
    int32_t* chosen = a.chosen + ((int64_t)(t0 + i) * a.kv_heads + h) * a.blocks;
    if (n <= a.blocks) {
      for (int j = threadIdx.x; j < a.blocks; j += threads) chosen[j] = j < n ? j : -1;
    } else {
      for (int j = threadIdx.x; j < a.sink; j += threads) chosen[j] = j;
      for (int j = threadIdx.x; j < a.local; j += threads) chosen[a.blocks - a.local + j] = n - a.local + j;
    }
  }
  if (!some) return;

  for (int row = wave; row < rows; row += waves) {
    const int i = row / a.per_token, gq = row % a.per_token;
    const bool live = gq < a.group && t0 + i < a.tokens;
    const T* q = static_cast<const T*>(a.q) + (t0 + i) * a.q_token + (int64_t)(h * a.group + gq) * a.q_head;
    float x[STEPS], m = 0.0f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int d = s * 64 + lane;
      x[s] = live && d < D ? (float)q[d] : 0.0f;
      m = fmaxf(m, fabsf(x[s]));
    }
#pragma unroll
    for (int s = 32; s; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
    const float f = m > 0.0f ? 127.0f * (1.0f / m) : 0.0f;
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
      m8[row * ROW + s * 64 + lane] = (int8_t)fminf(fmaxf(rintf(x[s] * f), -127.0f), 127.0f);
    if (lane == 0) top[row] = live ? m : -1.0f;
  }
  __syncthreads();

  const bool wide = D % 16 == 0;
  for (int i0 = 0; i0 < a.tile;) {  // tokens i0 ... i1 - 1 are of one sequence
    const int32_t seq = seqs[i0];
    int i1 = i0, most = 0;
    for (; i1 < a.tile && seqs[i1] == seq; ++i1) most = max(most, seen[i1]);
    const int count = most > a.blocks ? most - forced : 0;
    const int32_t* table = a.table + (int64_t)seq * a.max_blocks + a.sink;
    for (int b0 = wave * 64; b0 < count; b0 += waves * 64) {
      const int32_t entry = b0 + lane < count ? table[b0 + lane] : -1;
      const int32_t mine = entry < a.pages ? entry : -1;
      i32x4 m[4][STEPS];
      float scale[4];
      int32_t page[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        page[k] = __shfl(mine, k * 16 + r);
        const int64_t row = (int64_t)max(page[k], 0) * a.kv_heads + h;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) m[k][s] = load_mean(a.means + row * D, s * 64 + g * 16, D, wide);
        scale[k] = a.scales[row];
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (b0 + k * 16 >= count) break;
        const int b = b0 + k * 16 + r;
        float best[4];
        for (int row0 = 0; row0 < rows; row0 += 16) {
          i32x4 dot = {0, 0, 0, 0};
#pragma unroll
          for (int s = 0; s < STEPS; ++s) {
            const i32x4 qv = *reinterpret_cast<const i32x4*>(m8 + (row0 + r) * ROW + s * 64 + g * 16);
            dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(qv, m[k][s], dot, 0, 0, 0);
          }
          const f32x4 tq = *reinterpret_cast<const f32x4*>(top + row0 + 4 * g);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = tq[i] < 0.0f ? -INFINITY : (float)dot[i] * tq[i];
            best[i] = row0 == 0 ? x : fmaxf(best[i], x);
          }
        }
        // over the queries of a token
        int each = 1;  // of the four: a token's rows are `each` of them, or all four in several lane groups
        if (a.per_token >= 2) best[0] = fmaxf(best[0], best[1]), best[2] = fmaxf(best[2], best[3]), each = 2;
        if (a.per_token >= 4) best[0] = fmaxf(best[0], best[2]), each = 4;
        if (a.per_token >= 8) best[0] = fmaxf(best[0], __shfl_xor(best[0], 16));
        if (a.per_token >= 16) best[0] = fmaxf(best[0], __shfl_xor(best[0], 32));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int token = (4 * g + i) / a.per_token;
          if (i % each == 0 && (4 * g + i) % a.per_token == 0 && token >= i0 && token < i1 && b < count)
            keys[token * a.max_blocks + b] = page[k] < 0 ? 0u : ordered(best[i] * scale[k]);
        }
      }
    }
    i0 = i1;
  }
  __syncthreads();

  if (a.tile == 1) {
    const int count = seen[0] - forced;
    const Threshold th = group_threshold(keys, count, take, counts);
    const int run = (count + threads - 1) / threads;  // blocks of a thread, in order
    const int b0 = min((int)threadIdx.x * run, count), b1 = min(b0 + run, count);
    uint2 n = make_uint2(0, 0);
    for (int b = b0; b < b1; ++b) n.x += keys[b] > th.above, n.y += keys[b] == th.above;
    const uint2 prior = before(n, parts);
    uint32_t equal = prior.y, at = a.sink + prior.x + min(prior.y, th.equal);
    int32_t* chosen = a.chosen + ((int64_t)t0 * a.kv_heads + h) * a.blocks;
    for (int b = b0; b < b1; ++b) {
      const uint32_t k = keys[b];
      if (k > th.above || (k == th.above && equal++ < th.equal)) chosen[at++] = a.sink + b;
    }
    return;
  }
  for (int i = wave; i < a.tile; i += waves) {
    const int count = seen[i] - forced;
    if (seen[i] <= a.blocks) continue;
    uint32_t key[kWaveKeys];
#pragma unroll
    for (int k = 0; k < kWaveKeys; ++k)
      key[k] = k * 64 + lane < count ? keys[i * a.max_blocks + k * 64 + lane] : 0;
    const Threshold th = wave_threshold(key, count, take);
    int32_t* chosen = a.chosen + ((int64_t)(t0 + i) * a.kv_heads + h) * a.blocks + a.sink;
    const uint64_t lower = (1ull << lane) - 1;
    uint32_t at = 0, equal = 0;
#pragma unroll
    for (int k = 0; k < kWaveKeys; ++k) {
      if (k * 64 >= count) break;
      const bool in = k * 64 + lane < count;
      const bool same = in && key[k] == th.above;
      const uint64_t sames = __ballot(same);
      const bool taken = (in && key[k] > th.above) || (same && equal + __popcll(sames & lower) < th.equal);
      const uint64_t takens = __ballot(taken);
      if (taken) chosen[at + __popcll(takens & lower)] = a.sink + k * 64 + lane;
      at += __popcll(takens), equal += __popcll(sames);
    }
  }
}

template <typename T, int STEPS>
hipError_t start(const SelectArgs& a, int threads, hipStream_t stream) {
  const size_t lds = (size_t)a.tile * (a.per_token * (STEPS * 64 + 4) + (size_t)a.max_blocks * 4);
  if (lds > 60000) {  // with the kernel's own arrays past what a launch gives by default
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(select_kernel<T, STEPS>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  const unsigned grid = (unsigned)((a.tokens + a.tile - 1) / a.tile) * a.kv_heads;
  select_kernel<T, STEPS><<<grid, threads, lds, stream>>>(a);
  return hipGetLastError();
}

template <typename T>
hipError_t start_steps(const SelectArgs& a, int threads, hipStream_t stream) {
  if (a.head_dim <= 64) return start<T, 1>(a, threads, stream);
  if (a.head_dim <= 128) return start<T, 2>(a, threads, stream);
  return start<T, 4>(a, threads, stream);
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
  // Tiles of 16 rows hold several tokens where most of a tile's are of one sequence and a wave can select
  // alone; otherwise a workgroup has one token, and so many waves that each has some blocks.
  int rows = 1;
  while (rows < a.group && rows < 16) rows *= 2;
  const bool tiles = rows < 16 && t.tokens >= (int64_t)16 * t.sequences && t.max_blocks <= 64 * kWaveKeys &&
                     (int64_t)(t.tokens / (16 / rows)) * c.kv_heads >= 512;
  a.tile = tiles ? 16 / rows : 1;
  a.per_token = tiles ? rows : (a.group + 15) & ~15;
  int threads = 64;
  while (threads < 1024 && threads < t.max_blocks) threads *= 2;
  if (tiles) threads = 256;
  if (c.dtype == SDNN_F32) return start_steps<float>(a, threads, stream);
  if (c.dtype == SDNN_F16) return start_steps<_Float16>(a, threads, stream);
  return start_steps<__bf16>(a, threads, stream);
}

}  // namespace sdnn
