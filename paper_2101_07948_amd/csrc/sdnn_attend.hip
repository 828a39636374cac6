// Attention over the chosen blocks of the cache.
#include "sdnn_attend_device.h"

namespace sdnn {
namespace {

// A workgroup handles one token, cached head, tile of up to 16 of its queries and share of its
// blocks; its waves take blocks in turn and join their states through LDS.  Reading keys and values
// bounds it: each page is read once for the tile of queries that shares it.  32 tokens of 12 heads of 64 in 32 bits
// over up to 2048 tokens each: 55 us, 244 MB at 4.4 TB/s.  One token of 8 cached heads over 64 blocks of 64 tokens:
// 8 to 9 us for 17 MB, latency: list, page, keys and values, then two joins.
template <typename T, int CHUNKS>
__global__ __launch_bounds__(kWaves * 64, attend_waves(CHUNKS * Step<T>::kPiece / 4)) void attend_kernel(AttendArgs a) {
  constexpr int PIECE = Step<T>::kPiece;
  constexpr int TILES = CHUNKS * PIECE / 4;  // of 16 values of a head
  __shared__ JoinLds<TILES> lds;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane & 15, g = lane >> 4;
  int b = blockIdx.x;
  const int h = b % a.kv_heads;
  b /= a.kv_heads;
  const int split = b % a.splits;
  b /= a.splits;
  const int first = b % a.head_tiles * kRows;  // query of the group
  const int t = b / a.head_tiles;
  const int rows = min(kRows, a.group - first);
  const int64_t head = (int64_t)h * a.group + first + r;  // of this lane
  const int D = a.head_dim;
  const int32_t p = a.pos[t], seq = a.seq[t];
  const bool filler = p < 0 || (uint32_t)seq >= (uint32_t)a.sequences;
  const int own = p / a.block;
  const int n = filler ? 0 : a.chosen ? a.blocks : max(min(own + 1, a.max_blocks) - a.first, 0);
  const int32_t* chosen = a.chosen ? a.chosen + ((int64_t)t * a.kv_heads + h) * a.blocks : nullptr;
  const int32_t* table = a.table + (int64_t)seq * a.max_blocks;
  // Steps of all blocks, dealt to the waves of all shares in turn.  A lane looks up the block and the page of one of the
  // wave's next 64 steps, and those that hold something are taken one after the other.
  constexpr int N = Step<T>::kTokens;
  const int shift = __builtin_ctz(a.block / N), deal = a.splits * kWaves, last = n << shift;
  typename Step<T>::Piece q[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int d = (c * 4 + g) * PIECE;
    T x[PIECE] = {};
    if (r < rows && d < D)
      load_n<PIECE>(static_cast<const T*>(a.q) + t * a.q_token + head * a.q_head + d, a.q_aligned, x);
    __builtin_memcpy(&q[c], x, sizeof(x));
    if (a.negate) q[c] = -q[c];
  }
  State<TILES> st;
#pragma unroll
  for (int c = 0; c < TILES; ++c) st.o[c] = f32x4{0, 0, 0, 0};
  st.m = -INFINITY, st.l = 0.0f;
  for (int first_step = split * kWaves + wave; first_step < last; first_step += 64 * deal) {
    const int mine = first_step + lane * deal;
    int id = -1, page_mine = -1;
    if (lane < (last - first_step + deal - 1) / deal) id = chosen ? chosen[mine >> shift] : a.first + (mine >> shift);
    const auto seen_of = [&](int id, int t0) { return min(p - id * a.block - t0, a.block) + 1; };  // (p up to 2^31 - 1)
    const auto token_of = [&](int u) { return (u & ((1 << shift) - 1)) * N; };
    if (id >= 0 && id <= own && id < a.max_blocks && seen_of(id, token_of(mine)) > 0) page_mine = table[id];
    uint64_t todo = __ballot(page_mine >= 0 && page_mine < a.pages);
    for (; todo; todo &= todo - 1) {
      const int j = __builtin_ctzll(todo);
      const int page = __builtin_amdgcn_readlane(page_mine, j), t0 = token_of(first_step + j * deal);
      const int seen = seen_of(__builtin_amdgcn_readlane(id, j), t0);
      const int64_t at = ((int64_t)page * a.kv_heads + h) * a.block * D;
      const T* v = static_cast<const T*>(a.v_pages) + at + t0;
      // all keys and values are asked for before the first product (left to itself the compiler takes them one by one,
      // to save registers)
      typename Step<T>::Piece kk[TILES], vv[TILES];
      Step<T>::template load_keys<CHUNKS>(static_cast<const T*>(a.k_pages) + at + t0 * D, D, r, g, kk);
      // (the keys and values of a long head are more than the registers of two waves hold beside each other)
      if (TILES <= 8) Step<T>::template load_values<CHUNKS>(v, D, a.block, r, g, vv);
      __builtin_amdgcn_sched_barrier(0);
      float s[N / 4];
      Step<T>::template scores<CHUNKS>([&](int i) { return kk[i]; }, q, s);
      if (TILES > 8) {
        __builtin_amdgcn_sched_barrier(0);
        Step<T>::template load_values<CHUNKS>(v, D, a.block, r, g, vv);
        __builtin_amdgcn_sched_barrier(0);
      }
      attend_step<false, T, CHUNKS, TILES>(a.scale2, s, [&](int i) { return vv[i]; }, seen, seen, g, st);
    }
  }

  join_waves<T>(a, lds, split, t, head, r < rows, st);
}

// ---------------------------------------------------------------- many tokens of a sequence

// Attention of many tokens of a sequence.  A wave has a tile of 16 queries, 16 / group neighbouring tokens of one
// cached head; the WAVES waves of a workgroup, neighbouring tokens again, walk the union of their lists, block
// by block in ascending order, through LDS: a block is read from L2 once for all of them, the next one while
// they compute.  Waves whose tokens did not choose a block skip it; rows of a tile that did not are masked.
// The union is found on the way, a block ahead: each token offers its lowest block not yet passed.
//   2048 tokens of 32 queries on 8 cached heads of 128 in 16 bits, 16 blocks of 64 each: 148 us, 34 GFLOP at 232 TFLOP/s
// (the matrix unit does 2.6 times that: rows of tokens that did not choose a block, and probabilities in two
// parts).  Vector instructions (masks, exponentials, the parts) take 40 % of the time, matrix ones 25 %, and waves
// wait for a stage or the matrix unit in 58 % of theirs.  Half as many waves to a SIMD, for more registers: 212 us;
// 4 waves to a workgroup: 226; stages of 32 tokens: 174.
template <typename T, int CHUNKS, int STAGE, int WAVES>
__global__ __launch_bounds__(WAVES * 64, CHUNKS * sizeof(T) <= 8 ? 4 : 2) void attend_tiles(AttendArgs a) {
  typedef Tile<T, CHUNKS, STAGE> L;
  constexpr int TILES = CHUNKS * L::kPiece / 4, N = Step<T>::kTokens;
  constexpr int32_t END = 0x7fffffff;
  __shared__ __align__(16) unsigned char lds[2][2 * L::kBytes];
  __shared__ uint64_t turns[2];
  __shared__ uint64_t lowest[3];  // key and page of the lowest block that is offered, in turn
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane & 15, g = lane >> 4;
  int b = blockIdx.x;
  const int h = b % a.kv_heads;
  b /= a.kv_heads;
  const int split = b % a.splits;
  b /= a.splits;
  const int first = b % a.head_tiles * kRows;
  const int t0 = b / a.head_tiles * (a.tile_tokens * WAVES);
  const int rows = min(kRows, a.group - first);     // queries of a token
  const int per_token = kRows / a.tile_tokens;      // rows of the tile for a token (a power of two)
  const int t = t0 + wave * a.tile_tokens + r / per_token, qr = r % per_token;
  const bool row = t < a.tokens && qr < rows;
  const int head = h * a.group + first + qr;
  const int D = a.head_dim;
  typename Step<T>::Piece q[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int d = (c * 4 + g) * L::kPiece;
    T x[L::kPiece] = {};
    if (row && d < D)
      load_n<L::kPiece>(static_cast<const T*>(a.q) + t * a.q_token + head * a.q_head + d, a.q_aligned, x);
    __builtin_memcpy(&q[c], x, sizeof(x));
    if (a.negate) q[c] = -q[c];
  }
  State<TILES> st;
#pragma unroll
  for (int c = 0; c < TILES; ++c) st.o[c] = f32x4{0, 0, 0, 0};
  st.m = -INFINITY, st.l = 0.0f;

  // A block's key: the run of tokens of one sequence within the workgroup's, then the block, counted from the launch's first, as
  // positions are from here on (tiles_of bounds the blocks from there on by the key's 20 bits: a prefix may have as many before).
  // Bit i of `turns`: token i is of another sequence than token i - 1 (a workgroup has at most 16 WAVES).
  static_assert(16 * WAVES <= 128, "two words of bits");
  if (wave < 2) {
    const int i = wave * 64 + lane, ti = t0 + i;
    const bool turn = i > 0 && i < a.tile_tokens * WAVES && ti < a.tokens && a.seq[ti] != a.seq[ti - 1];
    const uint64_t bits = __ballot(turn);
    if (lane == 0) turns[wave] = bits;
  }
  if (threadIdx.x < 3) lowest[threadIdx.x] = ~0ull;
  int32_t p = -1, seq = -1;
  if (t < a.tokens) p = a.pos[t], seq = a.seq[t];
  __syncthreads();
  const int place = t - t0;
  const int32_t run = __popcll(turns[0] & (place >= 63 ? ~0ull : (2ull << place) - 1)) +
                      (place < 64 ? 0 : __popcll(turns[1] & (place == 127 ? ~0ull : (2ull << (place - 64)) - 1)));
  const bool filler = p < 0 || (uint32_t)seq >= (uint32_t)a.sequences;
  Cursor at;
  at.t = t, at.seq = seq, at.last = min(p / a.block, a.max_blocks - 1) - a.first, at.share = split;
  at.n = filler ? 0 : a.chosen ? a.blocks : at.last + 1;
  p -= filler ? 0 : a.first * a.block;
  at.start(a, h);
  const auto key = [&] { return at.valid(at.id) ? run << 20 | at.id : END; };
  // One row of each token offers its next block.
  const auto offer = [&](int turn) {
    if (g == 0 && qr == 0)
      atomicMin(reinterpret_cast<unsigned long long*>(&lowest[turn]),
                (unsigned long long)(uint32_t)key() << 32 | (uint32_t)at.page);
  };
  // The lowest block of those offered; what this lane's query sees of it is left in `seen`, and it is passed.  The
  // offers before it, which all waves have read, make room for the next but one.
  int32_t block_key = END, block_page = -1, seen = 0;
  const auto take = [&](int turn) {
    const uint64_t low = lowest[turn];
    if (threadIdx.x == 0) lowest[turn == 0 ? 2 : turn - 1] = ~0ull;
    block_key = __builtin_amdgcn_readfirstlane((int32_t)(low >> 32));
    block_page = __builtin_amdgcn_readfirstlane((int32_t)low);
    if (block_page >= a.pages) block_page = -1;
    const bool mine = block_key != END && key() == block_key;
    seen = mine && block_page >= 0 ? min(a.block - 1, p - at.id * a.block) + 1 : 0;
    if (mine) at.advance(a, h);
  };
  const int stage = min(STAGE, a.block), stages = a.block / stage;
  const auto fetch = [&](int s, int buffer) {
    if (block_page < 0) return;
    const int64_t from = ((int64_t)block_page * a.kv_heads + h) * a.block * D;
    L::template fetch<WAVES * 64>(static_cast<const T*>(a.k_pages) + from + (int64_t)s * stage * D,
                                  static_cast<const T*>(a.v_pages) + from + s * stage, stage, D, a.block, lds[buffer]);
  };

  int turn = 0, buffer = 0, s = 0;
  const auto next = [&] { return turn == 2 ? 0 : turn + 1; };
  offer(turn);
  __syncthreads();
  take(turn);
  offer(turn = next());
  if (block_key != END) fetch(0, 0);
  while (block_key != END) {
    const int32_t now_seen = seen - s * stage;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // the stage is in LDS, the other buffer is free, the offers are made
    if (++s == stages) {
      s = 0;
      take(turn);
      if (block_key != END) offer(turn = next());
    }
    if (block_key != END) fetch(s, buffer ^ 1);
    const auto scores = [&](int u, float (&x)[N / 4]) {
      Step<T>::template scores<CHUNKS>([&](int i) { return key_piece<T, CHUNKS, STAGE>(lds[buffer], i, u, D, r, g); }, q, x);
    };
    const auto step = [&](int u, float (&x)[N / 4], int stored) {
      attend_step<true, T, CHUNKS, TILES>(
          a.scale2, x, [&](int i) { return value_piece<T, CHUNKS, STAGE>(lds[buffer], i, u, r, g); }, now_seen - u, stored,
          g, st);
    };
    int u = 0;
    // two steps that some query sees all of: the second one's scores are under way while the first is taken in
    for (; u + 2 * N <= stage && __any(now_seen >= u + 2 * N); u += 2 * N) {
      float x[N / 4], y[N / 4];
      scores(u, x);
      scores(u + N, y);
      step(u, x, N);
      step(u + N, y, N);
    }
    for (; u < stage && __any(now_seen > u); u += N) {
      // of the tokens past every query's sight the values are taken for zeros
      int stored = N;
      if (!__any(now_seen >= u + N)) {
        stored = max(now_seen - u, 0);
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) stored = max(stored, __shfl_xor(stored, x));
      }
      float x[N / 4];
      scores(u, x);
      step(u, x, stored);
    }
    buffer ^= 1;
  }

  float l = over_groups_sum(st.l);
  if (!row) return;
  if (at.n <= 0) l = no_sums(st);
  if (a.parts > 1)
    store_part(a, split, t, head, g, st, l);
  else
    store_row<T>(a, t, head, g, st, st.m, l);
}

// Of all tokens' shared first blocks (AttendArgs::prefix): as attend_tiles, but all of a workgroup's waves go through the same
// blocks, which need no offers: 64 tokens of 32 queries on 8 heads of 128 over 16384, 39.5 us, 17 GFLOP at 435 TFLOP/s, and 42.5
// with offers; 8 tokens over 32768, a call, 48 and 52.
template <typename T, int CHUNKS, int STAGE>
__global__ __launch_bounds__(kTileWaves * 64, CHUNKS * sizeof(T) <= 8 ? 4 : 2) void prefix_tiles(AttendArgs a) {
  typedef Tile<T, CHUNKS, STAGE> L;
  constexpr int TILES = CHUNKS * L::kPiece / 4, N = Step<T>::kTokens;
  __shared__ __align__(16) unsigned char lds[2][2 * L::kBytes];
  __shared__ typename Walk<false, 1>::Lds walked;
  const TileRows<1> t(a);
  const int r = t.r, g = t.g, D = a.head_dim;
  typename Step<T>::Piece q[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int d = (c * 4 + g) * L::kPiece;
    T x[L::kPiece] = {};
    if (t.row(0) && d < D)
      load_n<L::kPiece>(static_cast<const T*>(a.q) + t.token(0) * a.q_token + t.head * a.q_head + d, a.q_aligned, x);
    __builtin_memcpy(&q[c], x, sizeof(x));
    if (a.negate) q[c] = -q[c];
  }
  State<TILES> st;
#pragma unroll
  for (int c = 0; c < TILES; ++c) st.o[c] = f32x4{0, 0, 0, 0};
  st.m = -INFINITY, st.l = 0.0f;
  Walk<false, 1> walk;
  walk.template start<true>(a, t, walked);
  const int stage = min(STAGE, a.block), stages = a.block / stage;
  const auto fetch = [&](int s, int buffer) {
    if (walk.page < 0) return;
    const int64_t from = ((int64_t)walk.page * a.kv_heads + t.h) * a.block * D;
    L::template fetch<kTileWaves * 64>(static_cast<const T*>(a.k_pages) + from + (int64_t)s * stage * D,
                                       static_cast<const T*>(a.v_pages) + from + s * stage, stage, D, a.block, lds[buffer]);
  };
  int buffer = 0, s = 0;
  if (walk.key != walk.END) fetch(0, 0);
  while (walk.key != walk.END) {
    const int32_t now_seen = walk.seen[0] - s * stage;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // the stage is in LDS, the other buffer is free
    if (++s == stages) s = 0, walk.advance(a, t, walked);
    if (walk.key != walk.END) fetch(s, buffer ^ 1);
    const auto scores = [&](int u, float (&x)[N / 4]) {
      Step<T>::template scores<CHUNKS>([&](int i) { return key_piece<T, CHUNKS, STAGE>(lds[buffer], i, u, D, r, g); }, q, x);
    };
    const auto step = [&](int u, float (&x)[N / 4], int stored) {
      attend_step<true, T, CHUNKS, TILES>(
          a.scale2, x, [&](int i) { return value_piece<T, CHUNKS, STAGE>(lds[buffer], i, u, r, g); }, now_seen - u, stored,
          g, st);
    };
    int u = 0;
    for (; u + 2 * N <= stage && __any(now_seen >= u + 2 * N); u += 2 * N) {
      float x[N / 4], y[N / 4];
      scores(u, x);
      scores(u + N, y);
      step(u, x, N);
      step(u + N, y, N);
    }
    for (; u < stage && __any(now_seen > u); u += N) {
      int stored = N;
      if (!__any(now_seen >= u + N)) {
        stored = max(now_seen - u, 0);
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) stored = max(stored, __shfl_xor(stored, x));
      }
      float x[N / 4];
      scores(u, x);
      step(u, x, stored);
    }
    buffer ^= 1;
  }
  float l = over_groups_sum(st.l);
  if (!t.row(0)) return;
  if (walk.filler(0)) l = no_sums(st);
  if (a.parts > 1)
    store_part(a, t.split, t.token(0), t.head, g, st, l);
  else
    store_row<T>(a, t.token(0), t.head, g, st, st.m, l);
}

template <typename T, int CHUNKS>
hipError_t start(const AttendArgs& a, const AttendShape& shape, hipStream_t stream) {
  if (a.tile_tokens > 0) {
    constexpr int LONG = power_of_two(CHUNKS) * 64;  // bytes of a head's row in LDS; 16 KiB of keys to a stage at most
    constexpr int STAGE = LONG <= 256 ? 64 : 16384 / LONG;
    const auto kernel =
        a.prefix ? prefix_tiles<T, CHUNKS, STAGE> : attend_tiles<T, CHUNKS, STAGE, kTileWaves>;
    kernel<<<(unsigned)shape.groups, shape.threads, 0, stream>>>(a);
  } else {
    attend_kernel<T, CHUNKS><<<(unsigned)shape.groups, shape.threads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

// Pieces of a lane: a head of up to 64, 96, 128, 192 or 256 values.
template <typename T>
hipError_t start_dim(const AttendArgs& a, const AttendShape& shape, hipStream_t stream) {
  constexpr int U = 8 / Step<T>::kPiece;  // pieces of 32 values
  if (a.head_dim <= 64) return start<T, 2 * U>(a, shape, stream);
  if (a.head_dim <= 96) return start<T, 3 * U>(a, shape, stream);
  if (a.head_dim <= 128) return start<T, 4 * U>(a, shape, stream);
  if (a.head_dim <= 192) return start<T, 6 * U>(a, shape, stream);
  return start<T, 8 * U>(a, shape, stream);
}

AttendArgs attend_args(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q, const sdnn_heads& o,
                       const int32_t* chosen, int32_t blocks, float scale, float* lse, float* workspace) {
  AttendArgs a = attend_args(t, q, o, c.kv_heads, c.head_dim, c.block, c.dtype, scale);
  a.k_pages = c.k_pages, a.v_pages = c.v_pages, a.pages = c.pages;
  a.chosen = chosen, a.blocks = blocks;
  a.lse = lse, a.part = workspace;
  return a;
}

template <typename F>
hipError_t by_type(int dtype, const F& f) {
  return dtype == SDNN_F32 ? f(float()) : dtype == SDNN_F16 ? f(_Float16()) : f(__bf16());
}

hipError_t start(AttendArgs a, const AttendShape& shape, int dtype, hipStream_t stream) {
  a.tile_tokens = shape.tile_tokens, a.splits = shape.splits;
  return by_type(dtype, [&](auto t) { return start_dim<decltype(t)>(a, shape, stream); });
}

}  // namespace

hipError_t launch_attend(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q,
                         const sdnn_heads& o, const int32_t* chosen, int32_t blocks, float scale,
                         float* lse, float* workspace, hipStream_t stream) {
  const AttendShape shape = attend_shape(c, t, q.heads, chosen ? blocks : 0);
  if (!launchable(shape.groups, shape.threads) || !launchable(shape.join_groups, 256)) return hipErrorInvalidConfiguration;
  AttendArgs a = attend_args(c, t, q, o, chosen, blocks, scale, lse, workspace);
  a.parts = shape.splits;
  const hipError_t e = start(a, shape, c.dtype, stream);
  if (e != hipSuccess) return e;
  return by_type(c.dtype, [&](auto ty) { return join<decltype(ty)>(a, shape.join_groups, stream); });
}

// Attention with a shared prefix: the prefix's part for all tokens together, each token's part of its own blocks, then the
// parts of both joined.
//   64 sequences of 1 to 700 tokens behind 16384 that they share, 32 queries on 8 heads of 128 in 16 bits: 84 us.  The prefix 39.5
// (17 GFLOP at 435 TFLOP/s; vector instructions beside the matrix unit, as in attend_tiles), the tokens' own blocks 33 (110 MB at
// 3.3 TB/s), the join of 33 parts 12.  Both in one launch, a prefix's workgroup in turn with two others: 122 us (for 87); the
// prefix's LDS leaves a compute unit two workgroups, and its registers are too few for the others.  Two tiles to a wave of the prefix: 48
// us for 42; half and a quarter as many shares of it are slower.
hipError_t launch_attend_shared(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q, const sdnn_heads& o,
                                int32_t shared, float scale, float* lse, float* workspace, hipStream_t stream) {
  const SharedShape s = shared_shape(c, t.tokens, t.sequences, t.max_blocks, q.heads, shared);
  if (!s.fits) return hipErrorInvalidConfiguration;
  AttendArgs a = attend_args(c, t, q, o, nullptr, t.max_blocks, scale, lse, workspace);
  a.parts = s.parts;
  a.prefix = shared;
  hipError_t e = start(a, s.prefix, c.dtype, stream);
  if (e != hipSuccess) return e;
  a.prefix = 0, a.first = shared, a.part_first = s.prefix.splits;
  if (s.own.splits > 0) e = start(a, s.own, c.dtype, stream);
  if (e != hipSuccess) return e;
  return by_type(c.dtype, [&](auto ty) { return join<decltype(ty)>(a, s.join_groups, stream); });
}

}  // namespace sdnn
