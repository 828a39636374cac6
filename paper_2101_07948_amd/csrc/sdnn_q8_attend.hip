// Attention over the cache in 8 bits.
#include "sdnn_attend_device.h"
#include "sdnn_serve_shape.h"

namespace sdnn {
namespace {

struct Q8AttendArgs : AttendArgs {
  const float* k_scales;
  const float* v_scales;
};

// The numbers of keys and values are whole and below 2^8: exact in 16-bit floats, which the matrix unit takes.  Queries and
// probabilities are sums of such parts, each a product of its own.  Queries: 3 parts in bf16 hold the 24 bits of a float; those of
// 16 bits are taken as they are, keys in their type.  Probabilities, whose exponents f16 has not: bf16, 2 parts (16 bits) where the
// output has 8 or 11, 3 where it has 24.  The scale of a key multiplies its score, that of a value its probability, both in 32
// bits.
template <typename T>
struct Parts {
  typedef __bf16 Key;
  typedef bf16x8 Key8;
  static constexpr int kQ = 1, kP = 2;
};
template <>
struct Parts<float> {
  typedef __bf16 Key;
  typedef bf16x8 Key8;
  static constexpr int kQ = 3, kP = 3;
};
template <>
struct Parts<_Float16> {
  typedef _Float16 Key;
  typedef f16x8 Key8;
  static constexpr int kQ = 1, kP = 2;
};

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight numbers as 16-bit floats.  bf16: the upper halves of 32-bit floats, which have no bits below.  f16: with 128 added (a
// bit turned) a number is the lower byte of 1024 + it; 1152 is subtracted.
__device__ __forceinline__ uint32_t widen2(int32_t w, int at) {
  const float a = (float)(int8_t)(w >> at), b = (float)(int8_t)(w >> (at + 8));
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ void widen(int32_t lo, int32_t hi, bf16x8* y) {
  const uint32_t x[4] = {widen2(lo, 0), widen2(lo, 16), widen2(hi, 0), widen2(hi, 16)};
  __builtin_memcpy(y, x, sizeof(x));
}
__device__ __forceinline__ void widen(int32_t lo, int32_t hi, f16x8* y) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  const uint32_t a = (uint32_t)lo ^ 0x80808080u, b = (uint32_t)hi ^ 0x80808080u;
  const uint32_t x[4] = {__builtin_amdgcn_perm(0x64646464u, a, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u),
                         __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u), __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)};
  f16x2 z[4];
  __builtin_memcpy(z, x, sizeof(x));
#pragma unroll
  for (int i = 0; i < 4; ++i) z[i] = z[i] - f16x2{(_Float16)1152.0f, (_Float16)1152.0f};
  __builtin_memcpy(y, z, sizeof(z));
}

template <int N, typename H>
__device__ __forceinline__ void split(float x, H (&out)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    out[i] = (H)x;
    if (i + 1 < N) x -= (float)out[i];
  }
}

// The queries' parts: piece i of a lane has values `at(i)` ... + 7 of its row.  Returns the largest magnitude of them.
template <typename T, int PIECES, typename AT>
__device__ __forceinline__ float load_queries(const AttendArgs& a, bool row, int t, int64_t head, const AT& at,
                                              typename Parts<T>::Key8 (&q)[Parts<T>::kQ][PIECES]) {
  float most = 0.0f;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int d = at(i);
    T x[8] = {};
    if (row && d < a.head_dim) {
      constexpr int V = 16 / sizeof(T);
#pragma unroll
      for (int j = 0; j < 8; j += V) {
        T y[V];
        load_n<V>(static_cast<const T*>(a.q) + t * a.q_token + head * a.q_head + d + j, a.q_aligned, y);
#pragma unroll
        for (int e = 0; e < V; ++e) x[j + e] = y[e];
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      typename Parts<T>::Key part[Parts<T>::kQ];
      split((float)x[e], part);
      most = fmaxf(most, fabsf((float)x[e]));
#pragma unroll
      for (int k = 0; k < Parts<T>::kQ; ++k) q[k][i][e] = a.negate ? -part[k] : part[k];
    }
  }
  return most;
}

// One step of E tokens to a lane, their scores s (without the keys' scales) given: tokens E g ... E g + E - 1 of which the
// first `seen` of the step's are within this lane's query's sight.  ks, scales: those of their keys and values.  EMPTY: see
// attend_step; a query that sees nothing of a step has m = infinity for it and so p = 0, if its scores, which are not masked
// where no query of the tile sees a part of the step, are finite.  odd: they may not be, or a value's scale is not (of a row that is
// not finite, or what memory held that no token was stored to): all that is out of sight is masked.  (Masks in all steps
// that some query sees nothing of: 2048 tokens over 16 of 128 blocks each 195 us for 169.)  A scale that is NaN within sight makes
// the query's sums NaN.  Leaves what multiplies the tokens' values, in parts.
template <bool EMPTY, typename T, int E, int TILES>
__device__ __forceinline__ void q8_weights(float scale2, float (&s)[E], const float (&ks)[E], const float (&scales)[E], bool odd,
                                           int seen, int g, State<TILES>& st, bf16x8 (&p)[Parts<T>::kP][E / 8]) {
  constexpr float HIGH = 8.0f;
  float vs[E];
#pragma unroll
  for (int j = 0; j < E; ++j) s[j] *= ks[j], vs[j] = scales[j];
  if (odd || __any(seen < 4 * E && (!EMPTY || seen > 0))) {
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const bool in_sight = E * g + j < seen;
      s[j] = in_sight ? s[j] : -INFINITY, vs[j] = in_sight ? vs[j] : 0.0f;
    }
  }
  float top = s[0];
#pragma unroll
  for (int j = 1; j < E; ++j) top = fmaxf(top, s[j]);
  const bool sees = !EMPTY || seen > 0;
  const float above = fmaf(top, scale2, -st.m);
  if (__any(sees && !(above <= HIGH))) {
    const float row = over_groups_max(sees ? top * scale2 : -INFINITY);
    const float m = fmaxf(row, st.m);
    const float f = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.m - m);
    st.l *= f;
    st.m = m;
#pragma unroll
    for (int c = 0; c < TILES; ++c) st.o[c] *= f;
  }
  const float m = sees ? st.m : INFINITY;
#pragma unroll
  for (int j = 0; j < E; ++j) s[j] = __builtin_amdgcn_exp2f(fmaf(s[j], scale2, -m));
  float sum = s[0];
#pragma unroll
  for (int j = 1; j < E; ++j) sum += s[j];
  st.l += sum;
#pragma unroll
  for (int j = 0; j < E; j += 2) {
    float x[2] = {s[j] * vs[j], s[j + 1] * vs[j + 1]};
#pragma unroll
    for (int k = 0; k < Parts<T>::kP; ++k) {
      typename VecOf<2, __bf16>::type h;
      take_pair(x, &h);
      p[k][j / 8][j % 8] = h[0], p[k][j / 8][j % 8 + 1] = h[1];
    }
  }
}

// Waves of a SIMD that the registers leave room for.
constexpr int q8_waves(int pieces) { return pieces <= 4 ? 2 : 1; }

// Single tokens: as attend_kernel, with steps of N tokens, 4 N / 16 to a lane.  A lane reads 16 numbers of a key at a time
// (DIMS pieces of 64 values for the four lane groups), and of a value N / 4 tokens' numbers: each instruction takes whole runs
// of 64 bytes and more of a page.  Everything a step needs is asked for before its first product.
//   Reading bounds it.  A token of 32 queries on 8 heads of 128 over 131072 tokens: 54 us, 277 MB at 5.1 TB/s, and 6 to join;
// 32 sequences of up to 4096 tokens, 12 heads of 64 in 32 bits: 36 us, 131 MB at 3.6 TB/s, and 5 to join (sequences of different
// lengths end at different times).
template <typename T, int DIMS, int N>
__global__ __launch_bounds__(kWaves * 64, q8_waves(2 * DIMS)) void q8_kernel(Q8AttendArgs a) {
  constexpr int TILES = DIMS * 4, E = N / 4, W = E / 4;  // W: words of a lane's piece of a value
  __shared__ JoinLds<TILES> lds;
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane & 15, g = lane >> 4;
  int b = blockIdx.x;
  const int h = b % a.kv_heads;
  b /= a.kv_heads;
  const int split_at = b % a.splits;
  b /= a.splits;
  const int first = b % a.head_tiles * kRows;
  const int t = b / a.head_tiles;
  const int rows = min(kRows, a.group - first);
  const int64_t head = (int64_t)h * a.group + first + r;
  const int D = a.head_dim, P = a.block;
  const int32_t p = a.pos[t], seq = a.seq[t];
  const bool filler = p < 0 || (uint32_t)seq >= (uint32_t)a.sequences;
  const int own = p / P;
  const int n = filler ? 0 : a.chosen ? a.blocks : max(min(own + 1, a.max_blocks) - a.first, 0);
  const int32_t* chosen = a.chosen ? a.chosen + ((int64_t)t * a.kv_heads + h) * a.blocks : nullptr;
  const int32_t* table = a.table + (int64_t)seq * a.max_blocks;
  const int shift = __builtin_ctz(P / N), deal = a.splits * kWaves, last = n << shift;
  typedef typename Parts<T>::Key8 Key8;
  Key8 q[Parts<T>::kQ][2 * DIMS];
  load_queries<T, 2 * DIMS>(a, r < rows, t, head, [&](int i) { return (i / 2 * 4 + g) * 16 + i % 2 * 8; }, q);
  State<TILES> st;
#pragma unroll
  for (int c = 0; c < TILES; ++c) st.o[c] = f32x4{0, 0, 0, 0};
  st.m = -INFINITY, st.l = 0.0f;
  for (int first_step = split_at * kWaves + wave; first_step < last; first_step += 64 * deal) {
    const int mine = first_step + lane * deal;
    int id = -1, page_mine = -1;
    if (lane < (last - first_step + deal - 1) / deal) id = chosen ? chosen[mine >> shift] : a.first + (mine >> shift);
    const auto seen_of = [&](int id, int t0) { return min(p - id * P - t0, P) + 1; };  // (p up to 2^31 - 1)
    const auto token_of = [&](int u) { return (u & ((1 << shift) - 1)) * N; };
    if (id >= 0 && id <= own && id < a.max_blocks && seen_of(id, token_of(mine)) > 0) page_mine = table[id];
    uint64_t todo = __ballot(page_mine >= 0 && page_mine < a.pages);
    for (; todo; todo &= todo - 1) {
      const int j = __builtin_ctzll(todo);
      const int page = __builtin_amdgcn_readlane(page_mine, j), t0 = token_of(first_step + j * deal);
      const int seen = seen_of(__builtin_amdgcn_readlane(id, j), t0);
      const int64_t at = ((int64_t)page * a.kv_heads + h) * P;
      const int8_t* k = static_cast<const int8_t*>(a.k_pages) + (at + t0) * D;
      const int8_t* v = static_cast<const int8_t*>(a.v_pages) + at * D + t0;
      i32x4 kk[N / 16][DIMS];
      typename VecOf<W, int32_t>::type vv[TILES];
#pragma unroll
      for (int x = 0; x < N / 16; ++x)
#pragma unroll
        for (int c = 0; c < DIMS; ++c) {
          const int token = E * (r >> 2) + 4 * x + (r & 3), d = min((c * 4 + g) * 16, D - 16);  // past the end: q is 0 there
          kk[x][c] = *reinterpret_cast<const i32x4*>(k + token * D + d);
        }
      float ks[E], vs[E];
#pragma unroll
      for (int x = 0; x < E; x += 4) {
        const f32x4 y = *reinterpret_cast<const f32x4*>(a.k_scales + at + t0 + E * g + x);
        const f32x4 z = *reinterpret_cast<const f32x4*>(a.v_scales + at + t0 + E * g + x);
#pragma unroll
        for (int e = 0; e < 4; ++e) ks[x + e] = y[e], vs[x + e] = z[e];
      }
#pragma unroll
      for (int c = 0; c < TILES; ++c)
        vv[c] = *reinterpret_cast<const typename VecOf<W, int32_t>::type*>(v + min(c * 16 + r, D - 1) * P + E * g);
      __builtin_amdgcn_sched_barrier(0);
      float s[E];
#pragma unroll
      for (int x = 0; x < N / 16; ++x) {
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < DIMS; ++c)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            Key8 y;
            widen(kk[x][c][2 * e], kk[x][c][2 * e + 1], &y);
#pragma unroll
            for (int part = 0; part < Parts<T>::kQ; ++part) acc = mfma(y, q[part][2 * c + e], acc);
          }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * x + i] = acc[i];
      }
      bf16x8 w[Parts<T>::kP][E / 8];
      q8_weights<false, T, E, TILES>(a.scale2, s, ks, vs, false, seen, g, st, w);
#pragma unroll
      for (int c = 0; c < TILES; ++c)
#pragma unroll
        for (int e = 0; e < E / 8; ++e) {
          bf16x8 y;
          widen(vv[c][2 * e], vv[c][2 * e + 1], &y);
#pragma unroll
          for (int x = 0; x < Parts<T>::kP; ++x) st.o[c] = mfma(y, w[x][e], st.o[c]);
        }
    }
  }
  join_waves<T>(a, lds, split_at, t, head, r < rows, st);
}

// ---------------------------------------------------------------- many tokens of a sequence

// Tiles of 16 queries to a wave of q8_tiles.  In 32 bits, whose parts make three products of what is read from LDS, two where
// they fit the registers; in 16 bits one, which leaves room for four waves to a SIMD.  (One and two: 2048 tokens at the end of
// 8192, 32 queries on 8 heads of 128, 450 us and 461; at the end of 4096, 12 heads of 64, 80 and 93; 512 tokens, 16 queries on 4
// heads of 192, 68 and 103; 512 tokens of 12 heads of 64 in 32 bits 55 and 48.)
template <typename T>
constexpr int q8_tiles_of(int chunks) {
  return sizeof(T) == 4 && chunks <= 3 ? 2 : 1;
}

// With scales of keys below the first, and queries (times the scale of scores, where that is above 1) below the second, a score of
// up to 256 numbers of up to 2^7 is below 2^127.
constexpr float kLargeScale = 0x1p20f, kLargeQuery = 0x1p92f;

// A stage of `tokens` tokens on its way to LDS: a thread holds pieces of 16 numbers of keys' rows and of values', and some of
// the threads a scale.  They are asked for while the stage before is computed, and widened on their way into the tile, so that
// its waves find matrix operands there.  Where a thread's pieces come from and go to is worked out once.
template <typename T, int CHUNKS, int STAGE, int WAVES>
struct Q8Stage {
  static constexpr int kThreads = WAVES * 64, kPieces = (STAGE * CHUNKS * 2 + kThreads - 1) / kThreads;
  typedef Tile<typename Parts<T>::Key, CHUNKS, STAGE> L;
  static_assert(2 * STAGE <= kThreads, "a scale to a thread");
  i32x4 k[kPieces], v[kPieces];
  float scale;
  int32_t from[kPieces], k_to[kPieces][2], v_to[kPieces][2];  // from: of values; those of keys lie one after the other
  bool there[kPieces], scaled;
  __device__ __forceinline__ Q8Stage(const AttendArgs& a, int tokens) {
    const int D = a.head_dim, per = tokens / 16;  // (2 or 4)
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int i = threadIdx.x + j * kThreads, d = i / per, y = i - d * per, row = i * 16 / D, x = (i * 16 - row * D) / 8;
      there[j] = i * 16 < tokens * D;
      from[j] = d * a.block + y * 16;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        k_to[j][e] = (int)(L::key(nullptr, row, x + e) - static_cast<const unsigned char*>(nullptr));
        v_to[j][e] = (int)(L::value(nullptr, d, y * 2 + e) - static_cast<const unsigned char*>(nullptr));
      }
      k[j] = v[j] = i32x4{0, 0, 0, 0};
    }
    scaled = threadIdx.x < 2 * STAGE && (int)threadIdx.x % STAGE < tokens;
    scale = 0.0f;
  }
  __device__ __forceinline__ void load(const Q8AttendArgs& a, int page, int h, int t0) {
    const int D = a.head_dim, P = a.block;
    const int64_t at = ((int64_t)page * a.kv_heads + h) * P;
    const int8_t* kp = static_cast<const int8_t*>(a.k_pages) + (at + t0) * D;
    const int8_t* vp = static_cast<const int8_t*>(a.v_pages) + at * D + t0;
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
      if (there[j]) {
        k[j] = *reinterpret_cast<const i32x4*>(kp + (threadIdx.x + j * kThreads) * 16);
        v[j] = *reinterpret_cast<const i32x4*>(vp + from[j]);
      }
    if (scaled) scale = (threadIdx.x < STAGE ? a.k_scales : a.v_scales)[at + t0 + threadIdx.x % STAGE];
  }
  // (odd: of each wave that has scales, whether one of them is large, infinite or not a number.)
  __device__ __forceinline__ void store(unsigned char* lds, float* scales, int32_t* odd) const {
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
      if (there[j]) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          widen(k[j][2 * e], k[j][2 * e + 1], reinterpret_cast<typename Parts<T>::Key8*>(lds + k_to[j][e]));
          widen(v[j][2 * e], v[j][2 * e + 1], reinterpret_cast<bf16x8*>(lds + v_to[j][e]));
        }
      }
    if (threadIdx.x < 2 * STAGE) {
      scales[threadIdx.x] = scale;
      const bool any = __any(!(fabsf(scale) < kLargeScale));
      if (threadIdx.x % 64 == 0) odd[threadIdx.x / 64] = any;
    }
  }
};

// As attend_tiles: a workgroup's waves, tiles of neighbouring tokens of one cached head, walk their blocks through LDS.
//   2048 tokens at the end of 8192, 32 queries on 8 heads of 128 in 16 bits: 415 to 431 us, 241 GFLOP at 570 TFLOP/s; over 16 of
// 128 blocks each 170 us.  A step is 24 matrix instructions, 8 of them for the probabilities' second part, and 140 vector ones
// (scales, exponentials, sums, parts).  Waiting bounds it: the vector unit is busy for half of the time, the matrix unit for a
// third, and waves wait in 44 % of theirs, those of a workgroup being in the same part of a step between the same barriers.  Blocks found by
// lists as in attend_tiles: 779 us; places in LDS worked out for each stage, two tiles to a wave: 459.  Two steps of 32 tokens
// under way at once: 524, registers spill.
template <typename T, int CHUNKS, int STAGE, bool LISTS, bool PREFIX>
__global__ __launch_bounds__(kTileWaves / q8_tiles_of<T>(CHUNKS) * 64, CHUNKS <= 4 && sizeof(T) == 2 ? 4 : 2)
void q8_tiles(Q8AttendArgs a) {
  typedef typename Parts<T>::Key Key;
  typedef Tile<Key, CHUNKS, STAGE> L;
  constexpr int TILES = CHUNKS * 2, N = 32, E = N / 4, R = q8_tiles_of<T>(CHUNKS), WAVES = kTileWaves / R;
  __shared__ __align__(16) unsigned char lds[2 * 2 * L::kBytes];
  __shared__ __align__(16) float scales[2 * 2 * STAGE];  // of keys, of values; twice
  __shared__ int32_t odd[2][2 * STAGE / 64];             // see Q8Stage::store
  __shared__ typename Walk<LISTS, R>::Lds walked;
  const TileRows<R> t(a);
  const int r = t.r, g = t.g, D = a.head_dim;
  typename Parts<T>::Key8 q[R][Parts<T>::kQ][CHUNKS];
  State<TILES> st[R];
  float most[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    most[i] = load_queries<T, CHUNKS>(a, t.row(i), t.token(i), t.head, [&](int c) { return (c * 4 + g) * 8; }, q[i]);
#pragma unroll
    for (int c = 0; c < TILES; ++c) st[i].o[c] = f32x4{0, 0, 0, 0};
    st[i].m = -INFINITY, st[i].l = 0.0f;
  }
  Walk<LISTS, R> walk;
  walk.template start<PREFIX>(a, t, walked);
  bool large = false;
#pragma unroll
  for (int i = 0; i < R; ++i) large = large || (!walk.filler(i) && !(most[i] * fmaxf(a.scale2, 1.0f) < kLargeQuery));
  large = __any(large);
  const int stage = min(STAGE, a.block), stages = a.block / stage;
  Q8Stage<T, CHUNKS, STAGE, WAVES> next_stage(a, stage);

  // Where this lane's pieces of a step's keys and values lie: 32 tokens on, and 4, keys' rows are permuted alike, and so are
  // values' 16 on.
  int key_at[CHUNKS], value_at[STAGE / N];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
    key_at[c] = (int)(L::key(nullptr, 8 * (r >> 2) + (r & 3), min(c * 4 + g, D / 8 - 1)) -
                      static_cast<const unsigned char*>(nullptr));
#pragma unroll
  for (int u = 0; u < STAGE; u += N)
    value_at[u / N] = (int)(L::value(nullptr, r, u / 8 + g) - static_cast<const unsigned char*>(nullptr));

  int buffer = 0, s = 0;
  if (walk.key != walk.END) {
    if (walk.page >= 0) next_stage.load(a, walk.page, t.h, 0);
    next_stage.store(lds, scales, odd[0]);
  }
  while (walk.key != walk.END) {
    int32_t now_seen[R];
#pragma unroll
    for (int i = 0; i < R; ++i) now_seen[i] = walk.seen[i] - s * stage;
    __syncthreads();  // the stage is in LDS, the other buffer is free, the offers are made
    if (++s == stages) {
      s = 0;
      walk.advance(a, t, walked);
    }
    const bool more = walk.key != walk.END && walk.page >= 0;
    if (more) next_stage.load(a, walk.page, t.h, s * stage);
    const unsigned char* tile = lds + buffer * 2 * L::kBytes;
    const float* factors = scales + buffer * 2 * STAGE + E * g;
    int32_t masked = large;  // (of each lane, so that it is not waited for before a step's scores are there)
#pragma unroll
    for (int i = 0; i < 2 * STAGE / 64; ++i) masked |= odd[buffer][i];
    // a step of tokens u ...
    const auto step = [&](int u) {
      float x[R][E], ks[E], vs[E];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        f32x4 acc[R];
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          const auto y = *reinterpret_cast<const typename Parts<T>::Key8*>(tile + key_at[c] + (u + 4 * half) * L::kKeyPieces * 16);
#pragma unroll
          for (int i = 0; i < R; ++i)
#pragma unroll
            for (int part = 0; part < Parts<T>::kQ; ++part) acc[i] = mfma(y, q[i][part][c], acc[i]);
        }
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[i][4 * half + e] = acc[i][e];
      }
#pragma unroll
      for (int i = 0; i < E; i += 4) {
        const f32x4 y = *reinterpret_cast<const f32x4*>(factors + u + i);
        const f32x4 z = *reinterpret_cast<const f32x4*>(factors + STAGE + u + i);
#pragma unroll
        for (int e = 0; e < 4; ++e) ks[i + e] = y[e], vs[i + e] = z[e];
      }
      bf16x8 w[R][Parts<T>::kP][1];
      const bool any = __builtin_amdgcn_readfirstlane(masked);
#pragma unroll
      for (int i = 0; i < R; ++i) q8_weights<true, T, E, TILES>(a.scale2, x[i], ks, vs, any, now_seen[i] - u, g, st[i], w[i]);
#pragma unroll
      for (int c = 0; c < TILES; ++c) {
        const bf16x8 v = *reinterpret_cast<const bf16x8*>(tile + value_at[u / N] + c * 16 * L::kValuePieces * 16);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int k = 0; k < Parts<T>::kP; ++k) st[i].o[c] = mfma(v, w[i][k][0], st[i].o[c]);
      }
    };
    int32_t most = now_seen[0];
#pragma unroll
    for (int i = 1; i < R; ++i) most = max(most, now_seen[i]);
#pragma unroll
    for (int u = 0; u < STAGE; u += N)
      if (u < stage && __any(most > u)) step(u);
    if (more) next_stage.store(lds + (buffer ^ 1) * 2 * L::kBytes, scales + (buffer ^ 1) * 2 * STAGE, odd[buffer ^ 1]);
    buffer ^= 1;
  }

#pragma unroll
  for (int i = 0; i < R; ++i) {
    float l = over_groups_sum(st[i].l);
    if (!t.row(i)) continue;
    if (walk.filler(i)) l = no_sums(st[i]);
    if (a.parts > 1)
      store_part(a, t.split, t.token(i), t.head, g, st[i], l);
    else
      store_row<T>(a, t.token(i), t.head, g, st[i], st[i].m, l);
  }
}

template <typename T, int DIMS, int CHUNKS>
hipError_t start(const Q8AttendArgs& a, const AttendShape& shape, hipStream_t stream) {
  if (a.tile_tokens > 0) {
    constexpr int LONG = power_of_two(CHUNKS) * 64, STAGE = LONG <= 256 ? 64 : 16384 / LONG;
    const auto kernel = a.prefix   ? q8_tiles<T, CHUNKS, STAGE, false, true>
                        : a.chosen ? q8_tiles<T, CHUNKS, STAGE, true, false>
                                   : q8_tiles<T, CHUNKS, STAGE, false, false>;
    kernel<<<(unsigned)shape.groups, kTileWaves / q8_tiles_of<T>(CHUNKS) * 64, 0, stream>>>(a);
  } else {
    const auto kernel = a.block == 32 ? q8_kernel<T, DIMS, 32> : q8_kernel<T, DIMS, 64>;
    kernel<<<(unsigned)shape.groups, shape.threads, 0, stream>>>(a);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t start_dim(const Q8AttendArgs& a, const AttendShape& shape, hipStream_t stream) {
  if (a.head_dim <= 64) return start<T, 1, 2>(a, shape, stream);
  if (a.head_dim <= 96) return start<T, 2, 3>(a, shape, stream);
  if (a.head_dim <= 128) return start<T, 2, 4>(a, shape, stream);
  if (a.head_dim <= 192) return start<T, 3, 6>(a, shape, stream);
  return start<T, 4, 8>(a, shape, stream);
}

template <typename F>
hipError_t by_type(int dtype, const F& f) {
  return dtype == SDNN_F32 ? f(float()) : dtype == SDNN_F16 ? f(_Float16()) : f(__bf16());
}

hipError_t start(Q8AttendArgs a, const AttendShape& shape, int dtype, hipStream_t stream) {
  a.tile_tokens = shape.tile_tokens, a.splits = shape.splits;
  return by_type(dtype, [&](auto t) { return start_dim<decltype(t)>(a, shape, stream); });
}

}  // namespace

hipError_t launch_q8_attend(const sdnn_q8_cache& c, const sdnn_tokens& t, int dtype, const sdnn_heads& q, const sdnn_heads& o,
                            const int32_t* chosen, int32_t blocks, int32_t shared, float scale, float* lse, float* workspace,
                            hipStream_t stream) {
  const sdnn_block_cache as = as_blocks(c);
  Q8AttendArgs a = {};
  static_cast<AttendArgs&>(a) = attend_args(t, q, o, c.kv_heads, c.head_dim, c.block, dtype, scale);
  a.k_pages = c.k_codes, a.v_pages = c.v_codes, a.k_scales = c.k_scales, a.v_scales = c.v_scales, a.pages = c.pages;
  a.chosen = chosen, a.blocks = blocks, a.lse = lse, a.part = workspace;
  int64_t joined = 0;
  hipError_t e;
  if (shared > 0 && t.sequences > 1) {
    const SharedShape s = shared_shape(as, t.tokens, t.sequences, t.max_blocks, q.heads, shared);
    if (!s.fits) return hipErrorInvalidConfiguration;
    a.parts = s.parts, joined = s.join_groups;
    a.prefix = shared;
    e = start(a, s.prefix, dtype, stream);
    if (e != hipSuccess) return e;
    a.prefix = 0, a.first = shared, a.part_first = s.prefix.splits;
    if (s.own.splits > 0) e = start(a, s.own, dtype, stream);
  } else {
    const AttendShape s = attend_shape(as, t, q.heads, chosen ? blocks : 0);
    if (!launchable(s.groups, s.threads) || !launchable(s.join_groups, 256)) return hipErrorInvalidConfiguration;
    a.parts = s.splits, joined = s.join_groups;
    e = start(a, s, dtype, stream);
  }
  if (e != hipSuccess) return e;
  return by_type(dtype, [&](auto ty) { return join<decltype(ty)>(a, joined, stream); });
}

}  // namespace sdnn
