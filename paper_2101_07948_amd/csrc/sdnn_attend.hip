// Attention over the chosen blocks of the cache.
#include "sdnn_decode_device.h"
#include "sdnn_decode_shape.h"

namespace sdnn {
namespace {

struct AttendArgs {
  const void* q;
  void* o;
  int64_t q_token, q_head, o_token, o_head;
  const void* k_pages;
  const void* v_pages;
  int64_t pages;
  const int32_t* pos;
  const int32_t* seq;
  const int32_t* table;
  const int32_t* chosen;  // NULL: every block
  float* lse;
  float* part;            // splits > 1: sums, then maxima and totals (see attend_join)
  int32_t tokens, sequences, max_blocks;
  int32_t heads, kv_heads, group, head_tiles, head_dim, block;
  int32_t blocks, splits;
  int32_t tile_tokens;    // 0: attend_kernel; else attend_tiles, tokens of a wave's tile
  float scale2;           // |scale| * log2 e
  int32_t negate;         // scale < 0: the queries are negated
  int32_t q_aligned, o_aligned;
};

// One step of a wave: TOKENS cached tokens against a tile of 16 queries.  The scores are computed
// turned, tokens by queries, so that a lane's results are scores of its own query (lane & 15) for
// tokens that the second product takes from it as its operand: probabilities never leave the
// registers.  Keys and values are read from the pages straight into operands, 16 bytes a lane.
//   CHUNKS: 16-byte pieces of a head that a lane holds (4 lane groups: 4 CHUNKS pieces a head).
template <typename T>
struct Step;

// 16-bit values: 32 tokens, v_mfma_f32_16x16x32.  Row r of half s of the keys is token
// 8 (r / 4) + 4 s + r % 4, so that lane group g ends up with scores of tokens 8 g ... 8 g + 7.
template <typename T, typename V8>
struct Step16 {
  static constexpr int kTokens = 32, kPiece = 8;
  typedef V8 Piece;
  static __device__ __forceinline__ f32x4 mfma(V8 a, V8 b, f32x4 c);

  static __device__ __forceinline__ int token(int half, int r) { return 8 * (r >> 2) + 4 * half + (r & 3); }

  // The keys and the values of a step: 2 CHUNKS pieces each.
  template <int CHUNKS>
  static __device__ __forceinline__ void load_keys(const T* k, int D, int r, int g, V8 (&kk)[2 * CHUNKS]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        const int d = min((c * 4 + g) * 8, D - 8);  // past the head's end: any of its values, q is 0 there
        kk[h * CHUNKS + c] = *reinterpret_cast<const V8*>(k + token(h, r) * D + d);
      }
  }
  template <int CHUNKS>
  static __device__ __forceinline__ void load_values(const T* v, int D, int P, int r, int g, V8 (&vv)[2 * CHUNKS]) {
#pragma unroll
    for (int c = 0; c < 2 * CHUNKS; ++c)
      vv[c] = *reinterpret_cast<const V8*>(v + min(c * 16 + r, D - 1) * P + 8 * g);
  }

  // kk(i), vv(i): piece i of the step's keys and values (what `load` puts there).
  template <int CHUNKS, typename K>
  static __device__ __forceinline__ void scores(const K& kk, const V8 (&q)[CHUNKS], float (&s)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) acc = mfma(kk(h * CHUNKS + c), q[c], acc);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * h + i] = acc[i];
    }
  }

  // o += p v.  p is split into two 16-bit parts: with one its rounding would add an error as large as that of o, with two
  // what is lost is 2^-17 of p in bf16 (a 256th of the rounding of o) and 2^-22 in f16, there at least 2^-25, which
  // attend_step keeps apart from what counts.  The sum of probabilities takes all 24 bits.
  // PART: tokens from `stored` on may hold anything (their p is 0).
  template <bool PART, int CHUNKS, typename V>
  static __device__ __forceinline__ void accumulate(const V& vv, const float (&p)[8], int g, int stored,
                                                    f32x4 (&o)[2 * CHUNKS]) {
    V8 hi, lo;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      hi[j] = (T)p[j];
      lo[j] = (T)(p[j] - (float)hi[j]);
    }
#pragma unroll
    for (int c = 0; c < 2 * CHUNKS; ++c) {
      V8 x = vv(c);
      if (PART) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (8 * g + j >= stored) x[j] = (T)0.0f;
      }
      o[c] = mfma(x, hi, o[c]);
      o[c] = mfma(x, lo, o[c]);
    }
  }
};
template <>
__device__ __forceinline__ f32x4 Step16<_Float16, f16x8>::mfma(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x4 Step16<__bf16, bf16x8>::mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
template <>
struct Step<_Float16> : Step16<_Float16, f16x8> {};
template <>
struct Step<__bf16> : Step16<__bf16, bf16x8> {};

// 32-bit values: 16 tokens, v_mfma_f32_16x16x4 (a lane gives one value of each operand; value e of
// a piece is step e, in both operands alike).
template <>
struct Step<float> {
  static constexpr int kTokens = 16, kPiece = 4;
  typedef f32x4 Piece;

  template <int CHUNKS>
  static __device__ __forceinline__ void load_keys(const float* k, int D, int r, int g, f32x4 (&kk)[CHUNKS]) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int d = min((c * 4 + g) * 4, D - 4);
      kk[c] = *reinterpret_cast<const f32x4*>(k + r * D + d);
    }
  }
  template <int CHUNKS>
  static __device__ __forceinline__ void load_values(const float* v, int D, int P, int r, int g, f32x4 (&vv)[CHUNKS]) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
      vv[c] = *reinterpret_cast<const f32x4*>(v + min(c * 16 + r, D - 1) * P + 4 * g);
  }

  template <int CHUNKS, typename K>
  static __device__ __forceinline__ void scores(const K& kk, const f32x4 (&q)[CHUNKS], float (&s)[4]) {
    f32x4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const f32x4 x = kk(c);
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], q[c][e], acc, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = acc[i];
  }

  template <bool PART, int CHUNKS, typename V>
  static __device__ __forceinline__ void accumulate(const V& vv, const float (&p)[4], int g, int stored,
                                                    f32x4 (&o)[CHUNKS]) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      f32x4 x = vv(c);
      if (PART) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (4 * g + j >= stored) x[j] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], p[e], o[c], 0, 0, 0);
    }
  }
};

// A wave's state: of query lane & 15 the reference that exponents are taken from (in units of log 2, see
// attend_step) and the lane's share of the total (tokens of its lane group), and the sums o[c][i] of value 16 c + 4 (lane / 16) + i.
template <int TILES>
struct State {
  f32x4 o[TILES];
  float m, l;
};

__device__ __forceinline__ float over_groups_max(float x) { return max_over_32(max_over_16(x)); }
__device__ __forceinline__ float over_groups_sum(float x) {
  float u, v;
  with_16(x, &u, &v);
  with_32(u + v, &u, &v);
  return u + v;
}

// The logarithm of a query's sum l of exponentials taken from m (in units of log 2).  l's exponent joins m first: where m
// is far from the maximum (see attend_step) both are large and cancel.
__device__ __forceinline__ float log_of_sum(float m, float l) {
  if (!(l > 0.0f)) return -INFINITY;
  return ((m + (float)__builtin_amdgcn_frexp_expf(l)) + __log2f(__builtin_amdgcn_frexp_mantf(l))) * 0.693147181f;
}

// A share's part of a query: the sums, then for all parts their reference and total.
template <int TILES>
__device__ __forceinline__ void store_part(const AttendArgs& a, int split, int t, int64_t head, int g, const State<TILES>& st,
                                           float l) {
  const int64_t row = ((int64_t)split * a.tokens + t) * a.heads + head;
#pragma unroll
  for (int c = 0; c < TILES; ++c)
    if (c * 16 + 4 * g < a.head_dim) *reinterpret_cast<f32x4*>(a.part + row * a.head_dim + c * 16 + 4 * g) = st.o[c];
  if (g == 0) {
    float* ml = a.part + (int64_t)a.splits * a.tokens * a.heads * a.head_dim + row * 2;
    ml[0] = st.m, ml[1] = l;
  }
}

// One step, its scores s given: tokens [0, seen) of its are within the sight of this lane's query, tokens from `stored` on may
// hold anything.  EMPTY: queries may see nothing here (seen <= 0), or have seen nothing yet (m = -infinity).
//   m is a reference near the running maximum rather than the maximum: it rises only where a score is over 2^HIGH times
// above it, so that most steps neither reduce over lanes nor rescale the sums.  Scores are masked one by one only where
// a query's sight ends within the step; a query that sees nothing of it gets m = infinity for the step, p = 0.
//   p is a float, and its parts in bf16 have its exponents.  Parts in f16 end at 2^-24, while what an output is made of may
// be far below the query's largest p, where that meets a value near 0.  So in f16 m is 2^HEAD below a new maximum (p up
// to 2^15): a p of 2^-21 of the largest keeps its 16 bits, and none above 2^-37 is dropped.  And where all scores of a
// step are below m, m comes down to them, as far as sums in 32 bits allow.  (2048 tokens over 16 of 128 blocks: 148 us
// and 147 without; with scores that spread five times as wide, where m falls in some step of most tiles, 173 and 148.)
template <bool EMPTY, typename T, int CHUNKS, int TILES, typename V>
__device__ __forceinline__ void attend_step(float scale2, float (&s)[Step<T>::kTokens / 4], const V& vv, int seen,
                                            int stored, int g, State<TILES>& st) {
  constexpr int N = Step<T>::kTokens, E = N / 4;
  constexpr bool HALF = __is_same(T, _Float16);
  constexpr float HEAD = HALF ? 12.0f : 0.0f, HIGH = HALF ? 15.0f : 8.0f, LOW = HALF ? 0.0f : -INFINITY;
  // What m may fall by in a step, and up to which sum: none gets past 2^94 times the largest value.
  constexpr float FALL = 30.0f, LONGEST = 0x1p64f;
  if (!EMPTY || __any(seen > 0 && seen < N)) {
#pragma unroll
    for (int j = 0; j < E; ++j) s[j] = E * g + j < seen ? s[j] : -INFINITY;
  }
  float top = s[0];
#pragma unroll
  for (int j = 1; j < E; ++j) top = fmaxf(top, s[j]);
  const bool sees = !EMPTY || seen > 0;
  const float above = fmaf(top, scale2, -st.m);  // of this lane's scores
  bool moves = __any(sees && above != __builtin_amdgcn_fmed3f(above, LOW, HIGH));
  if (HALF && moves) {  // (below m have to be all four lanes of a query)
    uint64_t low = __ballot(sees && above < LOW);
    low &= low >> 32;
    moves = (low & low >> 16 & 0xffff) || __any(sees && above > HIGH);
  }
  if (moves) {
    const float row = over_groups_max(sees ? top * scale2 : -INFINITY), sum = over_groups_max(st.l);  // of the query
    float m = fmaxf(row - HEAD, st.m);
    if (HALF && sees && row < st.m && sum < LONGEST) m = fmaxf(row - 0.5f * HEAD, st.m - FALL);
    // 0 where this is the first step that the query sees
    const float f = EMPTY && m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(st.m - m);
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
  if (stored < N)
    Step<T>::template accumulate<true, CHUNKS>(vv, s, g, stored, st.o);
  else
    Step<T>::template accumulate<false, CHUNKS>(vv, s, g, stored, st.o);
}

// A workgroup handles one token, cached head, tile of up to 16 of its queries and share of its
// blocks; its waves take blocks in turn and join their states through LDS.  Reading keys and values
// bounds it: each page is read once for the tile of queries that shares it.  32 tokens of 12 heads of 64 in 32 bits
// over up to 2048 tokens each: 55 us, 244 MB at 4.4 TB/s.  One token of 8 cached heads over 64 blocks of 64 tokens:
// 8 to 9 us for 17 MB, latency: list, page, keys and values, then two joins.
template <typename T, int CHUNKS>
__global__ __launch_bounds__(kWaves * 64, attend_waves(CHUNKS * Step<T>::kPiece / 4)) void attend_kernel(AttendArgs a) {
  constexpr int PIECE = Step<T>::kPiece;
  constexpr int TILES = CHUNKS * PIECE / 4;  // of 16 values of a head
  __shared__ float sums[2][kRows][TILES * 16 + 4];
  __shared__ float tops[kWaves][kRows], totals[kWaves][kRows];
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
  const int n = filler ? 0 : a.chosen ? a.blocks : min(own + 1, a.max_blocks);
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
    if (lane < (last - first_step + deal - 1) / deal) id = chosen ? chosen[mine >> shift] : mine >> shift;
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

  // join the waves: 2 and 3 into 0 and 1, then 1 into 0
  st.l = over_groups_sum(st.l);
  if (g == 0) tops[wave][r] = st.m, totals[wave][r] = st.l;
  __syncthreads();
  float m = tops[0][r];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m = fmaxf(m, tops[w][r]);
  float l = 0.0f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) l += m > -INFINITY ? totals[w][r] * __builtin_amdgcn_exp2f(tops[w][r] - m) : 0.0f;
  const float f = m > -INFINITY ? __builtin_amdgcn_exp2f(st.m - m) : 0.0f;
#pragma unroll
  for (int c = 0; c < TILES; ++c) st.o[c] *= f;
#pragma unroll
  for (int half = kWaves / 2; half; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int c = 0; c < TILES; ++c) *reinterpret_cast<f32x4*>(&sums[wave - half][r][c * 16 + 4 * g]) = st.o[c];
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int c = 0; c < TILES; ++c) st.o[c] += *reinterpret_cast<const f32x4*>(&sums[wave][r][c * 16 + 4 * g]);
    }
    __syncthreads();
  }
  if (wave != 0 || r >= rows) return;
  if (a.splits > 1) {
    st.m = m;
    store_part(a, split, t, head, g, st, l);
    return;
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  T* o = static_cast<T*>(a.o) + t * a.o_token + head * a.o_head;
#pragma unroll
  for (int c = 0; c < TILES; ++c) {
    const int d = c * 16 + 4 * g;
    if (d >= D) continue;
    T x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (T)(st.o[c][i] * inv);
    store_n<4>(o + d, a.o_aligned, x);
  }
  if (g == 0 && a.lse)
    a.lse[(int64_t)t * a.heads + head] = log_of_sum(m, l);
}

// Joins the parts of a token's head: a workgroup for each, a quarter of the parts to a wave.  Lane s has
// the maximum and the total of part s, so that all factors are known before the first sum is needed;
// the sums are loaded without conditions (a part that is not there repeats the last with factor 0), so
// that a wave's loads are all under way at once (one after the other they took 0.75 us each).
template <typename T>
__global__ __launch_bounds__(256) void attend_join(AttendArgs a) {
  constexpr int DIMS = kMaxHeadDim / 64, AHEAD = 8;
  __shared__ float sums[3][kMaxHeadDim];
  const int64_t row = blockIdx.x, rows = (int64_t)a.tokens * a.heads;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, D = a.head_dim;
  const float* ml = a.part + a.splits * rows * D;
  float m = -INFINITY, l = 0.0f;
  if (lane < a.splits) m = ml[(lane * rows + row) * 2], l = ml[(lane * rows + row) * 2 + 1];
  float o[DIMS] = {};
  float top = m;
#pragma unroll
  for (int s = 32; s; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
  const float f = m > -INFINITY ? __builtin_amdgcn_exp2f(m - top) : 0.0f;
  l *= f;
#pragma unroll
  for (int s = 32; s; s >>= 1) l += __shfl_xor(l, s);
  for (int s0 = wave; s0 < a.splits; s0 += 4 * AHEAD) {
    float x[AHEAD][DIMS], fs[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int s = min(s0 + 4 * k, a.splits - 1);
      fs[k] = s0 + 4 * k < a.splits ? __shfl(f, s) : 0.0f;
      const float* part = a.part + (s * rows + row) * D;
#pragma unroll
      for (int i = 0; i < DIMS; ++i)
        if (i * 64 < D) x[k][i] = part[min(i * 64 + lane, D - 1)];
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
#pragma unroll
      for (int i = 0; i < DIMS; ++i)
        if (i * 64 < D) o[i] = fmaf(x[k][i], fs[k], o[i]);
  }
  if (wave > 0) {
#pragma unroll
    for (int i = 0; i < DIMS; ++i) sums[wave - 1][i * 64 + lane] = o[i];
  }
  __syncthreads();
  if (wave > 0) return;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  T* y = static_cast<T*>(a.o) + row / a.heads * a.o_token + row % a.heads * a.o_head;
#pragma unroll
  for (int i = 0; i < DIMS; ++i) {
    const int d = i * 64 + lane;
    if (d < D) y[d] = (T)((((o[i] + sums[0][d]) + sums[1][d]) + sums[2][d]) * inv);
  }
  if (lane == 0 && a.lse) a.lse[row] = log_of_sum(top, l);
}

// The same for at most kFewParts parts: a thread has four values of a row and loads all that they are made of at once.
template <typename T>
__global__ __launch_bounds__(256) void attend_join_few(AttendArgs a) {
  const int D = a.head_dim, units = D / 4;
  const int64_t rows = (int64_t)a.tokens * a.heads, at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / units;
  if (row >= rows) return;
  const int d = (int)(at - row * units) * 4;
  const float* ml = a.part + a.splits * rows * D;
  float m[kFewParts], l[kFewParts];
  f32x4 x[kFewParts];
#pragma unroll
  for (int s = 0; s < kFewParts; ++s) {  // (past the last part: that again, with factor 0)
    const int64_t part = min(s, a.splits - 1) * rows + row;
    x[s] = *reinterpret_cast<const f32x4*>(a.part + part * D + d);
    m[s] = ml[part * 2], l[s] = ml[part * 2 + 1];
  }
  __builtin_amdgcn_sched_barrier(0);
  float top = m[0];
#pragma unroll
  for (int s = 1; s < kFewParts; ++s) top = fmaxf(top, m[s]);
  f32x4 o = {0, 0, 0, 0};
  float sum = 0.0f;
#pragma unroll
  for (int s = 0; s < kFewParts; ++s) {
    const float f = s < a.splits && m[s] > -INFINITY ? __builtin_amdgcn_exp2f(m[s] - top) : 0.0f;
    sum = fmaf(l[s], f, sum);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = fmaf(x[s][i], f, o[i]);
  }
  const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
  T y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = (T)(o[i] * inv);
  store_n<4>(static_cast<T*>(a.o) + row / a.heads * a.o_token + row % a.heads * a.o_head + d, a.o_aligned, y);
  if (d == 0 && a.lse) a.lse[row] = log_of_sum(top, sum);
}

// ---------------------------------------------------------------- many tokens of a sequence

// A stage of keys and values in LDS: STAGE tokens of a page, keys as rows of a head (of a power of two of
// bytes, also where the head is shorter), values as rows of STAGE tokens.  A row's 16-byte pieces are permuted by the
// row (piece x at x ^ swap) so that the 16 rows that a wave reads one piece of lie in different banks.
constexpr int power_of_two(int n) { return n <= 1 ? 1 : 2 * power_of_two((n + 1) / 2); }
template <typename T, int CHUNKS, int STAGE>
struct Tile {
  static constexpr int kPiece = 16 / sizeof(T);
  static constexpr int kKeyPieces = power_of_two(CHUNKS) * 4, kValuePieces = STAGE / kPiece;
  static constexpr int kDims = kKeyPieces * kPiece;
  static constexpr int kBytes = STAGE * kKeyPieces * 16;  // of either
  static_assert(kDims * kValuePieces * 16 == kBytes, "both hold the same values");
  static __device__ __forceinline__ int key_swap(int row) {
    const int x = sizeof(T) == 4 ? row & 15 : (row & 3) | (row >> 3 & 3) << 2;  // see Step16::token
    return x & (kKeyPieces - 1);
  }
  static __device__ __forceinline__ int value_swap(int d) {
    return kValuePieces >= 8 ? d & (kValuePieces - 1) & 15 : d >> 1 & (kValuePieces - 1);
  }
  // Starts the copies of `tokens` tokens (at most STAGE) by all THREADS threads.
  template <int THREADS>
  static __device__ __forceinline__ void fetch(const T* k, const T* v, int tokens, int D, int P, unsigned char* lds) {
    // Pieces past a row's end, and rows past the last, stay out.  The rows that a thread copies pieces of lie
    // KR (VR) apart: mostly so far that the permutation is the same in all of them.
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    constexpr int KR = THREADS / kKeyPieces, VR = THREADS / kValuePieces;
    constexpr bool SAME = KR % (sizeof(T) == 4 ? 16 : 32) == 0;
    static_assert(VR % 16 == 0, "value_swap has a period of at most 16");
    const int row = threadIdx.x / kKeyPieces, piece = threadIdx.x % kKeyPieces;
    const int d = threadIdx.x / kValuePieces, x = (threadIdx.x % kValuePieces) ^ value_swap(d);
    const T* from_k = k + row * D;
    const T* from_v = v + d * P + x * kPiece;
    unsigned char* to = lds + wave * 1024;
    const bool whole = D == kDims && tokens == STAGE;  // nothing is left out
#pragma unroll
    for (int i = 0; i < STAGE / KR; ++i) {
      const int kx = piece ^ key_swap(SAME ? row : row + i * KR);
      if (whole || (kx * kPiece < D && row + i * KR < tokens))
        copy_to_lds(from_k + i * KR * D + kx * kPiece, to + i * THREADS * 16);
    }
#pragma unroll
    for (int i = 0; i < kDims / VR; ++i)
      if (whole || (x * kPiece < tokens && d + i * VR < D)) copy_to_lds(from_v + i * VR * P, to + kBytes + i * THREADS * 16);
  }
  static __device__ __forceinline__ const unsigned char* key(const unsigned char* lds, int row, int piece) {
    return lds + (row * kKeyPieces + (piece ^ key_swap(row))) * 16;
  }
  static __device__ __forceinline__ const unsigned char* value(const unsigned char* lds, int d, int piece) {
    return lds + kBytes + (d * kValuePieces + (piece ^ value_swap(d))) * 16;
  }
};

// Piece i of the keys and of the values of the step of tokens t0 ... of a stage (see Step::load).
template <typename T, int CHUNKS, int STAGE>
__device__ __forceinline__ typename Step<T>::Piece key_piece(const unsigned char* lds, int i, int t0, int D, int r, int g) {
  typedef Tile<T, CHUNKS, STAGE> L;
  const int x = min(i % CHUNKS * 4 + g, D / L::kPiece - 1);
  const int row = t0 + (sizeof(T) == 4 ? r : 8 * (r >> 2) + 4 * (i / CHUNKS) + (r & 3));
  return *reinterpret_cast<const typename Step<T>::Piece*>(L::key(lds, row, x));
}
template <typename T, int CHUNKS, int STAGE>
__device__ __forceinline__ typename Step<T>::Piece value_piece(const unsigned char* lds, int i, int t0, int r, int g) {
  typedef Tile<T, CHUNKS, STAGE> L;
  return *reinterpret_cast<const typename Step<T>::Piece*>(L::value(lds, i * 16 + r, t0 / L::kPiece + g));
}

// Where a query is in the list of its blocks: the one it attends to next with its page, and what follows
// it, loaded ahead so that no step waits for a list.
struct Cursor {
  int32_t t, seq, n, j;
  int32_t last;   // block that the token may see
  int32_t share;  // blocks share, share + splits, ... are this workgroup's (splits: a power of two)
  int32_t id, page, next_id, next_page, after;
  // The next entry of the list that is this share's; -1 past its end.  Negative entries count for nothing, the
  // others ascend: nothing follows the last block or one past it (what -1 fill the end of a list is not read).
  __device__ __forceinline__ int32_t following(const AttendArgs& a, int h) {
    if (!a.chosen) {
      const int32_t b = j++ * a.splits + share;
      return b < n ? b : -1;
    }
    const int32_t* list = a.chosen + ((int64_t)t * a.kv_heads + h) * a.blocks;
    while (j < n) {
      const int32_t b = list[j++];
      if (b >= last) j = n;
      if (b >= 0 && (b & (a.splits - 1)) == share) return b;
    }
    return -1;
  }
  __device__ __forceinline__ bool valid(int32_t b) const { return b >= 0 && b <= last; }
  __device__ __forceinline__ int32_t page_of(const AttendArgs& a, int32_t b) const {
    return valid(b) ? a.table[(int64_t)seq * a.max_blocks + b] : -1;
  }
  __device__ __forceinline__ void start(const AttendArgs& a, int h) {
    j = 0;
    id = following(a, h), next_id = following(a, h), after = following(a, h);
    page = page_of(a, id), next_page = page_of(a, next_id);
  }
  __device__ __forceinline__ void advance(const AttendArgs& a, int h) {
    id = next_id, page = next_page;
    next_id = after, next_page = page_of(a, after);
    after = following(a, h);
  }
};

// Attention of many tokens of a sequence.  A wave has a tile of 16 queries, 16 / group neighbouring tokens of one
// cached head; the WAVES waves of a workgroup, neighbouring tokens again, walk the union of their lists, block
// by block in ascending order, through LDS: a block is read from L2 once for all of them, the next one while
// they compute.  Waves whose tokens did not choose a block skip it; rows of a tile that did not are masked.
// The union is found on the way, a block ahead: each token offers its lowest block not yet passed.
//   2048 tokens of 32 queries on 8 cached heads of 128 in 16 bits, 16 blocks of 64 each: 145 us, 34 GFLOP at 232 TFLOP/s
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

  // A block's key: the run of tokens of one sequence within the workgroup's, then the block.
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
  at.t = t, at.seq = seq, at.last = min(p / a.block, a.max_blocks - 1), at.share = split;
  at.n = filler ? 0 : a.chosen ? a.blocks : at.last + 1;
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

  const float l = over_groups_sum(st.l);
  if (!row) return;
  if (a.splits > 1) {
    store_part(a, split, t, head, g, st, l);
    return;
  }
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
  T* o = static_cast<T*>(a.o) + t * a.o_token + head * a.o_head;
#pragma unroll
  for (int c = 0; c < TILES; ++c) {
    const int d = c * 16 + 4 * g;
    if (d >= D) continue;
    T x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (T)(st.o[c][i] * inv);
    store_n<4>(o + d, a.o_aligned, x);
  }
  if (g == 0 && a.lse)
    a.lse[(int64_t)t * a.heads + head] = log_of_sum(st.m, l);
}

template <typename T>
hipError_t join(const AttendArgs& a, const AttendShape& shape, hipStream_t stream) {
  if (a.splits > 1 && a.splits <= kFewParts)
    attend_join_few<T><<<(unsigned)shape.join_groups, 256, 0, stream>>>(a);
  else if (a.splits > 1)
    attend_join<T><<<(unsigned)shape.join_groups, 256, 0, stream>>>(a);
  return hipGetLastError();
}

template <typename T, int CHUNKS>
hipError_t start(const AttendArgs& a, const AttendShape& shape, hipStream_t stream) {
  if (a.tile_tokens > 0) {
    constexpr int LONG = power_of_two(CHUNKS) * 64;  // bytes of a head's row in LDS; 16 KiB of keys to a stage at most
    constexpr int STAGE = LONG <= 256 ? 64 : 16384 / LONG;
    attend_tiles<T, CHUNKS, STAGE, kTileWaves><<<(unsigned)shape.groups, shape.threads, 0, stream>>>(a);
  } else {
    attend_kernel<T, CHUNKS><<<(unsigned)shape.groups, shape.threads, 0, stream>>>(a);
  }
  const hipError_t e = hipGetLastError();
  return e != hipSuccess ? e : join<T>(a, shape, stream);
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

}  // namespace

hipError_t launch_attend(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& q,
                         const sdnn_heads& o, const int32_t* chosen, int32_t blocks, float scale,
                         float* lse, float* workspace, hipStream_t stream) {
  AttendArgs a = {};
  a.q = q.data, a.q_token = q.token_stride, a.q_head = q.head_stride;
  a.o = o.data, a.o_token = o.token_stride, a.o_head = o.head_stride;
  a.k_pages = c.k_pages, a.v_pages = c.v_pages, a.pages = c.pages;
  a.pos = t.pos, a.seq = t.seq, a.table = t.table, a.chosen = chosen;
  a.lse = lse, a.part = workspace;
  a.tokens = t.tokens, a.sequences = t.sequences, a.max_blocks = t.max_blocks;
  a.heads = q.heads, a.kv_heads = c.kv_heads, a.group = q.heads / c.kv_heads;
  a.head_tiles = (a.group + kRows - 1) / kRows;
  a.head_dim = c.head_dim, a.block = c.block;
  const AttendShape shape = attend_shape(c, t, q.heads, chosen ? blocks : 0);
  if (!launchable(shape.groups, shape.threads) || !launchable(shape.join_groups, 256)) return hipErrorInvalidConfiguration;
  a.tile_tokens = shape.tile_tokens;
  a.blocks = blocks, a.splits = shape.splits;
  // (a scale of 0 makes all scores equal: so does one that is too small to part them)
  a.scale2 = fmaxf(fabsf(scale), 1e-30f) * 1.44269504f;
  a.negate = scale < 0.0f;
  const int e = dtype_bytes(c.dtype), piece = 16 / e;
  a.q_aligned = (uintptr_t)q.data % 16 == 0 && q.token_stride % piece == 0 && q.head_stride % piece == 0;
  a.o_aligned = (uintptr_t)o.data % (4 * e) == 0 && o.token_stride % 4 == 0 && o.head_stride % 4 == 0;
  if (c.dtype == SDNN_F32) return start_dim<float>(a, shape, stream);
  if (c.dtype == SDNN_F16) return start_dim<_Float16>(a, shape, stream);
  return start_dim<__bf16>(a, shape, stream);
}

}  // namespace sdnn
