// Attention over the cache in 8 bits.
#include "sdnn_attend_device.h"
#include "sdnn_serve_shape.h"

namespace sdnn {
namespace {

struct Q8AttendArgs : AttendArgs {
  const float* k_scales;
  const float* v_scales;
};

// The numbers of keys and values are whole and below 2^8: exact in bf16, which the matrix unit takes.  Queries and
// probabilities, which have more bits than bf16, are sums of bf16 parts, each a product of its own: 3 parts hold the 24 bits
// of a float, 2 the 11 of f16 (whose exponents bf16 has all of).  Probabilities keep 16 bits where the output has 8 or 11, and
// 24 where it has 24.  The scale of a key multiplies its score, that of a value its probability, both in 32 bits.
template <typename T>
struct Parts;
template <>
struct Parts<float> {
  static constexpr int kQ = 3, kP = 3;
};
template <>
struct Parts<_Float16> {
  static constexpr int kQ = 2, kP = 2;
};
template <>
struct Parts<__bf16> {
  static constexpr int kQ = 1, kP = 2;
};

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Eight numbers as bf16: those of a 32-bit float that has no bits below bf16's, so that its upper half is taken.
__device__ __forceinline__ uint32_t widen2(int32_t w, int at) {
  const float a = (float)(int8_t)(w >> at), b = (float)(int8_t)(w >> (at + 8));
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ __forceinline__ bf16x8 widen(int32_t lo, int32_t hi) {
  const uint32_t x[4] = {widen2(lo, 0), widen2(lo, 16), widen2(hi, 0), widen2(hi, 16)};
  bf16x8 y;
  __builtin_memcpy(&y, x, sizeof(y));
  return y;
}

template <int N>
__device__ __forceinline__ void split(float x, __bf16 (&out)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    out[i] = (__bf16)x;
    x -= (float)out[i];
  }
}

// The queries' parts: piece i of a lane has values `at(i)` ... + 7 of its row.
template <typename T, int PIECES, typename AT>
__device__ __forceinline__ void load_queries(const AttendArgs& a, bool row, int t, int64_t head, const AT& at,
                                             bf16x8 (&q)[Parts<T>::kQ][PIECES]) {
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
      __bf16 part[Parts<T>::kQ];
      split((float)x[e], part);
#pragma unroll
      for (int k = 0; k < Parts<T>::kQ; ++k) q[k][i][e] = a.negate ? -part[k] : part[k];
    }
  }
}

// One step of E tokens to a lane, their scores s (without the keys' scales) given: tokens E g ... E g + E - 1 of which the
// first `seen` of the step's are within this lane's query's sight.  vs: their values' scales.  EMPTY: see attend_step.
// value(c, e): piece e (tokens E g + 8 e ...) of values 16 c + r.
template <bool EMPTY, typename T, int E, int TILES, typename V>
__device__ __forceinline__ void q8_step(float scale2, float (&s)[E], const float (&ks)[E], const float (&vs)[E], const V& value,
                                        int seen, int g, State<TILES>& st) {
  constexpr float HIGH = 8.0f;
  const bool part = __any(seen < 4 * E && (!EMPTY || seen > 0));
#pragma unroll
  for (int j = 0; j < E; ++j) s[j] *= ks[j];
  if (part) {  // (the scales of tokens out of sight may be anything)
#pragma unroll
    for (int j = 0; j < E; ++j) s[j] = E * g + j < seen ? s[j] : -INFINITY;
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
  constexpr int P = Parts<T>::kP;
  bf16x8 p[P][E / 8];
#pragma unroll
  for (int j = 0; j < E; ++j) {
    __bf16 x[P];
    float w = s[j] * vs[j];
    if (part || EMPTY) w = s[j] > 0.0f ? w : 0.0f;  // (nor may what they are to values)
    split(w, x);
#pragma unroll
    for (int k = 0; k < P; ++k) p[k][j / 8][j % 8] = x[k];
  }
#pragma unroll
  for (int c = 0; c < TILES; ++c)
#pragma unroll
    for (int e = 0; e < E / 8; ++e) {
      const bf16x8 v = value(c, e);
#pragma unroll
      for (int k = 0; k < P; ++k) st.o[c] = mfma(v, p[k][e], st.o[c]);
    }
}

// Waves of a SIMD that the registers leave room for.
constexpr int q8_waves(int pieces) { return pieces <= 4 ? 2 : 1; }

// Single tokens: as attend_kernel, with steps of N tokens, 4 N / 16 to a lane.  A lane reads 16 numbers of a key at a time
// (DIMS pieces of 64 values for the four lane groups), and of a value N / 4 tokens' numbers: each instruction takes whole runs
// of 64 bytes and more of a page.  Everything a step needs is asked for before its first product.
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
  bf16x8 q[Parts<T>::kQ][2 * DIMS];
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
            const bf16x8 y = widen(kk[x][c][2 * e], kk[x][c][2 * e + 1]);
#pragma unroll
            for (int part = 0; part < Parts<T>::kQ; ++part) acc = mfma(y, q[part][2 * c + e], acc);
          }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * x + i] = acc[i];
      }
      q8_step<false, T, E, TILES>(
          a.scale2, s, ks, vs, [&](int c, int e) { return widen(vv[c][2 * e], vv[c][2 * e + 1]); }, seen, g, st);
    }
  }
  join_waves<T>(a, lds, split_at, t, head, r < rows, st);
}

// ---------------------------------------------------------------- many tokens of a sequence

// A stage of `tokens` tokens on its way to LDS: a thread holds 16 numbers of a key's row and 16 of a value's, and some of
// the threads a scale.  They are asked for while the stage before is computed, and widened on their way into the tile, so that
// its waves find matrix operands there.
template <int CHUNKS, int STAGE>
struct Q8Stage {
  typedef Tile<__bf16, CHUNKS, STAGE> L;
  i32x4 k, v;
  float scale;
  __device__ __forceinline__ void load(const Q8AttendArgs& a, int page, int h, int t0, int tokens) {
    const int D = a.head_dim, P = a.block, i = threadIdx.x;
    const int64_t at = ((int64_t)page * a.kv_heads + h) * P;
    const int8_t* kp = static_cast<const int8_t*>(a.k_pages) + (at + t0) * D;
    const int8_t* vp = static_cast<const int8_t*>(a.v_pages) + at * D + t0;
    if (i * 16 < tokens * D) {
      k = *reinterpret_cast<const i32x4*>(kp + i * 16);
      const int per = tokens / 16, d = i / per;  // (a power of two: 2 or 4)
      v = *reinterpret_cast<const i32x4*>(vp + d * P + (i - d * per) * 16);
    }
    if (i < 2 * STAGE && i % STAGE < tokens) scale = (i < STAGE ? a.k_scales : a.v_scales)[at + t0 + i % STAGE];
  }
  __device__ __forceinline__ void store(const Q8AttendArgs& a, int tokens, unsigned char* lds, float (&scales)[2][STAGE]) const {
    const int D = a.head_dim, i = threadIdx.x;
    if (i * 16 < tokens * D) {
      const int row = i * 16 / D, x = (i * 16 - row * D) / 8;
      const int per = tokens / 16, d = i / per, y = (i - d * per) * 2;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        *reinterpret_cast<bf16x8*>(const_cast<unsigned char*>(L::key(lds, row, x + e))) = widen(k[2 * e], k[2 * e + 1]);
        *reinterpret_cast<bf16x8*>(const_cast<unsigned char*>(L::value(lds, d, y + e))) = widen(v[2 * e], v[2 * e + 1]);
      }
    }
    if (i < 2 * STAGE) scales[i / STAGE][i % STAGE] = scale;
  }
};

// As attend_tiles: a wave has a tile of 16 queries, the workgroup's waves walk the union of their lists block by block
// through LDS.
template <typename T, int CHUNKS, int STAGE, int WAVES, bool PREFIX>
__global__ __launch_bounds__(WAVES * 64, CHUNKS <= 4 && sizeof(T) == 2 ? 4 : 2) void q8_tiles(Q8AttendArgs a) {
  typedef Tile<__bf16, CHUNKS, STAGE> L;
  constexpr int TILES = CHUNKS * 2, N = 32, E = N / 4;
  constexpr int32_t END = 0x7fffffff;
  __shared__ __align__(16) unsigned char lds[2][2 * L::kBytes];
  __shared__ __align__(16) float scales[2][2][STAGE];
  __shared__ uint64_t turns[2];
  __shared__ uint64_t lowest[3];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int r = lane & 15, g = lane >> 4;
  int b = blockIdx.x;
  const int h = b % a.kv_heads;
  b /= a.kv_heads;
  const int split_at = b % a.splits;
  b /= a.splits;
  const int first = b % a.head_tiles * kRows;
  const int t0 = b / a.head_tiles * (a.tile_tokens * WAVES);
  const int rows = min(kRows, a.group - first);
  const int per_token = kRows / a.tile_tokens;
  const int t = t0 + wave * a.tile_tokens + r / per_token, qr = r % per_token;
  const bool row = t < a.tokens && qr < rows;
  const int head = h * a.group + first + qr;
  const int D = a.head_dim;
  bf16x8 q[Parts<T>::kQ][CHUNKS];
  load_queries<T, CHUNKS>(a, row, t, head, [&](int i) { return (i * 4 + g) * 8; }, q);
  State<TILES> st;
#pragma unroll
  for (int c = 0; c < TILES; ++c) st.o[c] = f32x4{0, 0, 0, 0};
  st.m = -INFINITY, st.l = 0.0f;

  static_assert(16 * WAVES <= 128, "two words of bits");
  if (wave < 2) {
    const int i = wave * 64 + lane, ti = t0 + i;
    const bool turn = !PREFIX && i > 0 && i < a.tile_tokens * WAVES && ti < a.tokens && a.seq[ti] != a.seq[ti - 1];
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
  if (PREFIX) seq = 0, p = (int32_t)min((int64_t)p, (int64_t)a.prefix * a.block - 1);
  Cursor at;
  at.t = t, at.seq = seq, at.last = min(p / a.block, a.max_blocks - 1), at.share = split_at;
  at.n = filler ? 0 : a.chosen ? a.blocks : at.last + 1;
  at.start(a, h);
  const auto key = [&] { return at.valid(at.id) ? run << 20 | at.id : END; };
  const auto offer = [&](int turn) {
    if (g == 0 && qr == 0)
      atomicMin(reinterpret_cast<unsigned long long*>(&lowest[turn]),
                (unsigned long long)(uint32_t)key() << 32 | (uint32_t)at.page);
  };
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
  Q8Stage<CHUNKS, STAGE> next_stage = {};

  int turn = 0, buffer = 0, s = 0;
  const auto next = [&] { return turn == 2 ? 0 : turn + 1; };
  offer(turn);
  __syncthreads();
  take(turn);
  offer(turn = next());
  if (block_key != END) {
    if (block_page >= 0) next_stage.load(a, block_page, h, 0, stage);
    next_stage.store(a, stage, lds[0], scales[0]);
  }
  while (block_key != END) {
    const int32_t now_seen = seen - s * stage;
    __syncthreads();  // the stage is in LDS, the other buffer is free, the offers are made
    if (++s == stages) {
      s = 0;
      take(turn);
      if (block_key != END) offer(turn = next());
    }
    const bool more = block_key != END && block_page >= 0;
    if (more) next_stage.load(a, block_page, h, s * stage, stage);
    for (int u = 0; u < stage && __any(now_seen > u); u += N) {
      float x[E], ks[E], vs[E];
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        f32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
          const bf16x8 y = key_piece<__bf16, CHUNKS, STAGE>(lds[buffer], half * CHUNKS + c, u, D, r, g);
#pragma unroll
          for (int part = 0; part < Parts<T>::kQ; ++part) acc = mfma(y, q[part][c], acc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * half + i] = acc[i];
      }
#pragma unroll
      for (int i = 0; i < E; i += 4) {
        const f32x4 y = *reinterpret_cast<const f32x4*>(&scales[buffer][0][u + E * g + i]);
        const f32x4 z = *reinterpret_cast<const f32x4*>(&scales[buffer][1][u + E * g + i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) ks[i + e] = y[e], vs[i + e] = z[e];
      }
      q8_step<true, T, E, TILES>(
          a.scale2, x, ks, vs, [&](int c, int) { return value_piece<__bf16, CHUNKS, STAGE>(lds[buffer], c, u, r, g); },
          now_seen - u, g, st);
    }
    if (more) next_stage.store(a, stage, lds[buffer ^ 1], scales[buffer ^ 1]);
    buffer ^= 1;
  }

  const float l = over_groups_sum(st.l);
  if (!row) return;
  if (a.parts > 1)
    store_part(a, split_at, t, head, g, st, l);
  else
    store_row<T>(a, t, head, g, st, st.m, l);
}

template <typename T, int DIMS, int CHUNKS>
hipError_t start(const Q8AttendArgs& a, const AttendShape& shape, hipStream_t stream) {
  if (a.tile_tokens > 0) {
    constexpr int LONG = power_of_two(CHUNKS) * 64, STAGE = LONG <= 256 ? 64 : 16384 / LONG;
    static_assert(STAGE * CHUNKS * 32 <= kTileWaves * 64 * 16, "a thread has one piece of a stage's keys");
    const auto kernel = a.prefix ? q8_tiles<T, CHUNKS, STAGE, kTileWaves, true> : q8_tiles<T, CHUNKS, STAGE, kTileWaves, false>;
    kernel<<<(unsigned)shape.groups, shape.threads, 0, stream>>>(a);
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
