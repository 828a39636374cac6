// Attention over the chosen blocks of the cache.
#include "sdnn_decode_device.h"

namespace sdnn {
namespace {

constexpr int kWaves = 4;
constexpr int kRows = 16;  // queries of a tile: the columns of one matrix instruction

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
  float scale2;           // scale * log2 e
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

  // The keys and values of a step: 2 CHUNKS pieces each.
  template <int CHUNKS>
  static __device__ __forceinline__ void load(const T* k, const T* v, int D, int P, int r, int g,
                                              V8 (&kk)[2 * CHUNKS], V8 (&vv)[2 * CHUNKS]) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) {
        const int d = (c * 4 + g) * 8;
        kk[h * CHUNKS + c] = V8{};
        if (d < D) kk[h * CHUNKS + c] = *reinterpret_cast<const V8*>(k + token(h, r) * D + d);
      }
#pragma unroll
    for (int c = 0; c < 2 * CHUNKS; ++c)
      vv[c] = *reinterpret_cast<const V8*>(v + min(c * 16 + r, D - 1) * P + 8 * g);
  }

  template <int CHUNKS>
  static __device__ __forceinline__ void scores(const V8 (&kk)[2 * CHUNKS], const V8 (&q)[CHUNKS], float (&s)[8]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) acc = mfma(kk[h * CHUNKS + c], q[c], acc);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * h + i] = acc[i];
    }
  }

  // o += p v.  p is split into two 16-bit parts, so that it counts with all the bits that the sum
  // of probabilities counts it with (one part would add an error as large as the rounding of o).
  template <int CHUNKS>
  static __device__ __forceinline__ void accumulate(V8 (&vv)[2 * CHUNKS], const float (&p)[8], int g, int seen,
                                                    f32x4 (&o)[2 * CHUNKS]) {
    V8 hi, lo;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      hi[j] = (T)p[j];
      lo[j] = (T)(p[j] - (float)hi[j]);
    }
#pragma unroll
    for (int c = 0; c < 2 * CHUNKS; ++c) {
      if (seen < kTokens) {  // past the sequence's end a page holds anything
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (8 * g + j >= seen) vv[c][j] = (T)0.0f;
      }
      o[c] = mfma(vv[c], hi, o[c]);
      o[c] = mfma(vv[c], lo, o[c]);
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
  static __device__ __forceinline__ void load(const float* k, const float* v, int D, int P, int r, int g,
                                              f32x4 (&kk)[CHUNKS], f32x4 (&vv)[CHUNKS]) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      const int d = (c * 4 + g) * 4;
      kk[c] = f32x4{0, 0, 0, 0};
      if (d < D) kk[c] = *reinterpret_cast<const f32x4*>(k + r * D + d);
    }
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
      vv[c] = *reinterpret_cast<const f32x4*>(v + min(c * 16 + r, D - 1) * P + 4 * g);
  }

  template <int CHUNKS>
  static __device__ __forceinline__ void scores(const f32x4 (&kk)[CHUNKS], const f32x4 (&q)[CHUNKS], float (&s)[4]) {
    f32x4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(kk[c][e], q[c][e], acc, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = acc[i];
  }

  template <int CHUNKS>
  static __device__ __forceinline__ void accumulate(f32x4 (&vv)[CHUNKS], const float (&p)[4], int g, int seen,
                                                    f32x4 (&o)[CHUNKS]) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
      if (seen < kTokens) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (4 * g + j >= seen) vv[c][j] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vv[c][e], p[e], o[c], 0, 0, 0);
    }
  }
};

// A wave's state: of query lane & 15 the running maximum (in units of log 2) and the lane's share of
// the total (tokens of its lane group), and the sums o[c][i] of value 16 c + 4 (lane / 16) + i.
template <int TILES>
struct State {
  f32x4 o[TILES];
  float m, l;
};

__device__ __forceinline__ float over_groups_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float over_groups_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Tokens [0, seen) of the step's are within the query's sight (seen > 0).
template <typename T, int CHUNKS, int TILES, int PIECES>
__device__ __forceinline__ void attend_step(float scale2, const typename Step<T>::Piece (&kk)[PIECES],
                                            typename Step<T>::Piece (&vv)[PIECES], int seen,
                                            const typename Step<T>::Piece (&q)[CHUNKS], int g, State<TILES>& st) {
  constexpr int N = Step<T>::kTokens, E = N / 4;
  float s[E];
  Step<T>::template scores<CHUNKS>(kk, q, s);
  float top = -INFINITY;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    s[j] = E * g + j < seen ? s[j] * scale2 : -INFINITY;
    top = fmaxf(top, s[j]);
  }
  top = over_groups_max(top);
  if (__any(top > st.m)) {
    const float m = fmaxf(st.m, top);
    const float f = __builtin_amdgcn_exp2f(st.m - m);  // 0 for the first step (m is finite)
    st.l *= f;
    st.m = m;
#pragma unroll
    for (int c = 0; c < TILES; ++c) st.o[c] *= f;
  }
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < E; ++j) {
    s[j] = __builtin_amdgcn_exp2f(s[j] - st.m);
    sum += s[j];
  }
  st.l += sum;
  Step<T>::template accumulate<CHUNKS>(vv, s, g, seen, st.o);
}

// A workgroup handles one token, cached head, tile of up to 16 of its queries and share of its
// blocks; its waves take blocks in turn and join their states through LDS.  Reading keys and values
// bounds it: each page is read once for the tile of queries that shares it.
template <typename T, int CHUNKS>
__global__ __launch_bounds__(kWaves * 64) void attend_kernel(AttendArgs a) {
  constexpr int PIECE = Step<T>::kPiece;
  constexpr int TILES = CHUNKS * PIECE / 4;  // of 16 values of a head
  __shared__ float sums[2][kRows][TILES * 16 + 4];
  __shared__ float tops[kWaves][kRows], totals[kWaves][kRows];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, r = lane & 15, g = lane >> 4;
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
  typename Step<T>::Piece q[CHUNKS];
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c) {
    const int d = (c * 4 + g) * PIECE;
    T x[PIECE] = {};
    if (r < rows && d < D)
      load_n<PIECE>(static_cast<const T*>(a.q) + t * a.q_token + head * a.q_head + d, a.q_aligned, x);
    __builtin_memcpy(&q[c], x, sizeof(x));
  }
  State<TILES> st;
#pragma unroll
  for (int c = 0; c < TILES; ++c) st.o[c] = f32x4{0, 0, 0, 0};
  st.m = -INFINITY, st.l = 0.0f;
  const int32_t p = a.pos[t], seq = a.seq[t];
  const bool filler = p < 0 || (uint32_t)seq >= (uint32_t)a.sequences;
  const int own = p / a.block;
  const int n = filler ? 0 : a.chosen ? a.blocks : min(own + 1, a.max_blocks);
  const int32_t* chosen = a.chosen ? a.chosen + ((int64_t)t * a.kv_heads + h) * a.blocks : nullptr;
  const int32_t* table = a.table + (int64_t)seq * a.max_blocks;
  // steps of all blocks, dealt to the waves of all shares in turn
  constexpr int N = Step<T>::kTokens;
  const int per_block = a.block / N;
  for (int u = split * kWaves + wave; u < n * per_block; u += a.splits * kWaves) {
    const int j = u / per_block, t0 = (u - j * per_block) * N;
    const int id = chosen ? chosen[j] : j;
    if (id < 0 || id > own || id >= a.max_blocks) continue;
    const int64_t page = table[id];
    const int seen = p - id * a.block + 1 - t0;
    if (page < 0 || page >= a.pages || seen <= 0) continue;
    const int64_t at = (page * a.kv_heads + h) * (int64_t)a.block * D;
    typename Step<T>::Piece kk[TILES], vv[TILES];
    Step<T>::template load<CHUNKS>(static_cast<const T*>(a.k_pages) + at + (int64_t)t0 * D,
                                   static_cast<const T*>(a.v_pages) + at + t0, D, a.block, r, g, kk, vv);
    attend_step<T, CHUNKS, TILES>(a.scale2, kk, vv, seen, q, g, st);
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
    const int64_t row = ((int64_t)split * a.tokens + t) * a.heads + head;
#pragma unroll
    for (int c = 0; c < TILES; ++c)
      if (c * 16 + 4 * g < D) *reinterpret_cast<f32x4*>(a.part + row * D + c * 16 + 4 * g) = st.o[c];
    if (g == 0) {
      float* ml = a.part + (int64_t)a.splits * a.tokens * a.heads * D + row * 2;
      ml[0] = m, ml[1] = l;
    }
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
    a.lse[(int64_t)t * a.heads + head] = l > 0.0f ? (m + __log2f(l)) * 0.693147181f : -INFINITY;
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
  if (lane == 0 && a.lse) a.lse[row] = l > 0.0f ? (top + __log2f(l)) * 0.693147181f : -INFINITY;
}

template <typename T, int CHUNKS>
hipError_t start(const AttendArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)((int64_t)a.tokens * a.head_tiles * a.splits * a.kv_heads);
  attend_kernel<T, CHUNKS><<<grid, kWaves * 64, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.splits == 1) return e;
  attend_join<T><<<(unsigned)((int64_t)a.tokens * a.heads), 256, 0, stream>>>(a);
  return hipGetLastError();
}

// Pieces of a lane: a head of up to 64, 128 or 256 values.
template <typename T>
hipError_t start_dim(const AttendArgs& a, hipStream_t stream) {
  constexpr int U = 16 / Step<T>::kPiece;
  if (a.head_dim <= 64) return start<T, U>(a, stream);
  if (a.head_dim <= 128) return start<T, 2 * U>(a, stream);
  return start<T, 4 * U>(a, stream);
}

}  // namespace

// Shares of a token's blocks: so many that about 1024 workgroups (4 for each compute unit) are at
// work, each wave with a step of its own at least; at most 64 (the lanes of attend_join).
int attend_splits(const sdnn_block_cache& c, int32_t tokens, int32_t heads, int32_t blocks) {
  const int64_t units = (int64_t)tokens * c.kv_heads * ((heads / c.kv_heads + kRows - 1) / kRows);
  if (units == 0) return 1;
  const int step = c.dtype == SDNN_F32 ? 16 : 32;
  const int64_t steps = (int64_t)blocks * (c.block / step);
  const int64_t wanted = (1024 + units - 1) / units, most = (steps + kWaves - 1) / kWaves;
  const int64_t s = wanted < most ? wanted : most;
  return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}

int64_t attend_floats(const sdnn_block_cache& c, int32_t tokens, int32_t heads, int32_t blocks) {
  const int s = attend_splits(c, tokens, heads, blocks);
  return s > 1 ? (int64_t)s * tokens * heads * (c.head_dim + 2) : 0;
}

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
  a.blocks = blocks, a.splits = attend_splits(c, t.tokens, q.heads, blocks);
  a.scale2 = scale * 1.44269504f;
  const int e = dtype_bytes(c.dtype), piece = 16 / e;
  a.q_aligned = (uintptr_t)q.data % 16 == 0 && q.token_stride % piece == 0 && q.head_stride % piece == 0;
  a.o_aligned = (uintptr_t)o.data % (4 * e) == 0 && o.token_stride % 4 == 0 && o.head_stride % 4 == 0;
  if (c.dtype == SDNN_F32) return start_dim<float>(a, stream);
  if (c.dtype == SDNN_F16) return start_dim<_Float16>(a, stream);
  return start_dim<__bf16>(a, stream);
}

}  // namespace sdnn
