// Rotary positions, and the call that stores a step's keys and values in the cache.
#include <type_traits>

#include "sdnn_decode_device.h"
#include "sdnn_decode_shape.h"

namespace sdnn {
namespace {

constexpr int kThreads = kRopeThreads;

struct RopeRows {
  const void* x;
  void* y;
  int64_t x_token, x_head, y_token, y_head;
  const int32_t* pos;
  const int32_t* seq;  // NULL: every token has a row (sdnn_rope)
  const double* freq;
  double amplitude;
  int32_t sequences;
  int32_t tokens, heads, head_dim, pairs;
  int32_t vec;        // VP (see rope_rows)
  int32_t tile;       // tokens of a workgroup
  int32_t inverse;    // by the negative angles
  int32_t x_aligned, y_aligned;
};

// Values of a unit past the rotated part, where one of VP pairs turns: as many bytes as that takes in one access.
template <bool INTERLEAVED>
__host__ __device__ constexpr int rest_values(int vp) { return INTERLEAVED && vp > 1 ? 2 * vp : vp; }

// A workgroup rotates all heads of `tile` tokens.  The work is moving bytes: each value is read
// and written once.  The cosines and sines, 64-bit arithmetic, are computed once per token and pair
// and shared by the heads through LDS.  A thread keeps one unit of a row, VP pairs or the values
// of one access past the rotated part, and walks tokens and heads.  8192 tokens of 32 heads of 128 in 16 bits,
// half of each head rotated: 28.8 us, 134 MB at 4.66 TB/s, the rate of a large copy.  One token: 2.3 us, a launch.
template <typename T, int VP, bool INTERLEAVED>
__device__ __forceinline__ void rope_rows(const RopeRows& a, int block, float2* cs) {
  const int t0 = block * a.tile;
  const int n = min(a.tile, a.tokens - t0);
  for (int i = threadIdx.x; i < n * a.pairs; i += kThreads) {
    const int t = i / a.pairs;
    float2 f = rotation_of(a.freq, a.amplitude, a.pos[t0 + t], i - t * a.pairs);
    if (a.inverse) f.y = -f.y;
    cs[i] = f;
  }
  __syncthreads();
  constexpr int REST = rest_values<INTERLEAVED>(VP);
  const int turning = a.pairs / VP;
  const int units = turning + (a.head_dim - 2 * a.pairs) / REST;
  const int rows = kThreads / units;  // units <= head_dim <= kThreads
  const int u = threadIdx.x % units, h0 = threadIdx.x / units;
  if (h0 >= rows) return;
  for (int t = 0; t < n; ++t) {
    const T* xt = static_cast<const T*>(a.x) + (t0 + t) * a.x_token;
    T* yt = static_cast<T*>(a.y) + (t0 + t) * a.y_token;
    const bool empty =
        a.seq && (a.pos[t0 + t] < 0 || (uint32_t)a.seq[t0 + t] >= (uint32_t)a.sequences);
    if (u >= turning) {
      const int d = 2 * a.pairs + (u - turning) * REST;
      for (int h = h0; h < a.heads; h += rows) {
        T v[REST];
        load_n<REST>(xt + h * a.x_head + d, a.x_aligned, v);
        if (empty) {
#pragma unroll
          for (int i = 0; i < REST; ++i) v[i] = (T)0.0f;
        }
        store_n<REST>(yt + h * a.y_head + d, a.y_aligned, v);
      }
      continue;
    }
    float2 f[VP];
#pragma unroll
    for (int i = 0; i < VP; ++i) f[i] = empty ? make_float2(0, 0) : cs[t * a.pairs + u * VP + i];
    for (int h = h0; h < a.heads; h += rows) {
      const T* x = xt + h * a.x_head;
      T* y = yt + h * a.y_head;
      T lo[VP], hi[VP];
      if (INTERLEAVED) {
        T v[2 * VP];
        load_n<2 * VP>(x + 2 * u * VP, a.x_aligned, v);
#pragma unroll
        for (int i = 0; i < VP; ++i) lo[i] = v[2 * i], hi[i] = v[2 * i + 1];
      } else {
        load_n<VP>(x + u * VP, a.x_aligned, lo);
        load_n<VP>(x + a.pairs + u * VP, a.x_aligned, hi);
      }
#pragma unroll
      for (int i = 0; i < VP; ++i) {
        float y0, y1;
        rotate((float)lo[i], (float)hi[i], f[i], &y0, &y1);
        lo[i] = (T)(empty ? 0.0f : y0);
        hi[i] = (T)(empty ? 0.0f : y1);
      }
      if (INTERLEAVED) {
        T v[2 * VP];
#pragma unroll
        for (int i = 0; i < VP; ++i) v[2 * i] = lo[i], v[2 * i + 1] = hi[i];
        store_n<2 * VP>(y + 2 * u * VP, a.y_aligned, v);
      } else {
        store_n<VP>(y + u * VP, a.y_aligned, lo);
        store_n<VP>(y + a.pairs + u * VP, a.y_aligned, hi);
      }
    }
  }
}

template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void rope_rows_vec(const RopeRows& a, int block, float2* cs) {
  if (sizeof(T) == 2 && !INTERLEAVED && a.vec == 8)
    rope_rows<T, sizeof(T) == 2 && !INTERLEAVED ? 8 : 1, INTERLEAVED>(a, block, cs);
  else if (!(sizeof(T) == 4 && INTERLEAVED) && a.vec == 4)
    rope_rows<T, sizeof(T) == 4 && INTERLEAVED ? 1 : 4, INTERLEAVED>(a, block, cs);
  else if (a.vec == 2)
    rope_rows<T, 2, INTERLEAVED>(a, block, cs);
  else
    rope_rows<T, 1, INTERLEAVED>(a, block, cs);
}

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeRows a) {
  extern __shared__ __align__(16) unsigned char lds[];
  rope_rows_vec<T, INTERLEAVED>(a, blockIdx.x, reinterpret_cast<float2*>(lds));
}

// Pairs to a unit: as many as one 16-byte access holds (an interleaved pair is two values of it),
// fewer where a row's two parts do not divide by it.
int rope_vec(int dtype, int layout, int pairs, int head_dim) {
  int v = 16 / dtype_bytes(dtype) / (layout == SDNN_ROPE_INTERLEAVED ? 2 : 1);
  const bool il = layout == SDNN_ROPE_INTERLEAVED;
  while (v > 1 && (pairs % v || (head_dim - 2 * pairs) % (il ? rest_values<true>(v) : rest_values<false>(v)))) v /= 2;
  return v;
}

bool rows_aligned(const void* p, int64_t token_stride, int64_t head_stride, int values, int dtype) {
  return (uintptr_t)p % (values * dtype_bytes(dtype)) == 0 && token_stride % values == 0 &&
         head_stride % values == 0;
}

RopeRows rope_args(const sdnn_heads& x, const sdnn_heads& y, int dtype, int32_t tokens,
                   int32_t head_dim, const int32_t* pos, const sdnn_rotation* r) {
  RopeRows a = {};
  a.x = x.data, a.y = y.data;
  a.x_token = x.token_stride, a.x_head = x.head_stride;
  a.y_token = y.token_stride, a.y_head = y.head_stride;
  a.pos = pos;
  a.freq = r ? r->freq : nullptr, a.amplitude = r ? r->amplitude : 1.0;
  a.pairs = r ? r->pairs : 0;
  a.tokens = tokens, a.heads = x.heads, a.head_dim = head_dim;
  const int layout = r ? r->layout : SDNN_ROPE_HALF;
  a.vec = rope_vec(dtype, layout, a.pairs, head_dim);
  const int values = a.vec * (layout == SDNN_ROPE_INTERLEAVED ? 2 : 1);
  a.x_aligned = rows_aligned(x.data, x.token_stride, x.head_stride, values, dtype);
  a.y_aligned = rows_aligned(y.data, y.token_stride, y.head_stride, values, dtype);
  a.tile = rope_tile(tokens);
  return a;
}

// ---------------------------------------------------------------- append

struct AppendArgs {
  RopeRows q;      // heads 0: no queries
  int32_t kv_blocks;
  const void* k;
  const void* v;
  int64_t k_token, k_head, v_token, v_head;
  void* k_pages;
  void* v_pages;
  int8_t* means;
  float* mean_scales;
  int64_t pages;
  const int32_t* pos;
  const int32_t* seq;
  const int32_t* table;
  const double* freq;
  double amplitude;
  int32_t tokens, sequences, max_blocks;
  int32_t kv_heads, head_dim, block, pairs;
  int32_t window;  // tokens of a workgroup
  int32_t k_aligned, v_aligned;
  int32_t k_whole;  // keys can be read and rotated 16 bytes at a time
  int32_t k_pairs;  // or, where pairs are neighbours, a pair at a time
  int32_t before;   // bytes of LDS before the rows of a block's keys that lie before the window
  int32_t passes;   // of a mean, each with a part of those rows
};

// The window's rotated keys [token][head_dim], its values with rows a piece longer (so that the rows of one
// column lie in different banks), whose place the sums of a mean take afterwards.
struct AppendLds {
  int64_t page[kWindow];  // -1: nothing to store
  int32_t pos[kWindow], seq[kWindow];
  uint8_t there[128];
  float sum[kMaxHeadDim];
  float top;
};

// Sum of get(0) ... get(N - 1), halves added pairwise (i with i + N / 2 first).
template <int N, int STRIDE = 1, typename GET>
__device__ __forceinline__ float halves(const GET& get, int first = 0) {
  if constexpr (STRIDE == N)
    return get(first);
  else
    return halves<N, STRIDE * 2>(get, first) + halves<N, STRIDE * 2>(get, first + STRIDE);
}

// Rotates n keys into rows of LDS: key i, at position pos_of(i), from x_of(i) to y_of(i); those without a row (NULL)
// are left out.  VP: pairs (and values past the rotated part) of a thread's unit, as in rope_rows.
template <typename T, bool INTERLEAVED, int VP, typename X, typename Y, typename POS>
__device__ __forceinline__ void rotate_keys(const AppendArgs& a, int n, bool aligned, const X& x_of, const Y& y_of,
                                            const POS& pos_of) {
  constexpr int REST = rest_values<INTERLEAVED>(VP);
  const int D = a.head_dim, turning = a.pairs / VP, units = turning + (D - 2 * a.pairs) / REST;
#pragma unroll 2
  for (int j = threadIdx.x; j < n * units; j += kThreads) {
    const int i = j / units, u = j - i * units;
    T* y = y_of(i);
    if (!y) continue;
    const T* x = x_of(i);
    if (u >= turning) {
      const int d = 2 * a.pairs + (u - turning) * REST;
      T w[REST];
      load_n<REST>(x + d, aligned, w);
      store_n<REST>(y + d, VP > 1, w);
      continue;
    }
    T lo[VP], hi[VP];
    if (INTERLEAVED) {
      T w[2 * VP];
      load_n<2 * VP>(x + 2 * u * VP, aligned, w);
#pragma unroll
      for (int e = 0; e < VP; ++e) lo[e] = w[2 * e], hi[e] = w[2 * e + 1];
    } else {
      load_n<VP>(x + u * VP, aligned, lo);
      load_n<VP>(x + a.pairs + u * VP, aligned, hi);
    }
    const int32_t p = pos_of(i);
#pragma unroll
    for (int e = 0; e < VP; ++e) {
      float y0, y1;
      rotate((float)lo[e], (float)hi[e], rotation_of(a.freq, a.amplitude, p, u * VP + e), &y0, &y1);
      lo[e] = (T)y0, hi[e] = (T)y1;
    }
    if (INTERLEAVED) {
      T w[2 * VP];
#pragma unroll
      for (int e = 0; e < VP; ++e) w[2 * e] = lo[e], w[2 * e + 1] = hi[e];
      store_n<2 * VP>(y + 2 * u * VP, VP > 1, w);
    } else {
      store_n<VP>(y + u * VP, VP > 1, lo);
      store_n<VP>(y + a.pairs + u * VP, VP > 1, hi);
    }
  }
}

// The mean of the block that token i of the window fills.  Its keys come from the window's tile, from the
// call's tokens before the window (rotated again into `before`, since another workgroup stores them at this
// moment; `earlier`: the token before the window may be one) or from the page, where an earlier call stored
// them.  A thread adds keys q, q + P/8, ... of 16 bytes of a row, all loads under way together, and the P/8 sums
// are added from LDS.
template <typename T, bool INTERLEAVED>
__device__ void block_mean(const AppendArgs& a, AppendLds& l, const T* tile, T* before, float* sums, int t0, int i, int h,
                           bool earlier) {
  constexpr int V = 16 / sizeof(T), WIDE = V / (INTERLEAVED ? 2 : 1);
  const int P = a.block, D = a.head_dim, parts = P / kSumRows, chunks = D / V;
  const int32_t pos = l.pos[i], seq = l.seq[i];
  const int64_t row = l.page[i] * a.kv_heads + h;
  const T* page = static_cast<const T*>(a.k_pages) + row * P * D;
  const int missing = earlier ? min(P - 1 - i, t0) : 0;  // tokens t0 - 1, t0 - 2, ... that may be the block's
  for (int j = threadIdx.x; j < missing; j += kThreads)
    l.there[j] = a.seq[t0 - 1 - j] == seq && a.pos[t0 - 1 - j] == pos - i - 1 - j;
  // In a pass the sums q0 ... q0 + share - 1 are made, of all keys that go into them: key s of the block has row
  // place(s) of `before`.
  const int share = parts / a.passes;
  const auto place = [&](int s) { return s / parts * share + s % share; };
  for (int q0 = 0; q0 < parts; q0 += share) {
    __syncthreads();
    if (missing > 0) {
      const T* k = static_cast<const T*>(a.k) + (t0 - 1) * a.k_token + h * a.k_head;
      const auto x_of = [&](int j) { return k - j * a.k_token; };
      const auto y_of = [&](int j) -> T* {
        const int s = P - 2 - i - j, q = s % parts;
        return l.there[j] && q >= q0 && q < q0 + share ? before + place(s) * D : nullptr;
      };
      const auto pos_of = [&](int j) { return pos - i - 1 - j; };
      if (a.k_whole)
        rotate_keys<T, INTERLEAVED, WIDE>(a, missing, true, x_of, y_of, pos_of);
      else
        rotate_keys<T, INTERLEAVED, 1>(a, missing, a.k_pairs, x_of, y_of, pos_of);
      __syncthreads();
    }
    for (int j = threadIdx.x; j < share * chunks; j += kThreads) {
      const int q = q0 + j / chunks, d = j % chunks * V;
      T x[kSumRows][V];
#pragma unroll
      for (int k = 0; k < kSumRows; ++k)  // what the page holds, where it is from this call too: replaced below
        load_n<V>(page + (int64_t)(q + k * parts) * D + d, true, x[k]);
#pragma unroll
      for (int k = 0; k < kSumRows; ++k) {
        const int s = q + k * parts, back = P - 1 - s;  // tokens before the one that fills the block
        if (back <= i) {
          if (l.seq[i - back] == seq && l.pos[i - back] == pos - back) load_n<V>(tile + (i - back) * D + d, true, x[k]);
        } else if (back - i - 1 < missing && l.there[back - i - 1]) {
          load_n<V>(before + place(s) * D + d, true, x[k]);
        }
      }
#pragma unroll
      for (int e = 0; e < V; ++e) sums[q * D + d + e] = halves<kSumRows>([&](int k) { return (float)x[k][e]; });
    }
  }
  __syncthreads();
  for (int d = threadIdx.x; d < D; d += kThreads) {
    const auto get = [&](int q) { return sums[q * D + d]; };
    l.sum[d] = parts == 4 ? halves<4>(get) : parts == 8 ? halves<8>(get) : halves<16>(get);
  }
  __syncthreads();
  if (threadIdx.x < 64) {
    float m = 0.0f;
    for (int d = threadIdx.x; d < D; d += 64) m = fmaxf(m, fabsf(l.sum[d]));
#pragma unroll
    for (int s = 32; s; s >>= 1) m = fmaxf(m, __shfl_xor(m, s));
    if (threadIdx.x == 0) l.top = m;
  }
  __syncthreads();
  const float top = l.top;
  const float f = top > 0.0f ? 127.0f * (1.0f / top) : 0.0f;
  for (int d = threadIdx.x; d < D; d += kThreads)
    a.means[row * D + d] = (int8_t)fminf(fmaxf(rintf(l.sum[d] * f), -127.0f), 127.0f);
  if (threadIdx.x == 0) a.mean_scales[row] = top / (127.0f * P);
  __syncthreads();
}

// Workgroups below kv_blocks, which take longest and start first, each store one head of a window of tokens:
// keys rotated into an LDS tile and written as rows, values turned through LDS so that the tokens of a page
// lie side by side, and the mean of each block that the window fills; the others rotate queries.  One launch, no
// workgroup waits for another.
//   4093 tokens of 32 + 8 heads of 128 in 16 bits: 35 us, 101 MB at 2.9 TB/s: the windows' steps (read, rotate, turn,
// add) follow one another in a workgroup, 4 to a compute unit (8192 tokens: 64 us, without means 52).  One token
// each of 64 sequences: 8.9 us, latency (positions, then the page, then 64-bit cosines, then the block's keys where
// a mean is due).
//   VP: pairs (and values past the rotated part) of a thread's unit, as in rope_rows.  For single tokens 1: a
// thread's cosines and sines are then all that it waits for.
template <typename T, bool INTERLEAVED, int VP>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  extern __shared__ __align__(16) unsigned char lds[];
  __shared__ AppendLds l;
  if ((int)blockIdx.x >= a.kv_blocks) {
    rope_rows_vec<T, INTERLEAVED>(a.q, blockIdx.x - a.kv_blocks, reinterpret_cast<float2*>(lds));
    return;
  }
  constexpr int V = 16 / sizeof(T);
  const int b = blockIdx.x;
  // windows begin where the first token's block does, as if it had been stored from its first position on, so that
  // in a prompt they hold whole blocks
  const int h = b % a.kv_heads;
  const int begin = b / a.kv_heads * a.window - (a.pos[0] & (a.window - 1)), t0 = max(begin, 0);
  const int n = min(begin + a.window, a.tokens) - t0;
  if (n <= 0) return;
  const int P = a.block, D = a.head_dim, chunks = D / V, stride = D + V;
  T* tile = reinterpret_cast<T*>(lds);
  T* turn = reinterpret_cast<T*>(lds + key_bytes(a.window, D, sizeof(T)));
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int32_t p = a.pos[t0 + i], s = a.seq[t0 + i];
    int64_t page = -1;
    if (p >= 0 && (uint32_t)s < (uint32_t)a.sequences && p / P < a.max_blocks)
      page = a.table[(int64_t)s * a.max_blocks + p / P];
    if (page < 0 || page >= a.pages) page = -1;
    l.pos[i] = p, l.seq[i] = s, l.page[i] = page;
  }
  const T* v = static_cast<const T*>(a.v) + t0 * a.v_token + h * a.v_head;
#pragma unroll 4
  for (int j = threadIdx.x; j < n * chunks; j += kThreads) {
    const int i = j / chunks, d = (j - i * chunks) * V;
    T x[V];
    load_n<V>(v + i * a.v_token + d, a.v_aligned, x);
    store_n<V>(turn + i * stride + d, true, x);
  }
  const T* k = static_cast<const T*>(a.k) + t0 * a.k_token + h * a.k_head;
  rotate_keys<T, INTERLEAVED, VP>(
      a, n, a.k_aligned, [&](int i) { return k + i * a.k_token; }, [&](int i) { return tile + i * D; },
      [&](int i) { return a.pos[t0 + i]; });
  __syncthreads();
  T* kp = static_cast<T*>(a.k_pages);
  for (int j = threadIdx.x; j < n * chunks; j += kThreads) {
    const int i = j / chunks, d = (j - i * chunks) * V;
    if (l.page[i] < 0) continue;
    T x[V];
    load_n<V>(tile + i * D + d, true, x);
    store_n<V>(kp + ((l.page[i] * a.kv_heads + h) * P + l.pos[i] % P) * (int64_t)D + d, true, x);
  }
  // Values: runs of V tokens whose places are 16 bytes of a row of the page are written at once.  Groups of tokens
  // begin where the first token's place says that such runs do; the tokens before make a group too.
  T* vp = static_cast<T*>(a.v_pages);
  const int lead = a.window == 1 ? 0 : (V - (l.pos[0] & (V - 1))) & (V - 1);
  const int groups = (n - lead + V - 1) / V + (lead > 0);
  for (int j = threadIdx.x; j < groups * D; j += kThreads) {
    const int q = j / D, d = j - q * D;
    const int i0 = lead > 0 ? (q == 0 ? 0 : lead + (q - 1) * V) : q * V;
    const int i1 = min(lead > 0 && q == 0 ? lead : i0 + V, n);
    T x[V];
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = turn[min(i0 + e, n - 1) * stride + d];
    const int64_t page = i0 < n ? l.page[i0] : -1;
    const int32_t p = i0 < n ? l.pos[i0] : 0;
    // (the tokens of a sequence ascend by one, so that a run's ends tell of all of it)
    if (i1 - i0 == V && page >= 0 && p % V == 0 && l.pos[i0 + V - 1] == p + V - 1 && l.seq[i0 + V - 1] == l.seq[i0]) {
      store_n<V>(vp + ((page * a.kv_heads + h) * D + d) * (int64_t)P + p % P, true, x);
      continue;
    }
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (i0 + e < i1 && l.page[i0 + e] >= 0)
        vp[((l.page[i0 + e] * a.kv_heads + h) * D + d) * (int64_t)P + l.pos[i0 + e] % P] = x[e];
  }
  if (!a.means) return;
  const int i = threadIdx.x % 64;  // a window has at most 64 tokens: one to a lane, in every wave
  uint64_t full = __ballot(i < n && l.page[i] >= 0 && l.pos[i] % P == P - 1);
  if (!full) return;
  const bool earlier = t0 > 0 && a.seq[t0 - 1] == l.seq[0] && a.pos[t0 - 1] == l.pos[0] - 1;
  __syncthreads();  // the values are written: their place is free
  T* rows = reinterpret_cast<T*>(lds + a.before);
  for (; full; full &= full - 1)
    block_mean<T, INTERLEAVED>(a, l, tile, rows, reinterpret_cast<float*>(turn), t0, __builtin_ctzll(full), h, earlier);
}

template <typename F>
hipError_t by_type(int dtype, int layout, const F& f) {
  const bool il = layout == SDNN_ROPE_INTERLEAVED;
  if (dtype == SDNN_F32) return il ? f(float(), std::true_type()) : f(float(), std::false_type());
  if (dtype == SDNN_F16) return il ? f(_Float16(), std::true_type()) : f(_Float16(), std::false_type());
  return il ? f(__bf16(), std::true_type()) : f(__bf16(), std::false_type());
}

}  // namespace

hipError_t launch_rope(const sdnn_heads& x, const sdnn_heads& y, int dtype, int32_t tokens, int32_t head_dim,
                       const int32_t* pos, const sdnn_rotation& r, bool inverse, hipStream_t stream) {
  if (!launchable(rope_groups(tokens), kThreads)) return hipErrorInvalidConfiguration;
  RopeRows a = rope_args(x, y, dtype, tokens, head_dim, pos, &r);
  if (inverse) a.inverse = 1;
  const size_t lds = (size_t)a.tile * a.pairs * sizeof(float2);
  return by_type(dtype, r.layout, [&](auto t, auto il) {
    rope_kernel<decltype(t), decltype(il)::value><<<(unsigned)rope_groups(tokens), kThreads, lds, stream>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_append(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& k,
                         const sdnn_heads& v, const sdnn_rotation* r, const sdnn_heads* q,
                         const sdnn_heads* q_out, hipStream_t stream) {
  AppendArgs a = {};
  int64_t q_blocks = 0;
  if (q && q->heads > 0) {
    a.q = rope_args(*q, *q_out, c.dtype, t.tokens, c.head_dim, t.pos, r);
    a.q.seq = t.seq, a.q.sequences = t.sequences;
    q_blocks = rope_groups(t.tokens);
  }
  a.k = k.data, a.k_token = k.token_stride, a.k_head = k.head_stride;
  a.v = v.data, a.v_token = v.token_stride, a.v_head = v.head_stride;
  a.k_pages = c.k_pages, a.v_pages = c.v_pages, a.means = c.means, a.mean_scales = c.mean_scales;
  a.pages = c.pages;
  a.pos = t.pos, a.seq = t.seq, a.table = t.table;
  a.freq = r ? r->freq : nullptr, a.amplitude = r ? r->amplitude : 1.0, a.pairs = r ? r->pairs : 0;
  a.tokens = t.tokens, a.sequences = t.sequences, a.max_blocks = t.max_blocks;
  a.kv_heads = c.kv_heads, a.head_dim = c.head_dim, a.block = c.block;
  const int size = dtype_bytes(c.dtype), layout = r ? r->layout : SDNN_ROPE_HALF;
  const AppendShape shape = append_shape(c, t);
  const int64_t blocks = shape.windows * c.kv_heads + q_blocks;
  if (!launchable(blocks, kThreads)) return hipErrorInvalidConfiguration;
  a.window = shape.window, a.before = shape.before, a.passes = shape.passes;
  // The keys' units are 16-byte ones where windows have many and the head divides by them.
  const int wide = 16 / size / (layout == SDNN_ROPE_INTERLEAVED ? 2 : 1);
  const bool whole = rope_vec(c.dtype, layout, a.pairs, c.head_dim) == wide, vec = a.window > 1 && whole;
  a.k_whole = whole && rows_aligned(k.data, k.token_stride, k.head_stride, 16 / size, c.dtype);
  a.k_pairs = layout == SDNN_ROPE_HALF || rows_aligned(k.data, k.token_stride, k.head_stride, 2, c.dtype);
  a.k_aligned = vec ? a.k_whole : a.k_pairs;
  a.v_aligned = rows_aligned(v.data, v.token_stride, v.head_stride, 16 / size, c.dtype);
  size_t lds = shape.lds;  // or the queries' cosines and sines
  if (lds < (size_t)a.q.tile * a.q.pairs * sizeof(float2)) lds = (size_t)a.q.tile * a.q.pairs * sizeof(float2);
  a.kv_blocks = (int32_t)(shape.windows * c.kv_heads);
  return by_type(c.dtype, layout, [&](auto ty, auto il) {
    typedef decltype(ty) T;
    constexpr bool IL = decltype(il)::value;
    const auto kernel = vec ? append_kernel<T, IL, 16 / (int)sizeof(T) / (IL ? 2 : 1)> : append_kernel<T, IL, 1>;
    if (lds > 65536) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
    }
    kernel<<<(unsigned)blocks, kThreads, lds, stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace sdnn
