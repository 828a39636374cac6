// Rotary positions, and the call that stores a step's keys and values in the cache.
#include <type_traits>

#include "sdnn_decode_device.h"

namespace sdnn {
namespace {

constexpr int kThreads = 256;

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

// A workgroup rotates all heads of `tile` tokens.  The work is moving bytes: each value is read
// and written once.  The cosines and sines, 64-bit arithmetic, are computed once per token and pair
// and shared by the heads through LDS.  A thread keeps one unit of a row, VP pairs or VP values
// past the rotated part, and walks tokens and heads.
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
  const int turning = a.pairs / VP;
  const int units = turning + (a.head_dim - 2 * a.pairs) / VP;
  const int rows = kThreads / units;  // units <= head_dim <= kThreads
  const int u = threadIdx.x % units, h0 = threadIdx.x / units;
  if (h0 >= rows) return;
  for (int t = 0; t < n; ++t) {
    const T* xt = static_cast<const T*>(a.x) + (t0 + t) * a.x_token;
    T* yt = static_cast<T*>(a.y) + (t0 + t) * a.y_token;
    const bool empty =
        a.seq && (a.pos[t0 + t] < 0 || (uint32_t)a.seq[t0 + t] >= (uint32_t)a.sequences);
    if (u >= turning) {
      const int d = 2 * a.pairs + (u - turning) * VP;
      for (int h = h0; h < a.heads; h += rows) {
        T v[VP];
        load_n<VP>(xt + h * a.x_head + d, a.x_aligned, v);
        if (empty) {
#pragma unroll
          for (int i = 0; i < VP; ++i) v[i] = (T)0.0f;
        }
        store_n<VP>(yt + h * a.y_head + d, a.y_aligned, v);
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
  while (v > 1 && (pairs % v || (head_dim - 2 * pairs) % v)) v /= 2;
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
  a.tile = tokens >= 2048 ? 4 : 1;
  return a;
}

// ---------------------------------------------------------------- append

struct AppendArgs {
  RopeRows q;      // heads 0: no queries
  int32_t q_blocks;
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
};

constexpr int kWindow = 64;      // the most
constexpr int kTileBytes = 32768;
constexpr int kSumDims = 32;     // values of a head that are summed at a time

struct AppendLds {
  alignas(16) unsigned char tile[kTileBytes];  // the window's rotated keys, then its values
  float stage[128][kSumDims];                  // a full block's keys
  float part[8][kSumDims];
  float sum[kMaxHeadDim];
  int64_t page[kWindow];                       // -1: nothing to store
  int32_t pos[kWindow], seq[kWindow];
  float top;
};

// Sum of slots first, first + stride, ... below block, halves added pairwise (slot i with i +
// block / 2 first).
template <int STRIDE, int BLOCK, typename GET>
__device__ __forceinline__ float halves(int first, const GET& get) {
  if constexpr (STRIDE == BLOCK)
    return get(first);
  else
    return halves<STRIDE * 2, BLOCK>(first, get) + halves<STRIDE * 2, BLOCK>(first + STRIDE, get);
}

// Value d of the key of token t as it is stored.
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ T stored_key(const AppendArgs& a, int t, int h, int d) {
  const T* x = static_cast<const T*>(a.k) + t * a.k_token + h * a.k_head;
  if (d >= 2 * a.pairs) return x[d];
  const int i = INTERLEAVED ? d / 2 : d % a.pairs;
  const bool second = INTERLEAVED ? d & 1 : d >= a.pairs;
  const float2 f = rotation_of(a.freq, a.amplitude, a.pos[t], i);
  float y0, y1;
  rotate((float)x[INTERLEAVED ? 2 * i : i], (float)x[INTERLEAVED ? 2 * i + 1 : i + a.pairs], f, &y0, &y1);
  return (T)(second ? y1 : y0);
}

// The mean of the block that token i of the window fills.  Its keys come from the window's tile,
// from the call's earlier tokens (rotated again: another workgroup stores them at this moment) or
// from the page, where an earlier call stored them.
template <typename T, bool INTERLEAVED>
__device__ void block_mean(const AppendArgs& a, AppendLds& l, int t0, int i, int h) {
  const int P = a.block, D = a.head_dim, t = t0 + i;
  const int32_t pos = l.pos[i], seq = l.seq[i];
  const T* tile = reinterpret_cast<const T*>(l.tile);
  const T* page = static_cast<const T*>(a.k_pages) + (l.page[i] * a.kv_heads + h) * (int64_t)P * D;
  for (int d0 = 0; d0 < D; d0 += kSumDims) {
    __syncthreads();
    const int dn = min(kSumDims, D - d0);
    for (int j = threadIdx.x; j < P * kSumDims; j += kThreads) {
      const int s = j / kSumDims, d = j % kSumDims;
      if (d >= dn) continue;
      const int back = P - 1 - s;  // tokens before the one that fills the block
      const int from = t - back;
      T v;
      if (i >= back && l.seq[i - back] == seq && l.pos[i - back] == pos - back)
        v = tile[(i - back) * D + d0 + d];
      else if (from >= 0 && a.seq[from] == seq && a.pos[from] == pos - back)
        v = stored_key<T, INTERLEAVED>(a, from, h, d0 + d);
      else
        v = page[(int64_t)s * D + d0 + d];
      l.stage[s][d] = (float)v;
    }
    __syncthreads();
    const int d = threadIdx.x % kSumDims, u = threadIdx.x / kSumDims;  // 8 parts of each value
    const auto get = [&](int s) { return l.stage[s][d]; };
    const float part = P == 32 ? halves<8, 32>(u, get) : P == 64 ? halves<8, 64>(u, get) : halves<8, 128>(u, get);
    l.part[u][d] = part;
    __syncthreads();
    if (u == 0 && d < dn)
      l.sum[d0 + d] = ((l.part[0][d] + l.part[4][d]) + (l.part[2][d] + l.part[6][d])) +
                      ((l.part[1][d] + l.part[5][d]) + (l.part[3][d] + l.part[7][d]));
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
  const int64_t row = l.page[i] * a.kv_heads + h;
  for (int d = threadIdx.x; d < D; d += kThreads)
    a.means[row * D + d] = (int8_t)fminf(fmaxf(rintf(l.sum[d] * f), -127.0f), 127.0f);
  if (threadIdx.x == 0) a.mean_scales[row] = top / (127.0f * P);
  __syncthreads();
}

// Workgroups below q_blocks rotate queries; the others each store one head of a window of tokens:
// keys rotated into an LDS tile and written as rows, values turned through LDS so that the tokens
// of a page lie side by side, and the mean of each block that the window fills.  One launch,
// no workgroup waits for another.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  __shared__ AppendLds l;
  if ((int)blockIdx.x < a.q_blocks) {
    rope_rows_vec<T, INTERLEAVED>(a.q, blockIdx.x, reinterpret_cast<float2*>(l.tile));
    return;
  }
  const int b = blockIdx.x - a.q_blocks;
  const int h = b % a.kv_heads, t0 = b / a.kv_heads * a.window;
  const int n = min(a.window, a.tokens - t0);
  const int P = a.block, D = a.head_dim;
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int32_t p = a.pos[t0 + i], s = a.seq[t0 + i];
    int64_t page = -1;
    if (p >= 0 && (uint32_t)s < (uint32_t)a.sequences && p / P < a.max_blocks)
      page = a.table[(int64_t)s * a.max_blocks + p / P];
    if (page < 0 || page >= a.pages) page = -1;
    l.pos[i] = p, l.seq[i] = s, l.page[i] = page;
  }
  T* tile = reinterpret_cast<T*>(l.tile);
  const T* k = static_cast<const T*>(a.k) + t0 * a.k_token + h * a.k_head;
  const int units = D - a.pairs;  // pairs, then single values
  for (int j = threadIdx.x; j < n * units; j += kThreads) {
    const int i = j / units, u = j - i * units;
    const T* x = k + i * a.k_token;
    if (u < a.pairs) {
      const int d0 = INTERLEAVED ? 2 * u : u, d1 = INTERLEAVED ? 2 * u + 1 : u + a.pairs;
      float y0, y1;
      rotate((float)x[d0], (float)x[d1], rotation_of(a.freq, a.amplitude, a.pos[t0 + i], u), &y0, &y1);
      tile[i * D + d0] = (T)y0;
      tile[i * D + d1] = (T)y1;
    } else {
      tile[i * D + u + a.pairs] = x[u + a.pairs];
    }
  }
  __syncthreads();
  constexpr int V = 16 / sizeof(T);
  T* kp = static_cast<T*>(a.k_pages);
  const int chunks = D / V;
  for (int j = threadIdx.x; j < n * chunks; j += kThreads) {
    const int i = j / chunks, d = (j - i * chunks) * V;
    if (l.page[i] < 0) continue;
    T v[V];
    load_n<V>(tile + i * D + d, true, v);
    store_n<V>(kp + ((l.page[i] * a.kv_heads + h) * P + l.pos[i] % P) * (int64_t)D + d, true, v);
  }
  if (a.means) {
    const int i = threadIdx.x % 64;  // a window has at most 64 tokens: one to a lane, in every wave
    for (uint64_t full = __ballot(i < n && l.page[i] >= 0 && l.pos[i] % P == P - 1); full; full &= full - 1)
      block_mean<T, INTERLEAVED>(a, l, t0, __builtin_ctzll(full), h);
  }
  __syncthreads();
  const T* v = static_cast<const T*>(a.v) + t0 * a.v_token + h * a.v_head;
  for (int j = threadIdx.x; j < n * D; j += kThreads) {
    const int i = j / D, d = j - i * D;
    tile[j] = v[i * a.v_token + d];
  }
  __syncthreads();
  T* vp = static_cast<T*>(a.v_pages);
  for (int j = threadIdx.x; j < n * D; j += kThreads) {
    const int d = j / n, i = j - d * n;
    if (l.page[i] < 0) continue;
    vp[((l.page[i] * a.kv_heads + h) * D + d) * (int64_t)P + l.pos[i] % P] = tile[i * D + d];
  }
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
  RopeRows a = rope_args(x, y, dtype, tokens, head_dim, pos, &r);
  if (inverse) a.inverse = 1;
  const int blocks = (tokens + a.tile - 1) / a.tile;
  const size_t lds = (size_t)a.tile * a.pairs * sizeof(float2);
  return by_type(dtype, r.layout, [&](auto t, auto il) {
    rope_kernel<decltype(t), decltype(il)::value><<<blocks, kThreads, lds, stream>>>(a);
    return hipGetLastError();
  });
}

hipError_t launch_append(const sdnn_block_cache& c, const sdnn_tokens& t, const sdnn_heads& k,
                         const sdnn_heads& v, const sdnn_rotation* r, const sdnn_heads* q,
                         const sdnn_heads* q_out, hipStream_t stream) {
  AppendArgs a = {};
  if (q && q->heads > 0) {
    a.q = rope_args(*q, *q_out, c.dtype, t.tokens, c.head_dim, t.pos, r);
    a.q.seq = t.seq, a.q.sequences = t.sequences;
    a.q_blocks = (t.tokens + a.q.tile - 1) / a.q.tile;
  }
  a.k = k.data, a.k_token = k.token_stride, a.k_head = k.head_stride;
  a.v = v.data, a.v_token = v.token_stride, a.v_head = v.head_stride;
  a.k_pages = c.k_pages, a.v_pages = c.v_pages, a.means = c.means, a.mean_scales = c.mean_scales;
  a.pages = c.pages;
  a.pos = t.pos, a.seq = t.seq, a.table = t.table;
  a.freq = r ? r->freq : nullptr, a.amplitude = r ? r->amplitude : 1.0, a.pairs = r ? r->pairs : 0;
  a.tokens = t.tokens, a.sequences = t.sequences, a.max_blocks = t.max_blocks;
  a.kv_heads = c.kv_heads, a.head_dim = c.head_dim, a.block = c.block;
  // one token to a workgroup until they fill the device several times, then windows whose values
  // are written in runs
  a.window = 1;
  if ((int64_t)t.tokens * c.kv_heads > 4096)
    a.window = kWindow * c.head_dim * dtype_bytes(c.dtype) <= kTileBytes ? kWindow : kWindow / 2;
  const int64_t blocks = a.q_blocks + (int64_t)((t.tokens + a.window - 1) / a.window) * c.kv_heads;
  return by_type(c.dtype, r ? r->layout : SDNN_ROPE_HALF, [&](auto ty, auto il) {
    append_kernel<decltype(ty), decltype(il)::value><<<(unsigned)blocks, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace sdnn
