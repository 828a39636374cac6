// Norms of heads with the rotation in the same pass, and the cache in 8 bits as it is written and read back.
#include <type_traits>

#include "sdnn_decode_device.h"
#include "sdnn_serve_shape.h"

// Every operation is rounded by itself (no fused multiply-add, no product rounded straight to 16 bits), so that results are the
// same whichever kernel computes them.
#pragma clang fp contract(off)

namespace sdnn {
namespace {

struct HeadRows {
  const void* x;
  void* y;  // NULL: rows go to the cache
  const float* weight;  // NULL: 1
  int64_t x_token, x_head, y_token, y_head;
  int32_t heads, weight_head;
  int32_t x_aligned, y_aligned;
};

struct RowArgs {
  HeadRows q, k, v;  // v: only rows that go to the cache
  const int32_t* pos;
  const int32_t* seq;  // NULL: every token has rows (sdnn_norm_rope)
  const int32_t* table;
  const double* freq;
  double amplitude, eps;
  int32_t tokens, sequences, max_blocks, head_dim, pairs, norm;
  int32_t lanes, waves;
  // the cache
  int8_t* k_codes;
  int8_t* v_codes;
  float* k_scales;
  float* v_scales;
  int64_t pages;
  int32_t kv_heads, block;
  int32_t row_groups;  // workgroups below this one do rows, the others windows of values
  int32_t v_by_rows;   // values are written (read) with the keys, not by windows
  int32_t v_vec;       // windows: v's rows can be read 16 bytes at a time
};

// The page of a token's block, -1: nothing is stored there.
__device__ __forceinline__ int32_t page_of(const RowArgs& a, int32_t p, int32_t s) {
  if (p < 0 || (uint32_t)s >= (uint32_t)a.sequences || p / a.block >= a.max_blocks) return -1;
  const int32_t page = a.table[(int64_t)s * a.max_blocks + p / a.block];
  return page >= 0 && page < a.pages ? page : -1;
}

template <typename X>
__device__ __forceinline__ X over_lanes_sum(X x, int lanes) {
  for (int s = 1; s < lanes; s *= 2) x += __shfl_xor(x, s);
  return x;
}
__device__ __forceinline__ float over_lanes_max(float x, int lanes) {
  for (int s = 1; s < lanes; s *= 2) x = fmaxf(x, __shfl_xor(x, s));
  return x;
}

// What a row is multiplied by to become numbers from -127 to 127, and its scale.  (Below 2^-100 the factor would leave the
// floats: such rows are zeros.)
__device__ __forceinline__ float code_factor(float top, float* scale) {
  const bool some = top >= 0x1p-100f;
  *scale = some ? top * (1.0f / 127.0f) : 0.0f;
  return some ? 127.0f * (1.0f / top) : 0.0f;
}
__device__ __forceinline__ int8_t code_of(float x, float f) {
  return (int8_t)fminf(fmaxf(rintf(x * f), -127.0f), 127.0f);
}

// N codes in a row: one store where N bytes are a vector's.
template <int N>
__device__ __forceinline__ void store_codes(int8_t* p, const int8_t (&c)[N]) {
  store_n<N>(p, true, c);
}

// A wave's tasks: heads of one token, 64 / lanes of them at a time; a lane has 2 VP values of a row (ITER times: long heads
// whose parts only divide by one), pairs in place, so that norm, rotation and the largest value need no more than a few
// exchanges within a row's lanes.  The token's cosines and sines are computed once, by the wave together.
//   The sum of squares is one of 64-bit products, exact for 16-bit values, and its root is rounded once: a key comes out the
// same whatever lanes its values lie in.
template <typename T, int VP, bool INTERLEAVED, bool CACHE>
__device__ __forceinline__ void token_rows(const RowArgs& a, float2* cs) {
  constexpr int ITER = VP == 1 ? 2 : 1;
  const int lane = threadIdx.x % 64, D = a.head_dim;
  const int64_t w = (int64_t)blockIdx.x * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int t = (int)(w / a.waves), part = (int)(w % a.waves);
  const bool there = t < a.tokens;
  int32_t p = 0, page = -1;
  bool filler = false;
  if (there) {
    if (a.pos) p = a.pos[t];
    if (a.seq) {
      const int32_t s = a.seq[t];
      filler = p < 0 || (uint32_t)s >= (uint32_t)a.sequences;
      if (CACHE) page = page_of(a, p, s);
    }
    for (int i = lane; i < a.pairs; i += 64) cs[i] = rotation_of(a.freq, a.amplitude, p, i);
  }
  __syncthreads();
  if (!there) return;
  const int units = D / (2 * VP), turning = a.pairs / VP;
  const int u0 = lane & (a.lanes - 1), per = 64 / a.lanes, slot = lane / a.lanes;
  // this lane's values of a row: lo at d0, hi at d1 (neighbours: even and odd ones of 2 VP from d0)
  int d0[ITER], d1[ITER];
  float2 f[ITER][VP];
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    const int u = u0 + i * 64;
    if (INTERLEAVED)
      d0[i] = u * 2 * VP, d1[i] = d0[i] + VP;
    else if (u < turning)
      d0[i] = u * VP, d1[i] = a.pairs + u * VP;
    else
      d0[i] = 2 * a.pairs + (u - turning) * 2 * VP, d1[i] = d0[i] + VP;
#pragma unroll
    for (int e = 0; e < VP; ++e)
      if (u < turning) f[i][e] = cs[u * VP + e];
  }
  const auto has = [&](int i) { return u0 + i * 64 < units; };
  const auto load = [&](const T* x, bool aligned, int i, bool paired, float (&lo)[VP], float (&hi)[VP]) {
    if (INTERLEAVED && paired) {
      T v[2 * VP];
      load_n<2 * VP>(x + d0[i], aligned, v);
#pragma unroll
      for (int e = 0; e < VP; ++e) lo[e] = (float)v[2 * e], hi[e] = (float)v[2 * e + 1];
    } else {
      T l[VP], h[VP];
      load_n<VP>(x + d0[i], aligned, l);
      load_n<VP>(x + d1[i], aligned, h);
#pragma unroll
      for (int e = 0; e < VP; ++e) lo[e] = (float)l[e], hi[e] = (float)h[e];
    }
  };
  // Heads `h` of q or k: normed, rotated, then stored.
  const auto rows = [&](const HeadRows& r, bool keys, int first) {
    const int tasks = (r.heads + per - 1) / per;
    int task = part - first % a.waves;
    if (task < 0) task += a.waves;
    if (task >= tasks) return;
    float wl[ITER][VP], wh[ITER][VP];
    const auto weights = [&](int h) {
#pragma unroll
      for (int i = 0; i < ITER; ++i)
#pragma unroll
        for (int e = 0; e < VP; ++e) {
          wl[i][e] = wh[i][e] = 1.0f;
          if (a.norm && r.weight && has(i) && h < r.heads) {
            const float* w = r.weight + (int64_t)h * r.weight_head;
            wl[i][e] = w[INTERLEAVED ? d0[i] + 2 * e : d0[i] + e];
            wh[i][e] = w[INTERLEAVED ? d0[i] + 2 * e + 1 : d1[i] + e];
          }
        }
    };
    if (r.weight_head == 0) weights(0);
    for (; task < tasks; task += a.waves) {
      const int h = task * per + slot;
      const bool row = h < r.heads;
      if (r.weight_head) weights(h);
      float lo[ITER][VP] = {}, hi[ITER][VP] = {};
      const T* x = static_cast<const T*>(r.x) + (int64_t)t * r.x_token + (int64_t)h * r.x_head;
#pragma unroll
      for (int i = 0; i < ITER; ++i)
        if (row && has(i)) load(x, r.x_aligned, i, true, lo[i], hi[i]);
      if (a.norm) {
        double s = 0.0;
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
          for (int e = 0; e < VP; ++e) {
            s = fma((double)lo[i][e], (double)lo[i][e], s);
            s = fma((double)hi[i][e], (double)hi[i][e], s);
          }
        s = over_lanes_sum(s, a.lanes);
        const float root = (float)(1.0 / sqrt(s / D + a.eps));
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
          for (int e = 0; e < VP; ++e) lo[i][e] = lo[i][e] * root * wl[i][e], hi[i][e] = hi[i][e] * root * wh[i][e];
      }
#pragma unroll
      for (int i = 0; i < ITER; ++i)
        if (u0 + i * 64 < turning) {
#pragma unroll
          for (int e = 0; e < VP; ++e) rotate(lo[i][e], hi[i][e], f[i][e], &lo[i][e], &hi[i][e]);
        }
      if (CACHE && keys) {
        float top = 0.0f, scale;
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
          for (int e = 0; e < VP; ++e) top = fmaxf(top, fmaxf(fabsf(lo[i][e]), fabsf(hi[i][e])));
        const float c = code_factor(over_lanes_max(top, a.lanes), &scale);
        if (!row || page < 0) continue;
        const int64_t at = ((int64_t)page * a.kv_heads + h) * a.block + p % a.block;
        int8_t* y = a.k_codes + at * D;
        if (u0 == 0) a.k_scales[at] = scale;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
          if (!has(i)) continue;
          int8_t n[2 * VP];
#pragma unroll
          for (int e = 0; e < VP; ++e) {
            n[INTERLEAVED ? 2 * e : e] = code_of(lo[i][e], c);
            n[INTERLEAVED ? 2 * e + 1 : VP + e] = code_of(hi[i][e], c);
          }
          if (INTERLEAVED) {
            store_codes<2 * VP>(y + d0[i], n);
          } else {
            int8_t l[VP], g[VP];
#pragma unroll
            for (int e = 0; e < VP; ++e) l[e] = n[e], g[e] = n[VP + e];
            store_codes<VP>(y + d0[i], l);
            store_codes<VP>(y + d1[i], g);
          }
        }
        continue;
      }
      if (!row) continue;
      T* y = static_cast<T*>(r.y) + (int64_t)t * r.y_token + (int64_t)h * r.y_head;
#pragma unroll
      for (int i = 0; i < ITER; ++i) {
        if (!has(i)) continue;
        if (INTERLEAVED) {
          T v[2 * VP];
#pragma unroll
          for (int e = 0; e < VP; ++e) v[2 * e] = (T)(filler ? 0.0f : lo[i][e]), v[2 * e + 1] = (T)(filler ? 0.0f : hi[i][e]);
          store_n<2 * VP>(y + d0[i], r.y_aligned, v);
        } else {
          T l[VP], g[VP];
#pragma unroll
          for (int e = 0; e < VP; ++e) l[e] = (T)(filler ? 0.0f : lo[i][e]), g[e] = (T)(filler ? 0.0f : hi[i][e]);
          store_n<VP>(y + d0[i], r.y_aligned, l);
          store_n<VP>(y + d1[i], r.y_aligned, g);
        }
      }
    }
  };
  const int q_tasks = (a.q.heads + per - 1) / per, k_tasks = (a.k.heads + per - 1) / per;
  rows(a.q, false, 0);
  rows(a.k, CACHE, q_tasks);
  if (!CACHE || !a.v_by_rows || page < 0) return;
  // Values of single tokens: a byte to each of the page's rows.
#pragma unroll
  for (int i = 0; i < ITER; ++i) d0[i] = (u0 + i * 64) * 2 * VP, d1[i] = d0[i] + VP;
  const int tasks = (a.v.heads + per - 1) / per;
  int task = part - (q_tasks + k_tasks) % a.waves;
  if (task < 0) task += a.waves;
  for (; task < tasks; task += a.waves) {
    const int h = task * per + slot;
    const bool row = h < a.v.heads;
    float lo[ITER][VP] = {}, hi[ITER][VP] = {}, top = 0.0f, scale;
    const T* x = static_cast<const T*>(a.v.x) + (int64_t)t * a.v.x_token + (int64_t)h * a.v.x_head;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
      if (row && has(i)) load(x, a.v.x_aligned, i, false, lo[i], hi[i]);
#pragma unroll
      for (int e = 0; e < VP; ++e) top = fmaxf(top, fmaxf(fabsf(lo[i][e]), fabsf(hi[i][e])));
    }
    const float c = code_factor(over_lanes_max(top, a.lanes), &scale);
    if (!row) continue;
    const int64_t head = (int64_t)page * a.kv_heads + h;
    const int place = p % a.block;
    if (u0 == 0) a.v_scales[head * a.block + place] = scale;
    int8_t* y = a.v_codes + head * D * a.block + place;
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
      if (!has(i)) continue;
#pragma unroll
      for (int e = 0; e < VP; ++e) {
        y[(int64_t)(d0[i] + e) * a.block] = code_of(lo[i][e], c);
        y[(int64_t)(d1[i] + e) * a.block] = code_of(hi[i][e], c);
      }
    }
  }
}

// The turned values of a window of tokens in LDS, [token][value], rows a bank longer than the head.
struct TurnLds {
  int32_t pos[kQ8Window], seq[kQ8Window], page[kQ8Window];
  float scale[kQ8Window];
  __align__(16) int8_t codes[kQ8Window * (kMaxHeadDim + 4)];
};

__device__ __forceinline__ void load_window(const RowArgs& a, TurnLds& l, int t0, int n) {
  for (int i = threadIdx.x; i < n; i += kRowThreads) {
    const int32_t p = a.pos[t0 + i], s = a.seq[t0 + i];
    l.pos[i] = p, l.seq[i] = s, l.page[i] = page_of(a, p, s);
  }
  __syncthreads();
}

// Four tokens by four values: x[i] has tokens 0 ... 3 of value i, y[j] values 0 ... 3 of token j, or the other way round.
__device__ __forceinline__ void turn4(const uint32_t (&x)[4], uint32_t (&y)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u);
  const uint32_t c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
  y[0] = __builtin_amdgcn_perm(c, a, 0x05040100u), y[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  y[2] = __builtin_amdgcn_perm(d, b, 0x05040100u), y[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// Groups of four tokens of a window whose places begin at a multiple of four: group q begins with token `lead` - 4 + 4 q
// (lead: of the window's first token; in a window of several sequences groups of the later ones may not, which are taken
// token by token).
struct Groups {
  int lead, count;
  __device__ __forceinline__ Groups(const TurnLds& l, int n) {
    lead = (4 - (l.pos[0] & 3)) & 3;
    if (l.pos[0] < 0) lead = 0;
    count = 1 + (max(n - lead, 0) + 3) / 4;
  }
  __device__ __forceinline__ int first(int q) const { return lead - 4 + 4 * q; }
  // The four are neighbours of one page.
  __device__ __forceinline__ bool whole(const TurnLds& l, int i, int n) const {
    if (i < 0 || i + 4 > n || l.page[i] < 0 || (l.pos[i] & 3)) return false;
    bool same = true;
#pragma unroll
    for (int j = 1; j < 4; ++j) same = same && l.seq[i + j] == l.seq[i] && l.pos[i + j] == l.pos[i] + j;
    return same;
  }
};

// Values of a prompt: a window of one head's tokens is quantised, a row to a few lanes, and turned through LDS, so that four
// tokens' numbers are one store and the window's are runs of 64 bytes of the page's rows.
template <typename T>
__device__ __forceinline__ void append_window(const RowArgs& a, TurnLds& l, int b) {
  constexpr int V = 16 / sizeof(T);
  const int h = b % a.v.heads, t0 = b / a.v.heads * kQ8Window, n = min(kQ8Window, a.tokens - t0);
  const int D = a.head_dim, stride = D + 4;
  load_window(a, l, t0, n);
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int lanes = 1 << (32 - __builtin_clz(D / V - 1)), per = 64 / lanes;  // D / V >= 2
  const int u = lane & (lanes - 1), d = u * V;
  for (int i = wave * per + lane / lanes; i < n; i += kRowWaves * per) {
    T x[V] = {};
    if (d < D)
      load_n<V>(static_cast<const T*>(a.v.x) + (t0 + i) * a.v.x_token + h * a.v.x_head + d, a.v_vec, x);
    float top = 0.0f, scale;
#pragma unroll
    for (int e = 0; e < V; ++e) top = fmaxf(top, fabsf((float)x[e]));
    const float c = code_factor(over_lanes_max(top, lanes), &scale);
    if (u == 0 && l.page[i] >= 0)
      a.v_scales[((int64_t)l.page[i] * a.kv_heads + h) * a.block + l.pos[i] % a.block] = scale;
    if (d < D) {
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) w |= (uint32_t)(uint8_t)code_of((float)x[e + j], c) << (8 * j);
        *reinterpret_cast<uint32_t*>(l.codes + i * stride + d + e) = w;
      }
    }
  }
  __syncthreads();
  const Groups groups(l, n);
  // tokens first: 16 lanes write 64 bytes of a row of the page
  for (int j = threadIdx.x; j < groups.count * (D / 4); j += kRowThreads) {
    const int q = j % groups.count, x0 = j / groups.count * 4, i = groups.first(q);
    if (groups.whole(l, i, n)) {
      uint32_t x[4], y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = *reinterpret_cast<const uint32_t*>(l.codes + (i + e) * stride + x0);
      turn4(x, y);
      int8_t* to = a.v_codes + (((int64_t)l.page[i] * a.kv_heads + h) * D + x0) * a.block + l.pos[i] % a.block;
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(to + (int64_t)e * a.block) = y[e];
      continue;
    }
    for (int k = max(i, 0); k < min(i + 4, n); ++k) {
      if (l.page[k] < 0) continue;
      int8_t* to = a.v_codes + (((int64_t)l.page[k] * a.kv_heads + h) * D + x0) * a.block + l.pos[k] % a.block;
#pragma unroll
      for (int e = 0; e < 4; ++e) to[(int64_t)e * a.block] = l.codes[k * stride + x0 + e];
    }
  }
}

template <typename T, bool INTERLEAVED, bool CACHE>
__device__ __forceinline__ void token_rows_vec(const RowArgs& a, int vec, float2* cs) {
  constexpr int WIDE = 16 / sizeof(T) / (INTERLEAVED ? 2 : 1);
  if (vec == WIDE)
    token_rows<T, WIDE, INTERLEAVED, CACHE>(a, cs);
  else if (WIDE > 4 && vec == 4)
    token_rows<T, (WIDE > 4 ? 4 : 1), INTERLEAVED, CACHE>(a, cs);
  else if (WIDE > 2 && vec == 2)
    token_rows<T, (WIDE > 2 ? 2 : 1), INTERLEAVED, CACHE>(a, cs);
  else
    token_rows<T, 1, INTERLEAVED, CACHE>(a, cs);
}

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kRowThreads) void norm_kernel(RowArgs a, int vec) {
  __shared__ float2 cs[kRowWaves][kMaxHeadDim / 2];
  token_rows_vec<T, INTERLEAVED, false>(a, vec, cs[threadIdx.x / 64]);
}

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kRowThreads) void q8_append_kernel(RowArgs a, int vec) {
  __shared__ union {
    float2 cs[kRowWaves][kMaxHeadDim / 2];
    TurnLds turn;
  } l;
  if ((int)blockIdx.x >= a.row_groups)
    append_window<T>(a, l.turn, blockIdx.x - a.row_groups);
  else
    token_rows_vec<T, INTERLEAVED, true>(a, vec, l.cs[threadIdx.x / 64]);
}

// ---------------------------------------------------------------- means

// Sum of get(0) ... get(N - 1), halves added pairwise (i with i + N / 2 first).
template <int N, int STRIDE = 1, typename GET>
__device__ __forceinline__ float halves(const GET& get, int first = 0) {
  if constexpr (STRIDE == N)
    return get(first);
  else
    return halves<N, STRIDE * 2>(get, first) + halves<N, STRIDE * 2>(get, first + STRIDE);
}

// The means of the blocks that the call's tokens fill, after all of its keys are stored.  A workgroup looks through `range`
// tokens for one head; a thread adds one value of the block's keys.
__global__ __launch_bounds__(kRowThreads) void q8_means_kernel(sdnn_q8_cache c, sdnn_tokens t, int range) {
  __shared__ float tops[kRowWaves];
  const int h = blockIdx.x % c.kv_heads, t0 = blockIdx.x / c.kv_heads * range;
  const int lane = threadIdx.x % 64, P = c.block, D = c.head_dim, d = threadIdx.x;
  int32_t page = -1;
  if (lane < range && t0 + lane < t.tokens) {
    const int32_t p = t.pos[t0 + lane], s = t.seq[t0 + lane];
    if (p >= 0 && p % P == P - 1 && (uint32_t)s < (uint32_t)t.sequences && p / P < t.max_blocks)
      page = t.table[(int64_t)s * t.max_blocks + p / P];
    if (page >= c.pages) page = -1;
  }
  for (uint64_t full = __ballot(page >= 0); full; full &= full - 1) {
    const int64_t row = (int64_t)__builtin_amdgcn_readlane(page, __builtin_ctzll(full)) * c.kv_heads + h;
    float sum = 0.0f;
    if (d < D) {
      const int8_t* k = c.k_codes + row * P * D + d;
      const float* scale = c.k_scales + row * P;
      const auto get = [&](int i) { return scale[i] * (float)k[i * D]; };
      sum = P == 32 ? halves<32>(get) : P == 64 ? halves<64>(get) : halves<128>(get);
    }
    float top = fabsf(sum);
#pragma unroll
    for (int s = 32; s; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
    if (lane == 0) tops[threadIdx.x / 64] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    __syncthreads();
    const float f = top > 0.0f ? 127.0f * (1.0f / top) : 0.0f;
    if (d < D) c.means[row * D + d] = (int8_t)fminf(fmaxf(rintf(sum * f), -127.0f), 127.0f);
    if (d == 0) c.mean_scales[row] = top / (127.0f * P);
  }
}

// ---------------------------------------------------------------- reading back

// Eight numbers times their scale, as a row's values.
template <typename T>
__device__ __forceinline__ void write8(const int8_t (&n)[8], float scale, T* y, bool aligned) {
  constexpr int V = sizeof(T) == 4 ? 4 : 8;
#pragma unroll
  for (int i = 0; i < 8; i += V) {
    T x[V];
#pragma unroll
    for (int e = 0; e < V; ++e) x[e] = (T)(scale * (float)n[i + e]);
    store_n<V>(y + i, aligned, x);
  }
}

// A token's rows, a row to `lanes` lanes of 8 values: keys, and values where they are read one by one.
template <typename T>
__device__ __forceinline__ void read_rows(const RowArgs& a) {
  const int lane = threadIdx.x % 64, D = a.head_dim;
  const int64_t w = (int64_t)blockIdx.x * kRowWaves + threadIdx.x / 64;
  const int t = (int)(w / a.waves), part = (int)(w % a.waves);
  if (t >= a.tokens) return;
  const int32_t p = a.pos[t], page = page_of(a, p, a.seq[t]);
  const int d = (lane & (a.lanes - 1)) * 8, per = 64 / a.lanes, slot = lane / a.lanes;
  if (d >= D) return;
  const int k_tasks = (a.k.heads + per - 1) / per, tasks = k_tasks + (a.v_by_rows ? (a.v.heads + per - 1) / per : 0);
  const int place = page >= 0 ? p % a.block : 0;
  for (int task = part; task < tasks; task += a.waves) {
    const bool keys = task < k_tasks;
    const HeadRows& r = keys ? a.k : a.v;
    const int h = (keys ? task : task - k_tasks) * per + slot;
    if (h >= r.heads) continue;
    int8_t n[8] = {};
    float scale = 0.0f;
    if (page >= 0) {
      const int64_t head = (int64_t)page * a.kv_heads + h;
      scale = (keys ? a.k_scales : a.v_scales)[head * a.block + place];
      if (keys) {
        load_n<8>(a.k_codes + (head * a.block + place) * D + d, true, n);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = a.v_codes[(head * D + d + e) * a.block + place];
      }
    }
    write8<T>(n, scale, static_cast<T*>(r.y) + t * r.y_token + h * r.y_head + d, r.y_aligned);
  }
}

// Values of neighbouring tokens: as append_window, the other way round.
template <typename T>
__device__ __forceinline__ void read_window(const RowArgs& a, TurnLds& l, int b) {
  const int h = b % a.v.heads, t0 = b / a.v.heads * kQ8Window, n = min(kQ8Window, a.tokens - t0);
  const int D = a.head_dim, stride = D + 4;
  load_window(a, l, t0, n);
  for (int i = threadIdx.x; i < n; i += kRowThreads)
    l.scale[i] = l.page[i] < 0 ? 0.0f : a.v_scales[((int64_t)l.page[i] * a.kv_heads + h) * a.block + l.pos[i] % a.block];
  const Groups groups(l, n);
  for (int j = threadIdx.x; j < groups.count * (D / 4); j += kRowThreads) {
    const int q = j % groups.count, x0 = j / groups.count * 4, i = groups.first(q);
    if (groups.whole(l, i, n)) {
      const int8_t* from = a.v_codes + (((int64_t)l.page[i] * a.kv_heads + h) * D + x0) * a.block + l.pos[i] % a.block;
      uint32_t x[4], y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = *reinterpret_cast<const uint32_t*>(from + (int64_t)e * a.block);
      turn4(x, y);
#pragma unroll
      for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(l.codes + (i + e) * stride + x0) = y[e];
      continue;
    }
    for (int k = max(i, 0); k < min(i + 4, n); ++k) {
      const int8_t* from = a.v_codes + (((int64_t)max(l.page[k], 0) * a.kv_heads + h) * D + x0) * a.block + (l.pos[k] & (a.block - 1));
#pragma unroll
      for (int e = 0; e < 4; ++e) l.codes[k * stride + x0 + e] = l.page[k] < 0 ? 0 : from[(int64_t)e * a.block];
    }
  }
  __syncthreads();
  for (int j = threadIdx.x; j < n * (D / 8); j += kRowThreads) {
    const int i = j / (D / 8), d = (j - i * (D / 8)) * 8;
    int8_t x[8];
    __builtin_memcpy(x, l.codes + i * stride + d, 4);
    __builtin_memcpy(x + 4, l.codes + i * stride + d + 4, 4);
    write8<T>(x, l.scale[i], static_cast<T*>(a.v.y) + (t0 + i) * a.v.y_token + h * a.v.y_head + d, a.v.y_aligned);
  }
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void q8_read_kernel(RowArgs a) {
  __shared__ TurnLds l;
  if ((int)blockIdx.x >= a.row_groups)
    read_window<T>(a, l, blockIdx.x - a.row_groups);
  else
    read_rows<T>(a);
}

// ---------------------------------------------------------------- launches

bool rows_aligned(const sdnn_heads& r, int values, int dtype) {
  return (uintptr_t)r.data % (values * dtype_bytes(dtype)) == 0 && r.token_stride % values == 0 && r.head_stride % values == 0;
}

HeadRows head_rows(const sdnn_heads& x, const sdnn_heads* y, const float* weight, int32_t weight_head, int values, int dtype) {
  HeadRows r = {};
  r.x = x.data, r.x_token = x.token_stride, r.x_head = x.head_stride, r.heads = x.heads;
  r.x_aligned = rows_aligned(x, values, dtype);
  r.weight = weight, r.weight_head = weight ? weight_head : 0;
  if (y) r.y = y->data, r.y_token = y->token_stride, r.y_head = y->head_stride, r.y_aligned = rows_aligned(*y, values, dtype);
  return r;
}

template <typename F>
hipError_t by_type(int dtype, const F& f) {
  return dtype == SDNN_F32 ? f(float()) : dtype == SDNN_F16 ? f(_Float16()) : f(__bf16());
}
template <typename F>
hipError_t by_type(int dtype, int layout, const F& f) {
  return by_type(dtype, [&](auto t) {
    return layout == SDNN_ROPE_INTERLEAVED ? f(t, std::true_type()) : f(t, std::false_type());
  });
}

void set_rotation(RowArgs& a, const sdnn_rotation* r) {
  a.freq = r ? r->freq : nullptr, a.amplitude = r ? r->amplitude : 1.0, a.pairs = r ? r->pairs : 0;
}
void set_cache(RowArgs& a, const sdnn_q8_cache& c, const sdnn_tokens& t) {
  a.pos = t.pos, a.seq = t.seq, a.table = t.table;
  a.tokens = t.tokens, a.sequences = t.sequences, a.max_blocks = t.max_blocks;
  a.head_dim = c.head_dim, a.kv_heads = c.kv_heads, a.block = c.block, a.pages = c.pages;
  a.k_codes = c.k_codes, a.v_codes = c.v_codes, a.k_scales = c.k_scales, a.v_scales = c.v_scales;
}

}  // namespace

hipError_t launch_norm(const sdnn_heads& q, const sdnn_heads& q_out, const sdnn_heads* k, const sdnn_heads* k_out, int dtype,
                       int32_t tokens, int32_t head_dim, const int32_t* pos, const sdnn_head_norm& norm,
                       const sdnn_rotation* rotation, hipStream_t stream) {
  const int layout = rotation ? rotation->layout : SDNN_ROPE_HALF, pairs = rotation ? rotation->pairs : 0;
  const int vec = row_pairs(dtype, layout, pairs, head_dim), values = layout == SDNN_ROPE_INTERLEAVED ? 2 * vec : vec;
  RowArgs a = {};
  a.q = head_rows(q, &q_out, norm.q_weight, norm.q_head_stride, values, dtype);
  if (k) a.k = head_rows(*k, k_out, norm.k_weight, norm.k_head_stride, values, dtype);
  a.pos = pairs ? pos : nullptr;
  set_rotation(a, rotation);
  a.eps = norm.eps, a.norm = 1, a.tokens = tokens, a.head_dim = head_dim;
  const RowShape s = row_shape(tokens, head_dim / (2 * vec), {a.q.heads, a.k.heads, 0});
  if (!launchable(s.groups, kRowThreads)) return hipErrorInvalidConfiguration;
  a.lanes = s.lanes, a.waves = s.waves;
  return by_type(dtype, layout, [&](auto t, auto il) {
    norm_kernel<decltype(t), decltype(il)::value><<<(unsigned)s.groups, kRowThreads, 0, stream>>>(a, vec);
    return hipGetLastError();
  });
}

hipError_t launch_q8_append(const sdnn_q8_cache& c, const sdnn_tokens& t, int dtype, const sdnn_heads& k, const sdnn_heads& v,
                            const sdnn_head_norm* norm, const sdnn_rotation* rotation, const sdnn_heads* q,
                            const sdnn_heads* q_out, hipStream_t stream) {
  const int layout = rotation ? rotation->layout : SDNN_ROPE_HALF, pairs = rotation ? rotation->pairs : 0;
  const int vec = row_pairs(dtype, layout, pairs, c.head_dim), values = layout == SDNN_ROPE_INTERLEAVED ? 2 * vec : vec;
  RowArgs a = {};
  set_cache(a, c, t);
  set_rotation(a, rotation);
  if (norm) a.norm = 1, a.eps = norm->eps;
  if (q) a.q = head_rows(*q, q_out, norm ? norm->q_weight : nullptr, norm ? norm->q_head_stride : 0, values, dtype);
  a.k = head_rows(k, nullptr, norm ? norm->k_weight : nullptr, norm ? norm->k_head_stride : 0, values, dtype);
  a.v = head_rows(v, nullptr, nullptr, 0, vec, dtype);
  a.v_vec = rows_aligned(v, 16 / dtype_bytes(dtype), dtype);
  const bool windows = by_windows(t);
  const RowShape s = row_shape(t.tokens, c.head_dim / (2 * vec), {a.q.heads, a.k.heads, windows ? 0 : a.v.heads});
  const int64_t groups = s.groups + (windows ? window_groups(t, c.kv_heads) : 0);
  if (!launchable(groups, kRowThreads) || !launchable(mean_groups(t, c.kv_heads), kRowThreads))
    return hipErrorInvalidConfiguration;
  a.lanes = s.lanes, a.waves = s.waves, a.row_groups = (int32_t)s.groups;
  a.v_by_rows = !windows;
  const hipError_t e = by_type(dtype, layout, [&](auto ty, auto il) {
    q8_append_kernel<decltype(ty), decltype(il)::value><<<(unsigned)groups, kRowThreads, 0, stream>>>(a, vec);
    return hipGetLastError();
  });
  if (e != hipSuccess || !c.means) return e;
  const int range = mean_range(t, c.kv_heads);
  q8_means_kernel<<<(unsigned)mean_groups(t, c.kv_heads), kRowThreads, 0, stream>>>(c, t, range);
  return hipGetLastError();
}

hipError_t launch_q8_read(const sdnn_q8_cache& c, const sdnn_tokens& t, int dtype, const sdnn_heads* k, const sdnn_heads* v,
                          hipStream_t stream) {
  RowArgs a = {};
  set_cache(a, c, t);
  const int values = dtype == SDNN_F32 ? 4 : 8;
  if (k) a.k = head_rows(*k, k, nullptr, 0, values, dtype);
  if (v) a.v = head_rows(*v, v, nullptr, 0, values, dtype);
  const bool windows = v && by_windows(t);
  const RowShape s = row_shape(t.tokens, c.head_dim / 8, {a.k.heads, windows ? 0 : a.v.heads, 0});
  const int64_t rows = s.tasks > 0 ? s.groups : 0, groups = rows + (windows ? window_groups(t, c.kv_heads) : 0);
  if (!launchable(groups, kRowThreads)) return hipErrorInvalidConfiguration;
  if (groups == 0) return hipSuccess;
  a.lanes = s.lanes, a.waves = s.waves, a.row_groups = (int32_t)rows;
  a.v_by_rows = !windows;
  return by_type(dtype, [&](auto ty) {
    q8_read_kernel<decltype(ty)><<<(unsigned)groups, kRowThreads, 0, stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace sdnn
