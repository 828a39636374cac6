// Norms of heads with the rotation in the same pass, and the cache in 8 bits as it is written and read back.
#include <type_traits>

#include "sdnn_decode_device.h"
#include "sdnn_serve_shape.h"

// Every operation is rounded by itself (no fused multiply-add, no product rounded straight to 16 bits), so that results are the
// same whichever kernel computes them.
#pragma clang fp contract(off)

namespace sdnn {
namespace {

// A number in 32 bits as a row's value.  (The compiler would make one instruction of a product and its conversion to f16 even so,
// which rounds once.)
template <typename T>
__device__ __forceinline__ T value_of(float x) {
  asm("" : "+v"(x));
  return (T)x;
}

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
  double amplitude, eps, inverse_dim;
  int32_t tokens, sequences, max_blocks, head_dim, pairs, norm;
  int32_t lanes, waves, run, shares;  // see RowShape (waves) and RunShape (run, shares)
  // the cache
  int8_t* k_codes;
  int8_t* v_codes;
  float* k_scales;
  float* v_scales;
  int64_t pages;
  int32_t kv_heads, block;
  int32_t row_groups;  // workgroups below this one do rows, the others windows of values
  int32_t v_by_rows;   // values are written with the keys, not by windows
  int32_t v_vec;       // windows: v's rows can be read 16 bytes at a time
};

// The page of a token's block, -1: nothing is stored there.
__device__ __forceinline__ int32_t page_of(const RowArgs& a, int32_t p, int32_t s) {
  const int32_t b = p >> __builtin_ctz(a.block);
  if (p < 0 || (uint32_t)s >= (uint32_t)a.sequences || b >= a.max_blocks) return -1;
  const int32_t page = a.table[(int64_t)s * a.max_blocks + b];
  return page >= 0 && page < a.pages ? page : -1;
}

// x of another lane of its row of 16: quad_perm (0 to 0xff), mirrored (0x140), mirrored by halves (0x141).
template <int CTRL>
__device__ __forceinline__ float other(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ double other(double x) {
  const int64_t b = __double_as_longlong(x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, 0xf, 0xf, true);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, 0xf, 0xf, true);
  return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
// Over groups of `lanes` lanes (a power of two, uniform; every lane of the wave takes part), neighbours first.
template <typename X, typename F>
__device__ __forceinline__ X over_lanes(X x, int lanes, const F& f) {
  if (lanes >= 2) x = f(x, other<0xb1>(x));
  if (lanes >= 4) x = f(x, other<0x4e>(x));
  if (lanes >= 8) x = f(x, other<0x141>(x));
  if (lanes >= 16) x = f(x, other<0x140>(x));
  if (lanes >= 32) x = f(x, __shfl_xor(x, 16));
  if (lanes >= 64) x = f(x, __shfl_xor(x, 32));
  return x;
}
__device__ __forceinline__ double over_lanes_sum(double x, int lanes) {
  return over_lanes(x, lanes, [](double a, double b) { return a + b; });
}
// The larger of both, or NaN where one is.
__device__ __forceinline__ float max_or_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float over_lanes_max(float x, int lanes) {
  return over_lanes(x, lanes, [](float a, float b) { return max_or_nan(a, b); });
}

// What a row is multiplied by to become numbers from -127 to 127, and its scale.  (Below 2^-100 the factor would leave the
// floats: such rows are zeros.  A row whose largest magnitude is infinite or not a number has no numbers: its scale says so.)
__device__ __forceinline__ float code_factor(float top, float* scale) {
  const bool some = top >= 0x1p-100f;
  *scale = !(top < INFINITY) ? NAN : some ? top * (1.0f / 127.0f) : 0.0f;
  return some ? 127.0f * (1.0f / top) : 0.0f;
}
__device__ __forceinline__ int8_t code_of(float x, float f) {
  return (int8_t)fminf(fmaxf(rintf(x * f), -127.0f), 127.0f);
}

// One kind's rows: fields of q, k or v by a uniform choice, value by value (a reference to one of them would put the kernel's
// arguments into scratch memory).
__device__ __forceinline__ HeadRows pick(const RowArgs& a, int kind) {
  const bool q = kind == 0, k = kind == 1;
  HeadRows r;
  r.x = q ? a.q.x : k ? a.k.x : a.v.x;
  r.y = q ? a.q.y : k ? a.k.y : a.v.y;
  r.weight = q ? a.q.weight : k ? a.k.weight : a.v.weight;
  r.x_token = q ? a.q.x_token : k ? a.k.x_token : a.v.x_token;
  r.x_head = q ? a.q.x_head : k ? a.k.x_head : a.v.x_head;
  r.y_token = q ? a.q.y_token : k ? a.k.y_token : a.v.y_token;
  r.y_head = q ? a.q.y_head : k ? a.k.y_head : a.v.y_head;
  r.heads = q ? a.q.heads : k ? a.k.heads : a.v.heads;
  r.weight_head = q ? a.q.weight_head : k ? a.k.weight_head : a.v.weight_head;
  r.x_aligned = q ? a.q.x_aligned : k ? a.k.x_aligned : a.v.x_aligned;
  r.y_aligned = q ? a.q.y_aligned : k ? a.k.y_aligned : a.v.y_aligned;
  return r;
}

// 1 / sqrt(m), rounded to 32 bits.  The instruction's estimate y has 20 bits at the least; with e = 1 - m y^2 what it lacks is
// the factor 1 + e / 2 + 3/8 e^2 + ..., whose next term is below 2^-56.  (0 and infinity have the estimate's own answers.)
// A root and a division of the library, one after the other, take several times the instructions.
__device__ __forceinline__ float inverse_root(double m) {
  const double y = __builtin_amdgcn_rsq(m), e = fma(-m * y, y, 1.0);
  const double z = fma(y * e, fma(e, 0.375, 0.5), y);
  return (float)(m > 0.0 && m < INFINITY ? z : y);
}

// What a workgroup of rows holds for its run of tokens.
struct RunLds {
  float2 cs[kRowRun * kMaxHeadDim / 2];
  int32_t pos[kRowRun], page[kRowRun], filler[kRowRun];
};

// A workgroup has a run of tokens.  Their cosines and sines, 64-bit arithmetic, are computed once for all heads; an item of a
// wave is 64 / lanes heads (a task) of B tokens, loaded while the item before is worked on; a wave has neighbouring
// items, of few tasks, so that it seldom reads weights.  A lane has 2 VP values of a row (ITER
// times: long heads whose parts only divide by one), pairs in place, so that norm, rotation and the largest value need no more
// than a few exchanges within a row's lanes.
//   The work is moving bytes.  Norms of 8001 tokens of 40 heads of 128 in 16 bits with weights of each head: 42.5 us, 164 MB
// at 3.9 TB/s; of 32768 tokens 137 to 140 us, 4.8 TB/s, a large copy's rate.  With a token to a wave, which read the weights of
// every head anew: 52 us.  B = 4 where a lane has 16 values: 163 instead of 129 registers, and 169 us instead of 137.
//   The sum of squares is one of 64-bit products, exact for 16-bit values, and its root is rounded once: a key comes out the
// same whatever lanes its values lie in.  Where a row has lanes enough, lane b of a quad takes the root for token b of the batch.
template <typename T, int VP, bool INTERLEAVED, bool CACHE>
__device__ __forceinline__ void token_rows(const RowArgs& a, RunLds& l) {
  constexpr int ITER = VP == 1 ? 2 : 1, B = VP >= 8 ? 2 : 4;
  const int lane = threadIdx.x % 64, D = a.head_dim, block = blockIdx.x;
  const int t0 = (block / a.shares) * a.run, n = min(a.run, a.tokens - t0);
  const int wave = block % a.shares * kRowWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int units = D / (2 * VP), turning = a.pairs / VP;
  const int u0 = lane & (a.lanes - 1), per = 64 / a.lanes, slot = lane / a.lanes;
  // this lane's values of a row: lo at d0, hi at d1 (neighbours: even and odd ones of 2 VP from d0)
  int d0[ITER], d1[ITER];
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    const int u = u0 + i * 64;
    if (INTERLEAVED)
      d0[i] = u * 2 * VP, d1[i] = d0[i] + VP;
    else if (u < turning)
      d0[i] = u * VP, d1[i] = a.pairs + u * VP;
    else
      d0[i] = 2 * a.pairs + (u - turning) * 2 * VP, d1[i] = d0[i] + VP;
  }
  const auto has = [&](int i) { return u0 + i * 64 < units; };
  const int q_tasks = (a.q.heads + per - 1) / per, k_tasks = (a.k.heads + per - 1) / per;
  const int v_tasks = CACHE && a.v_by_rows ? (a.v.heads + per - 1) / per : 0;
  const int shift = a.run > B ? __builtin_ctz(a.run / B) : 0;  // batches of a run: a power of two
  const int items = (q_tasks + k_tasks + v_tasks) << shift, each = (items + a.shares * kRowWaves - 1) / (a.shares * kRowWaves);
  const int first = wave * each, end = min(first + each, items);
  const auto kind_of = [&](int task) { return task < q_tasks ? 0 : task < q_tasks + k_tasks ? 1 : 2; };
  const auto task_head = [&](int task, int kind) {
    return kind == 0 ? task : kind == 1 ? task - q_tasks : task - q_tasks - k_tasks;
  };
  T next[B][ITER][2 * VP];
  const auto load = [&](int item) {
    const int task = item >> shift, b0 = (item - (task << shift)) * B;
    const int kind = kind_of(task), h = task_head(task, kind) * per + slot;
    const HeadRows r = pick(a, kind);
    const T* x = static_cast<const T*>(r.x) + (t0 + b0) * r.x_token + (int64_t)h * r.x_head;
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int i = 0; i < ITER; ++i) {
#pragma unroll
        for (int e = 0; e < 2 * VP; ++e) next[b][i][e] = (T)0.0f;
        if (b0 + b >= n || h >= r.heads || !has(i)) continue;
        const T* y = x + b * r.x_token;
        if (INTERLEAVED) {
          load_n<2 * VP>(y + d0[i], r.x_aligned, next[b][i]);
        } else {
          T lo[VP], hi[VP];
          load_n<VP>(y + d0[i], r.x_aligned, lo);
          load_n<VP>(y + d1[i], r.x_aligned, hi);
#pragma unroll
          for (int e = 0; e < VP; ++e) next[b][i][e] = lo[e], next[b][i][VP + e] = hi[e];
        }
      }
  };
  if (first < end) load(first);
  if (threadIdx.x < (unsigned)n) {
    const int t = t0 + threadIdx.x;
    const int32_t p = a.pos ? a.pos[t] : 0, s = a.seq ? a.seq[t] : 0;
    l.pos[threadIdx.x] = p;
    l.filler[threadIdx.x] = a.seq && (p < 0 || (uint32_t)s >= (uint32_t)a.sequences);
    l.page[threadIdx.x] = CACHE ? page_of(a, p, s) : -1;
  }
  if (a.pairs)
    for (int i = threadIdx.x; i < n * a.pairs; i += kRowThreads) {
      const int t = i / a.pairs;
      l.cs[i] = rotation_of(a.freq, a.amplitude, a.pos[t0 + t], i - t * a.pairs);
    }
  __syncthreads();
  float w[ITER][2 * VP];  // the weights of `weighted`'s heads
  int weighted = -1;
  for (int item = first; item < end; ++item) {
    const int task = item >> shift, b0 = (item - (task << shift)) * B;
    const int kind = kind_of(task), h = task_head(task, kind) * per + slot;
    const bool queries = kind == 0, values = kind == 2;
    const HeadRows r = pick(a, kind);
    const bool row = h < r.heads;
    float x[B][ITER][2 * VP];  // pairs as they lie (neighbours), or firsts and then seconds
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int i = 0; i < ITER; ++i)
#pragma unroll
        for (int e = 0; e < 2 * VP; ++e) x[b][i][e] = (float)next[b][i][e];
    if (item + 1 < end) load(item + 1);
    if (!values) {
      if (a.norm) {
        if (task != weighted) {
          weighted = task;
#pragma unroll
          for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int e = 0; e < 2 * VP; ++e) {
              w[i][e] = 1.0f;
              if (r.weight && has(i) && row)
                w[i][e] = r.weight[(int64_t)h * r.weight_head + (INTERLEAVED || e < VP ? d0[i] + e : d1[i] + e - VP)];
            }
        }
        double s[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
          s[b] = 0.0;
#pragma unroll
          for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int e = 0; e < 2 * VP; ++e) s[b] = fma((double)x[b][i][e], (double)x[b][i][e], s[b]);
          s[b] = over_lanes_sum(s[b], a.lanes);
        }
        float root[B];
        const auto root_of = [&](double s) { return inverse_root(fma(s, a.inverse_dim, a.eps)); };
        if (a.lanes >= B) {
          double mine = s[0];
#pragma unroll
          for (int b = 1; b < B; ++b) mine = (lane & (B - 1)) == b ? s[b] : mine;
          const float r = root_of(mine);
          if constexpr (B == 2)
            root[0] = other<0xa0>(r), root[1] = other<0xf5>(r);
          else
            root[0] = other<0x00>(r), root[1] = other<0x55>(r), root[2] = other<0xaa>(r), root[3] = other<0xff>(r);
        } else {
#pragma unroll
          for (int b = 0; b < B; ++b) root[b] = root_of(s[b]);
        }
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
          for (int i = 0; i < ITER; ++i)
#pragma unroll
            for (int e = 0; e < 2 * VP; ++e) x[b][i][e] = x[b][i][e] * root[b] * w[i][e];
      }
#pragma unroll
      for (int i = 0; i < ITER; ++i) {
        const int u = u0 + i * 64;
        if (u >= turning) continue;
#pragma unroll
        for (int b = 0; b < B; ++b) {
          if (b0 + b >= n) continue;
#pragma unroll
          for (int e = 0; e < VP; ++e) {
            const float2 f = l.cs[(b0 + b) * a.pairs + u * VP + e];
            float& lo = x[b][i][INTERLEAVED ? 2 * e : e];
            float& hi = x[b][i][INTERLEAVED ? 2 * e + 1 : VP + e];
            rotate(lo, hi, f, &lo, &hi);
          }
        }
      }
    }
    if (CACHE && !queries) {
#pragma unroll
      for (int b = 0; b < B; ++b) {
        float top = 0.0f, scale;
#pragma unroll
        for (int i = 0; i < ITER; ++i)
#pragma unroll
          for (int e = 0; e < 2 * VP; ++e) top = max_or_nan(top, fabsf(x[b][i][e]));
        const float c = code_factor(over_lanes_max(top, a.lanes), &scale);
        if (b0 + b >= n || !row || l.page[b0 + b] < 0) continue;
        const int place = l.pos[b0 + b] & (a.block - 1);
        const int64_t head = (int64_t)l.page[b0 + b] * a.kv_heads + h;
        if (u0 == 0) (values ? a.v_scales : a.k_scales)[head * a.block + place] = scale;
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
          if (!has(i)) continue;
          int8_t c8[2 * VP];
#pragma unroll
          for (int e = 0; e < 2 * VP; ++e) c8[e] = code_of(x[b][i][e], c);
          if (values) {  // single tokens: a byte to each of the page's rows
            int8_t* y = a.v_codes + head * D * a.block + place;
#pragma unroll
            for (int e = 0; e < 2 * VP; ++e) y[(INTERLEAVED || e < VP ? d0[i] + e : d1[i] + e - VP) * a.block] = c8[e];
            continue;
          }
          int8_t* y = a.k_codes + (head * a.block + place) * D;
          if (INTERLEAVED) {
            store_n<2 * VP>(y + d0[i], true, c8);
          } else {
            int8_t lo[VP], hi[VP];
#pragma unroll
            for (int e = 0; e < VP; ++e) lo[e] = c8[e], hi[e] = c8[VP + e];
            store_n<VP>(y + d0[i], true, lo);
            store_n<VP>(y + d1[i], true, hi);
          }
        }
      }
      continue;
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      if (b0 + b >= n || !row) continue;
      const bool filler = l.filler[b0 + b];
      T* y = static_cast<T*>(r.y) + (t0 + b0 + b) * r.y_token + (int64_t)h * r.y_head;
#pragma unroll
      for (int i = 0; i < ITER; ++i) {
        if (!has(i)) continue;
        T v[2 * VP];
#pragma unroll
        for (int e = 0; e < 2 * VP; ++e) v[e] = value_of<T>(filler ? 0.0f : x[b][i][e]);
        if (INTERLEAVED) {
          store_n<2 * VP>(y + d0[i], r.y_aligned, v);
        } else {
          T lo[VP], hi[VP];
#pragma unroll
          for (int e = 0; e < VP; ++e) lo[e] = v[e], hi[e] = v[VP + e];
          store_n<VP>(y + d0[i], r.y_aligned, lo);
          store_n<VP>(y + d1[i], r.y_aligned, hi);
        }
      }
    }
  }
}

// The turned values of a window of tokens in LDS, [token][value], rows a bank longer than the head.
//   The tokens whose places in a page share a word of four are moved together if they are neighbours: group q has tokens
// `lead` - 4 + 4 q ... + 3 of the window (lead: of the window's first token; in a window of several sequences the later ones' may
// not fit).  group[q]: their page; -1: those that are in the window are taken one by one, from the list.
struct TurnLds {
  int32_t pos[kQ8Window], page[kQ8Window], loose[kQ8Window];
  int32_t group[kQ8Window / 4 + 1], lead, singles;
  float k_scale[kQ8Window], v_scale[kQ8Window];
  __align__(16) int8_t codes[kQ8Window * (kMaxHeadDim + 4)];
};

// PARTS: groups with fewer than four tokens in the window count as such (they can be read, but not written, by words).
template <bool PARTS>
__device__ __forceinline__ void load_window(const RowArgs& a, TurnLds& l, int t0, int n) {
  const int i = threadIdx.x;
  if (i < kQ8Window) {  // the first wave
    static_assert(kQ8Window == 64, "a wave");
    int32_t p = -1, s = -1, page = -1;
    if (i < n) p = a.pos[t0 + i], s = a.seq[t0 + i], page = page_of(a, p, s);
    l.pos[i] = p, l.page[i] = page;
    const int32_t p0 = __builtin_amdgcn_readfirstlane(p), lead = p0 < 0 ? 0 : -p0 & 3;
    const int q = (i - lead + 4) >> 2, begin = lead - 4 + 4 * q;  // this token's group and that one's first token
    // Does the token lie where its group says?  Sequences' and pages' neighbours have neighbouring lanes.
    const int from = max(begin, 0);
    const int32_t fp = __shfl(p, from), fs = __shfl(s, from), fpage = __shfl(page, from);
    const bool fits = page >= 0 && fpage == page && fs == s && p - fp == i - from && ((p - i + begin) & 3) == 0;
    const uint64_t fit = __ballot(fits), there = __ballot(i < n);
    const uint64_t mine = begin < 0 ? 15ull >> -begin : 15ull << begin;
    const bool all = (there & mine) == (fit & mine) && (there & mine), four = begin >= 0 && begin + 4 <= min(n, kQ8Window);
    const bool together = all && (PARTS || four);
    if (i == from) l.group[q] = together ? page : -1;
    if (i == 0 && lead == 0) l.group[0] = -1;  // no token is in it
    const uint64_t singles = __ballot(i < n && !together);
    if (i < n && !together) l.loose[__popcll(singles & ((1ull << i) - 1))] = i;
    if (i == 0) l.lead = lead, l.singles = __popcll(singles);
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

// What moves a window's tokens that no group has: f(token, value), the tokens dealt to the waves.
template <typename F>
__device__ __forceinline__ void each_loose(const TurnLds& l, int D, const F& f) {
  for (int k = threadIdx.x / 64; k < l.singles; k += kRowWaves)
    for (int d = threadIdx.x % 64; d < D; d += 64) f(l.loose[k], d);
}

// Values of a prompt: a window of one head's tokens is quantised, a row to a few lanes, and turned through LDS, so that four
// tokens' numbers are one store and the window's are runs of 64 bytes of the page's rows.
template <typename T>
__device__ __forceinline__ void append_window(const RowArgs& a, TurnLds& l, int b) {
  constexpr int V = 16 / sizeof(T), B = 4;
  const int h = b % a.v.heads, t0 = b / a.v.heads * kQ8Window, n = min(kQ8Window, a.tokens - t0);
  const int D = a.head_dim, stride = D + 4;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int lanes = 1 << (32 - __builtin_clz(D / V - 1)), per = 64 / lanes;  // D / V >= 2
  const int d = (lane & (lanes - 1)) * V, step = kRowWaves * per;
  for (int i0 = wave * per + lane / lanes, first = 1; first || i0 - lane / lanes < n; i0 += B * step, first = 0) {
    T x[B][V] = {};
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int i = i0 + j * step;
      if (i < n && d < D)
        load_n<V>(static_cast<const T*>(a.v.x) + (t0 + i) * a.v.x_token + h * a.v.x_head + d, a.v_vec, x[j]);
    }
    if (first) load_window<false>(a, l, t0, n);
#pragma unroll
    for (int j = 0; j < B; ++j) {
      const int i = i0 + j * step;
      float top = 0.0f, scale;
#pragma unroll
      for (int e = 0; e < V; ++e) top = max_or_nan(top, fabsf((float)x[j][e]));
      const float c = code_factor(over_lanes_max(top, lanes), &scale);
      if (i >= n || d >= D) continue;
      if (d == 0 && l.page[i] >= 0)
        a.v_scales[((int64_t)l.page[i] * a.kv_heads + h) * a.block + (l.pos[i] & (a.block - 1))] = scale;
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        uint32_t w = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) w |= (uint32_t)(uint8_t)code_of((float)x[j][e + k], c) << (8 * k);
        *reinterpret_cast<uint32_t*>(l.codes + i * stride + d + e) = w;
      }
    }
  }
  __syncthreads();
  // tokens first: 16 lanes write 64 bytes of a row of the page (group 0 has fewer than four tokens or none)
  constexpr int G = kQ8Window / 4;
  for (int j = threadIdx.x; j < G * (D / 4); j += kRowThreads) {
    const int q = 1 + j % G, x0 = j / G * 4, page = l.group[q];
    if (page < 0) continue;
    const int i = l.lead - 4 + 4 * q;
    uint32_t x[4], y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = *reinterpret_cast<const uint32_t*>(l.codes + (i + e) * stride + x0);
    turn4(x, y);
    int8_t* to = a.v_codes + (((int64_t)page * a.kv_heads + h) * D + x0) * a.block + (l.pos[i] & (a.block - 1));
#pragma unroll
    for (int e = 0; e < 4; ++e) *reinterpret_cast<uint32_t*>(to + e * a.block) = y[e];
  }
  each_loose(l, D, [&](int i, int d) {
    if (l.page[i] >= 0)
      a.v_codes[(((int64_t)l.page[i] * a.kv_heads + h) * D + d) * a.block + (l.pos[i] & (a.block - 1))] =
          l.codes[i * stride + d];
  });
}

template <typename T, bool INTERLEAVED, bool CACHE>
__device__ __forceinline__ void token_rows_vec(const RowArgs& a, int vec, RunLds& l) {
  constexpr int WIDE = 16 / sizeof(T) / (INTERLEAVED ? 2 : 1);
  if (vec == WIDE)
    token_rows<T, WIDE, INTERLEAVED, CACHE>(a, l);
  else if (WIDE > 4 && vec == 4)
    token_rows<T, (WIDE > 4 ? 4 : 1), INTERLEAVED, CACHE>(a, l);
  else if (WIDE > 2 && vec == 2)
    token_rows<T, (WIDE > 2 ? 2 : 1), INTERLEAVED, CACHE>(a, l);
  else
    token_rows<T, 1, INTERLEAVED, CACHE>(a, l);
}

template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kRowThreads) void norm_kernel(RowArgs a, int vec) {
  __shared__ RunLds l;
  token_rows_vec<T, INTERLEAVED, false>(a, vec, l);
}

// (Registers for three waves to a SIMD: with a few more, for two, 4093 tokens of 32 + 8 heads of 128 take 32 us for 29.)
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(kRowThreads, 3) void q8_append_kernel(RowArgs a, int vec) {
  __shared__ union {
    RunLds run;
    TurnLds turn;
  } l;
  if ((int)blockIdx.x >= a.row_groups)
    append_window<T>(a, l.turn, blockIdx.x - a.row_groups);
  else
    token_rows_vec<T, INTERLEAVED, true>(a, vec, l.run);
}

// ---------------------------------------------------------------- means

// Sum of get(0) ... get(N - 1), halves added pairwise (i with i + N / 2 first).
template <int N, int STRIDE, typename GET>
__device__ __forceinline__ f32x4 halves(const GET& get, int first) {
  if constexpr (STRIDE == N)
    return get(first);
  else
    return halves<N, STRIDE * 2>(get, first) + halves<N, STRIDE * 2>(get, first + STRIDE);
}

// The means of the blocks that the call's tokens fill, after all of its keys are stored.  A workgroup looks through `range`
// tokens for one head; a lane adds four values of a quarter of the block's keys, and the quarters meet in LDS.  It is the latency
// of a launch and of token, page and keys one after the other: with 8 heads of 128 in blocks of 64, 64 tokens 3.2 us, 4096 tokens
// 4.7, 32768 17 (34 MB).
__global__ __launch_bounds__(kRowThreads) void q8_means_kernel(sdnn_q8_cache c, sdnn_tokens t, int range) {
  __shared__ f32x4 part[kRowWaves][kMaxHeadDim / 4];
  static_assert(kRowWaves == 4, "quarters");
  const int h = blockIdx.x % c.kv_heads, t0 = blockIdx.x / c.kv_heads * range;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, P = c.block, D = c.head_dim;
  int32_t page = -1;
  if (lane < range && t0 + lane < t.tokens) {
    const int32_t p = t.pos[t0 + lane], s = t.seq[t0 + lane];
    if (p >= 0 && p % P == P - 1 && (uint32_t)s < (uint32_t)t.sequences && p / P < t.max_blocks)
      page = t.table[(int64_t)s * t.max_blocks + p / P];
    if (page >= c.pages) page = -1;
  }
  for (uint64_t full = __ballot(page >= 0); full; full &= full - 1) {
    const int64_t row = (int64_t)__builtin_amdgcn_readlane(page, __builtin_ctzll(full)) * c.kv_heads + h;
    if (lane < D / 4) {
      const int8_t* k = c.k_codes + row * P * D + 4 * lane;
      const float* scale = c.k_scales + row * P;
      const auto get = [&](int i) {
        typedef int8_t i8x4 __attribute__((ext_vector_type(4)));
        const i8x4 n = *reinterpret_cast<const i8x4*>(k + i * D);
        return scale[i] * f32x4{(float)n[0], (float)n[1], (float)n[2], (float)n[3]};
      };
      part[wave][lane] = P == 32 ? halves<32, 4>(get, wave) : P == 64 ? halves<64, 4>(get, wave) : halves<128, 4>(get, wave);
    }
    __syncthreads();
    if (wave == 0) {
      f32x4 sum = {0, 0, 0, 0};
      if (lane < D / 4) sum = (part[0][lane] + part[2][lane]) + (part[1][lane] + part[3][lane]);
      float top = 0.0f;  // (0 where a key's scale is not a number, and so all sums: such a block's mean counts as 0)
#pragma unroll
      for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(sum[e]));
      top = over_lanes_max(top, 64);
      const float f = top > 0.0f ? 127.0f * (1.0f / top) : 0.0f;
      if (lane < D / 4) {
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) w |= (uint32_t)(uint8_t)code_of(sum[e], f) << (8 * e);
        *reinterpret_cast<uint32_t*>(c.means + row * D + 4 * lane) = w;
      }
      if (lane == 0) c.mean_scales[row] = top / (127.0f * P);
    }
    __syncthreads();
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
    for (int e = 0; e < V; ++e) x[e] = value_of<T>(scale * (float)n[i + e]);
    store_n<V>(y + i, aligned, x);
  }
}

// A token's rows, a row to `lanes` lanes of 8 values.
template <typename T>
__device__ __forceinline__ void read_rows(const RowArgs& a) {
  const int lane = threadIdx.x % 64, D = a.head_dim;
  const int64_t w = (int64_t)blockIdx.x * kRowWaves + threadIdx.x / 64;
  const int t = (int)(w / a.waves), part = (int)(w % a.waves);
  if (t >= a.tokens) return;
  const int32_t p = a.pos[t], page = page_of(a, p, a.seq[t]);
  const int d = (lane & (a.lanes - 1)) * 8, per = 64 / a.lanes, slot = lane / a.lanes;
  if (d >= D) return;
  const int k_tasks = (a.k.heads + per - 1) / per, tasks = k_tasks + (a.v.heads + per - 1) / per;
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

// A window of neighbouring tokens of one head: keys as they lie, values turned as in append_window.  All of a thread's loads
// are under way before the first is used, and tokens of words that the window shares with others are read with them too: taken one by
// one they had two more latencies and 91 us for 32 thousand tokens of 8 heads of 128 instead of 50 (199 MB at 4.0 TB/s).
template <typename T>
__device__ __forceinline__ void read_window(const RowArgs& a, TurnLds& l, int b) {
  constexpr int G = kQ8Window / 4, U = G * (kMaxHeadDim / 4) / kRowThreads + 1, W = 4;
  const int heads = max(a.k.heads, a.v.heads);
  const int h = b % heads, t0 = b / heads * kQ8Window, n = min(kQ8Window, a.tokens - t0);
  const int D = a.head_dim, stride = D + 4, row8 = D / 8;
  load_window<true>(a, l, t0, n);
  const int tid = threadIdx.x;
  const auto place = [&](int i) { return l.pos[i] & (a.block - 1); };
  const auto head = [&](int page) { return (int64_t)page * a.kv_heads + h; };
  float scale = 0.0f;
  if (tid < 2 * kQ8Window) {
    const int i = tid % kQ8Window;
    const float* from = tid < kQ8Window ? a.k_scales : a.v_scales;
    if (l.page[i] >= 0 && (tid < kQ8Window ? a.k.y : a.v.y)) scale = from[head(l.page[i]) * a.block + place(i)];
  }
  // groups 1 ... 16, tokens first; then group 0
  const auto unit = [&](int u, int* q, int* x0) {
    const int j = tid + u * kRowThreads;
    *q = u < U - 1 ? 1 + j % G : 0, *x0 = u < U - 1 ? j / G * 4 : tid * 4;
    return *x0 < D && l.group[*q] >= 0;
  };
  uint32_t x[U][4] = {};
  if (a.v.y) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int q, x0;
      if (!unit(u, &q, &x0)) continue;
      const int8_t* from = a.v_codes + (head(l.group[q]) * D + x0) * a.block + (place(max(l.lead - 4 + 4 * q, 0)) & ~3);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[u][e] = *reinterpret_cast<const uint32_t*>(from + e * a.block);
    }
  }
  // a thread's pieces of keys: W at a time
  const auto piece = [&](int j, int* i, int* d) {
    *i = j / row8, *d = (j - *i * row8) * 8;
    return j < n * row8;
  };
  int8_t key[W][8] = {};
  const auto load_keys = [&](int j0) {
#pragma unroll
    for (int w = 0; w < W; ++w) {
      int i, d;
      if (!piece(j0 + w * kRowThreads, &i, &d)) continue;
      if (l.page[i] >= 0)
        load_n<8>(a.k_codes + (head(l.page[i]) * a.block + place(i)) * D + d, true, key[w]);
      else
        __builtin_memset(key[w], 0, 8);
    }
  };
  if (a.k.y) load_keys(tid);
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(x[u][e]));
  if (tid < kQ8Window)
    l.k_scale[tid] = scale;
  else if (tid < 2 * kQ8Window)
    l.v_scale[tid - kQ8Window] = scale;
  if (a.v.y) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int q, x0;
      if (!unit(u, &q, &x0)) continue;
      uint32_t y[4];
      turn4(x[u], y);
      const int i = l.lead - 4 + 4 * q;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i + e >= 0 && i + e < n) *reinterpret_cast<uint32_t*>(l.codes + (i + e) * stride + x0) = y[e];
    }
    each_loose(l, D, [&](int i, int d) {
      l.codes[i * stride + d] = l.page[i] < 0 ? 0 : a.v_codes[(head(l.page[i]) * D + d) * a.block + place(i)];
    });
  }
  __syncthreads();
  if (a.k.y) {
    for (int j0 = tid; j0 < n * row8; j0 += W * kRowThreads) {
      if (j0 != tid) load_keys(j0);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        int i, d;
        if (!piece(j0 + w * kRowThreads, &i, &d)) continue;
        write8<T>(key[w], l.k_scale[i], static_cast<T*>(a.k.y) + (t0 + i) * a.k.y_token + h * a.k.y_head + d, a.k.y_aligned);
      }
    }
  }
  if (!a.v.y) return;
  for (int j = tid; j < n * row8; j += kRowThreads) {
    int i, d;
    piece(j, &i, &d);
    int8_t v[8];
    __builtin_memcpy(v, l.codes + i * stride + d, 4);
    __builtin_memcpy(v + 4, l.codes + i * stride + d + 4, 4);
    write8<T>(v, l.v_scale[i], static_cast<T*>(a.v.y) + (t0 + i) * a.v.y_token + h * a.v.y_head + d, a.v.y_aligned);
  }
}

template <typename T>
__global__ __launch_bounds__(kRowThreads) void q8_read_kernel(RowArgs a) {
  __shared__ TurnLds l;
  if (a.row_groups == 0)
    read_window<T>(a, l, blockIdx.x);
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
  a.eps = norm.eps, a.inverse_dim = 1.0 / head_dim, a.norm = 1, a.tokens = tokens, a.head_dim = head_dim;
  const RunShape s = run_shape(tokens, head_dim / (2 * vec), {a.q.heads, a.k.heads, 0});
  if (!launchable(s.groups, kRowThreads)) return hipErrorInvalidConfiguration;
  a.lanes = s.lanes, a.run = s.run, a.shares = s.shares;
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
  if (norm) a.norm = 1, a.eps = norm->eps, a.inverse_dim = 1.0 / c.head_dim;
  if (q) a.q = head_rows(*q, q_out, norm ? norm->q_weight : nullptr, norm ? norm->q_head_stride : 0, values, dtype);
  a.k = head_rows(k, nullptr, norm ? norm->k_weight : nullptr, norm ? norm->k_head_stride : 0, values, dtype);
  a.v = head_rows(v, nullptr, nullptr, 0, values, dtype);
  a.v_vec = rows_aligned(v, 16 / dtype_bytes(dtype), dtype);
  const bool windows = by_windows(t);
  const RunShape s = run_shape(t.tokens, c.head_dim / (2 * vec), {a.q.heads, a.k.heads, windows ? 0 : a.v.heads});
  const int64_t groups = s.groups + (windows ? window_groups(t, c.kv_heads) : 0);
  if (!launchable(groups, kRowThreads) || !launchable(mean_groups(t, c.kv_heads), kRowThreads))
    return hipErrorInvalidConfiguration;
  a.lanes = s.lanes, a.run = s.run, a.shares = s.shares, a.row_groups = (int32_t)s.groups;
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
  const bool windows = by_windows(t);
  const RowShape s = row_shape(t.tokens, c.head_dim / 8, {a.k.heads, a.v.heads, 0});
  const int64_t groups = windows ? window_groups(t, c.kv_heads) : s.groups;
  if (!launchable(groups, kRowThreads)) return hipErrorInvalidConfiguration;
  a.lanes = s.lanes, a.waves = s.waves, a.row_groups = windows ? 0 : (int32_t)s.groups;
  return by_type(dtype, [&](auto ty) {
    q8_read_kernel<decltype(ty)><<<(unsigned)groups, kRowThreads, 0, stream>>>(a);
    return hipGetLastError();
  });
}

}  // namespace sdnn
