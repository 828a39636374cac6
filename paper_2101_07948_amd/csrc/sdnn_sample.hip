// The choice of the next token.
#include <type_traits>

#include "sdnn_decode_device.h"
#include "sdnn_serve_shape.h"

// Every operation is rounded by itself, so that a token's weight is the same wherever it is computed.
#pragma clang fp contract(off)

namespace sdnn {
namespace {

constexpr int kThreads = kSampleThreads, kWavesOf = kThreads / 64;  // of a workgroup that has a row
constexpr int kPass = kSamplePass, kPassWaves = kPass / 64;         // and of one that passes over a part of one
constexpr int kBins = kSampleBins, kGroups = kBins / 64;
constexpr int kList = kSampleList, kListEach = kList / kThreads;
constexpr int kOctaves = 46;  // bins divide the weights from 1 down to 2^-46, evenly in their logarithm
constexpr int kUnit = 44;     // weights are whole numbers of 2^-kUnit
constexpr int kRanked = 256;  // tokens that are put in order by counting those before each
constexpr int kFew = 1024;    // a top_k that a list has room for, with its last bin
static_assert(kBins >= kList, "a list's weights take the bins' place");

struct SampleArgs {
  const void* logits;
  int64_t row_stride;
  int32_t vocab, parts;
  const float* u;
  sdnn_sampling settings;
  int32_t* token;
  float* logprob;
  SampleSpace* space;  // a row's, where it is shared out over workgroups
};

// The exponent of a token's weight, not above 0; -infinity (or not a number, which has no weight either) where the logit is.
// (Where the largest logit is infinite it counts as 0 and all others as -infinity: see Row.)
__device__ __forceinline__ double exponent_of(const Weights& w, float l) { return ((double)l - (double)w.top) * w.scale; }
// 2^z as a whole number of 2^-kUnit: the fraction's power is a float of 24 bits, shifted by the whole part.  It is off by 2^-22 of
// itself at the most: the fraction's rounding 2^-26, the instruction's last place 2^-23, the cut to a whole number 2^-23.5.
__device__ __forceinline__ uint64_t weight_of(double z) {
  if (!(z > -(double)kOctaves)) return 0;
  const double n = rint(z);
  const float x = __builtin_amdgcn_exp2f((float)(z - n)) * 0x1p23f;
  return ((uint64_t)(uint32_t)x << (kUnit - 23)) >> -(int)n;
}
constexpr double kBinsAnOctave = (double)kBins / kOctaves;
__device__ __forceinline__ int bin_of(double z) {
  return z > -(double)kOctaves ? min((int)(-z * kBinsAnOctave), kBins - 1) : kBins - 1;
}

// Tokens in order: larger logits first, equal ones by index.  (-0 and 0 are equal.)
__device__ __forceinline__ uint32_t ascending_of(float l) {
  const int32_t b = __float_as_int(l == 0.0f ? 0.0f : l);
  return (uint32_t)b ^ (b < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float float_of(uint32_t ascending) {
  return __uint_as_float(ascending & 0x80000000u ? ascending ^ 0x80000000u : ~ascending);
}
__device__ __forceinline__ uint64_t order_of(float l, int i) { return (uint64_t)~ascending_of(l) << 32 | (uint32_t)i; }
__device__ __forceinline__ float logit_of(uint64_t order) { return float_of(~(uint32_t)(order >> 32)); }

// The lowest float for which holds(x) is true, which is true for all larger ones: its 32 bits are found 6 at a time, each lane
// asking about one of 64 parts.  (So that a pass over a row compares floats in place of what `holds` computes.)
template <typename F>
__device__ __forceinline__ float lowest_where(const F& holds) {
  constexpr uint32_t LEAST = 0x007fffffu;  // -infinity, in ascending order
  const int lane = threadIdx.x % 64;
  uint32_t from = 0;
#pragma unroll
  for (int bits = 26; bits >= 0; bits -= bits > 2 ? 6 : 2) {
    const uint64_t end = (uint64_t)from + ((uint64_t)(lane + 1) << bits) - 1;  // of this lane's part
    const bool past = end > 0xff800000u;                                       // (infinity is the last)
    const uint64_t yes = __ballot(past || (end >= LEAST && holds(float_of((uint32_t)end))));
    from += (uint32_t)(yes ? __builtin_ctzll(yes) : 63) << bits;
  }
  return float_of(from);
}

// A row, read in pieces of 16 bytes that lie where 16-byte loads may; those at its ends value by value.  Piece g has the
// tokens g V - lead ... g V - lead + V - 1.
template <typename T>
struct Row {
  static constexpr int V = 16 / sizeof(T);
  struct Piece {
    T v[V];
  };
  const T* x;
  int lead, pieces, vocab;
  bool infinite = false;  // the largest logit is infinity: it and its like count as 0, all others as -infinity
  __device__ __forceinline__ Row(const SampleArgs& a, int r) {
    x = static_cast<const T*>(a.logits) + r * a.row_stride;
    vocab = a.vocab;
    lead = (int)((uintptr_t)x % 16 / sizeof(T));
    pieces = (lead + vocab + V - 1) / V;
  }
  __device__ __forceinline__ Piece load(int g) const {
    const int i = g * V - lead;
    Piece p;
    if (i >= 0 && i + V <= vocab) {
      load_n<V>(x + i, true, p.v);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) p.v[e] = i + e >= 0 && i + e < vocab ? x[i + e] : (T)-INFINITY;
    }
    return p;
  }
  // A token's logit, NaN as -infinity; -infinity also past the row's ends.
  __device__ __forceinline__ float logit(const Piece& p, int e) const {
    const float l = (float)p.v[e];
    if (infinite) return l == INFINITY ? 0.0f : -INFINITY;
    return l == l ? l : -INFINITY;
  }
  // f(index, logit) of all tokens of pieces begin, begin + step ... below end, several loads under way at once.
  template <typename F>
  __device__ __forceinline__ void each(int begin, int end, int step, const F& f) const {
    constexpr int AHEAD = 4;
    for (int g = begin; g < end; g += AHEAD * step) {
      Piece p[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (g + k * step < end) p[k] = load(g + k * step);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k)
        if (g + k * step < end) {
#pragma unroll
          for (int e = 0; e < V; ++e) f((g + k * step) * V - lead + e, logit(p[k], e));
        }
    }
  }
};

// What a row asks for (see Limits).
__device__ __forceinline__ Limits limits_of(const SampleArgs& a, int r) {
  const sdnn_sampling& s = a.settings;
  // (all loads under way before the first is needed)
  const float temperature = s.temperature ? s.temperature[r] : 1.0f, top_p = s.top_p ? s.top_p[r] : 1.0f;
  const float min_p = s.min_p ? s.min_p[r] : 0.0f;
  const int32_t top_k = s.top_k ? s.top_k[r] : 0;
  Limits l;
  l.u = a.u[r];
  l.temperature = temperature;
  l.top_k = top_k > 0 && top_k < a.vocab ? top_k : 0;
  l.top_p = top_p < 1.0f ? top_p : 1.0f;
  l.min_p = min_p > 0.0f ? min_p : 0.0f;
  l.first = !(temperature > 0.0f) || top_k == 1 || !(l.top_p > 0.0f) || l.min_p > 1.0f;
  return l;
}
__device__ __forceinline__ bool by_bins(const Limits& l) { return l.top_k > 0 || l.top_p < 1.0f; }
// The bins' masses are needed, not only their counts: a limit that a list does not settle goes by them.
__device__ __forceinline__ bool by_masses(const Limits& l) { return l.top_p < 1.0f && (l.top_k == 0 || l.top_k > kFew); }
__device__ __forceinline__ double least_of(const Limits& l) { return l.min_p > 0.0f ? log2((double)l.min_p) : -INFINITY; }

// ---------------------------------------------------------------- sums over a wave

// x of the lane that CTRL names (see DPP's row_shr, row_bcast), `none` where there is none.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t from_lane(uint64_t x, uint64_t none) {
  const int lo = __builtin_amdgcn_update_dpp((int)(uint32_t)none, (int)(uint32_t)x, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp((int)(none >> 32), (int)(x >> 32), CTRL, ROWS, 0xf, false);
  return (uint64_t)(uint32_t)hi << 32 | (uint32_t)lo;
}
// f over this lane and all before it: within rows of 16 lanes, then the rows before.
template <typename F>
__device__ __forceinline__ uint64_t running(uint64_t x, uint64_t none, const F& f) {
  x = f(x, from_lane<0x111, 0xf>(x, none));
  x = f(x, from_lane<0x112, 0xf>(x, none));
  x = f(x, from_lane<0x114, 0xf>(x, none));
  x = f(x, from_lane<0x118, 0xf>(x, none));
  x = f(x, from_lane<0x142, 0xa>(x, none));
  return f(x, from_lane<0x143, 0xc>(x, none));
}
__device__ __forceinline__ uint64_t of_lane(uint64_t x, int lane) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}
__device__ __forceinline__ uint64_t wave_running_sum(uint64_t x) {
  return running(x, 0, [](uint64_t a, uint64_t b) { return a + b; });
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t x) { return of_lane(wave_running_sum(x), 63); }
__device__ __forceinline__ uint64_t wave_least(uint64_t x) {
  return of_lane(running(x, ~0ull, [](uint64_t a, uint64_t b) { return a < b ? a : b; }), 63);
}

// Sums over a workgroup's waves through LDS: of all threads, or of this one and all before it.
template <int WAVES>
__device__ __forceinline__ uint64_t block_sum(uint64_t (&lds)[kWavesOf], uint64_t x) {
  x = wave_sum(x);
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) x += lds[w];
  __syncthreads();
  return x;
}
__device__ __forceinline__ uint64_t block_running_sum(uint64_t (&lds)[kWavesOf], uint64_t x) {
  x = wave_running_sum(x);
  if (threadIdx.x % 64 == 63) lds[threadIdx.x / 64] = x;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWavesOf; ++w)
    if (w < (int)threadIdx.x / 64) x += lds[w];
  __syncthreads();
  return x;
}

// ---------------------------------------------------------------- a row's first token

// The first token in the order of pieces begin ... end - 1, for all threads of WAVES waves.
template <int WAVES, typename T>
__device__ __forceinline__ uint64_t first_of(uint64_t (&lds)[kWavesOf], const Row<T>& row, int begin, int end) {
  float top = -INFINITY;
  int at = 0x7fffffff;
  row.each(begin + threadIdx.x, end, 64 * WAVES, [&](int i, float x) {
    if (x > top) top = x, at = i;  // (a thread's tokens ascend)
  });
  uint64_t first = wave_least(order_of(top, at));
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = first;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < WAVES; ++v) first = lds[v] < first ? lds[v] : first;
  __syncthreads();
  return first;
}

template <typename T>
__device__ __forceinline__ Weights weights_of(uint64_t first, const Limits& limits, Row<T>& row) {
  const float top = logit_of(first);
  row.infinite = top == INFINITY;
  return {row.infinite ? 0.0f : top, 1.4426950408889634 / (double)limits.temperature};
}

// A row of which nothing or only its first token is left.
__device__ __forceinline__ bool settled(uint64_t first, const Limits& limits) {
  return limits.first || logit_of(first) == -INFINITY;
}
__device__ __forceinline__ void store_first(const SampleArgs& a, int r, uint64_t first) {
  if (threadIdx.x > 0) return;
  const bool none = logit_of(first) == -INFINITY;
  a.token[r] = none ? -1 : (int32_t)(uint32_t)first;
  if (a.logprob) a.logprob[r] = none ? -INFINITY : 0.0f;
}

__device__ __forceinline__ void store_token(const SampleArgs& a, int r, int token, double exponent, uint64_t total) {
  a.token[r] = token;
  if (a.logprob) a.logprob[r] = (float)((exponent + ((double)kUnit - log2((double)total))) * 0.6931471805599453);
}

// Where u points to in running sums up to `total`.
__device__ __forceinline__ uint64_t target_of(float u, uint64_t total) {
  const double x = (double)(u > 0.0f ? u : 0.0f) * (double)total;
  const uint64_t t = x < (double)total ? (uint64_t)x : total;
  return t < total ? t : total - 1;
}
// The last whole number below top_p of `kept`: a token is kept where the weights before it sum to no more.
__device__ __forceinline__ uint64_t limit_of(float top_p, uint64_t kept) {
  return (uint64_t)ceil((double)top_p * (double)kept) - 1;
}

// ---------------------------------------------------------------- bins

struct Bins {
  uint64_t mass[kBins];
  uint32_t count[kBins];
};

// The bins of pieces begin ... end - 1: tokens' numbers, and where asked for their weights.
template <int WAVES, typename T>
__device__ __forceinline__ void fill_bins(Bins& b, const Row<T>& row, const Weights& w, int begin, int end, bool masses) {
  for (int i = threadIdx.x; i < kBins; i += 64 * WAVES) b.mass[i] = 0, b.count[i] = 0;
  __syncthreads();
  row.each(begin + threadIdx.x, end, 64 * WAVES, [&](int, float x) {
    if (!(x > -INFINITY)) return;
    const double z = exponent_of(w, x);
    const int at = bin_of(z);
    atomicAdd(&b.count[at], 1u);
    if (masses) atomicAdd(reinterpret_cast<unsigned long long*>(&b.mass[at]), (unsigned long long)weight_of(z));
  });
  __syncthreads();
}

// Sums of 64 bins each, which is where a search begins.
struct Groups {
  uint64_t mass[kGroups];
  uint32_t count[kGroups];
};
template <int WAVES>
__device__ __forceinline__ void sum_groups(const Bins& b, Groups& g) {
  const int lane = threadIdx.x % 64;
  for (int i = threadIdx.x / 64; i < kGroups; i += WAVES) {
    const uint64_t m = wave_sum(b.mass[i * 64 + lane]), c = wave_sum(b.count[i * 64 + lane]);
    if (lane == 0) g.mass[i] = m, g.count[i] = (uint32_t)c;
  }
  __syncthreads();
}

// The bin with which the running sums, counts or masses, pass `target`, and the sums before it (bin -1: none does).  By one wave.
struct Found {
  int bin;
  uint32_t count;
  uint64_t mass;
};
__device__ __forceinline__ Found find_bin(const Bins& b, const Groups& g, bool by_count, uint64_t target) {
  const int lane = threadIdx.x % 64;
  Found f = {-1, 0, 0};
  int first = 0;
#pragma unroll
  for (int level = 0; level < 2; ++level) {
    const bool there = level == 1 || lane < kGroups;
    const uint64_t m = !there ? 0 : level ? b.mass[first + lane] : g.mass[lane];
    const uint32_t c = !there ? 0 : level ? b.count[first + lane] : g.count[lane];
    const uint64_t m1 = wave_running_sum(m), c1 = wave_running_sum(c);
    const uint64_t past = __ballot(target < (by_count ? f.count + c1 : f.mass + m1));
    if (!past) return {-1, 0, 0};
    const int at = __builtin_ctzll(past);
    f.mass += of_lane(m1 - m, at), f.count += (uint32_t)of_lane(c1 - c, at);
    if (level == 1) f.bin = first + at;
    first = at * 64;
  }
  return f;
}

// What the bins tell of a row's limits (of several waves one; see CutKind).  With top_k the last bin is of no account: what is in
// it has no weight.
__device__ __forceinline__ Cut cut_of(const Bins& b, const Groups& g, const Limits& limits) {
  const int lane = threadIdx.x % 64;
  Cut c = {};
  c.kind = kWhole, c.edge = c.edge_p = c.end_p = -1;
  const bool by_p = limits.top_p < 1.0f;
  c.total = wave_sum(lane < kGroups ? g.mass[lane] : 0);
  uint64_t low = c.total, high = c.total;  // what top_k leaves has a mass from low to high
  if (limits.top_k > 0) {
    const Found f = find_bin(b, g, true, (uint64_t)(limits.top_k - 1));
    if (f.bin >= 0 && f.bin < kBins - 1) {
      c.edge = f.bin, c.tokens = b.count[f.bin], c.rank = (uint32_t)(limits.top_k - 1) - f.count, c.mass = f.mass;
      const uint32_t all = f.count + c.tokens;
      c.kind = all <= kList ? kShort : c.tokens <= kList ? kEdges : kOther;
      // the first of a bin are no lighter than its mean, and by no more than the bin's width
      const double part = (double)b.mass[c.edge] / c.tokens * (c.rank + 1);
      low = c.mass + (uint64_t)(part * 0.999999), high = c.mass + (uint64_t)(part * 1.024) + c.rank + 1;
      if (c.kind == kShort) c.tokens = all;
    } else {  // fewer tokens than top_k have a weight
      const uint32_t n = (uint32_t)wave_sum(lane < kGroups ? g.count[lane] : 0) - b.count[kBins - 1];
      if (n <= kList) c.kind = kShort, c.edge = kBins - 2, c.tokens = n;
    }
  }
  if (c.kind == kShort || !by_p) return c;
  if (!by_masses(limits)) {
    c.kind = kOther;
    return c;
  }
  const Found f = find_bin(b, g, false, limit_of(limits.top_p, low));
  if (f.bin < 0) return c;
  const Found h = find_bin(b, g, false, limit_of(limits.top_p, min(high, c.total)));
  c.edge_p = f.bin, c.end_p = h.bin;
  c.tokens_p = h.count + b.count[h.bin] - f.count, c.mass_p = f.mass;
  if (c.edge < 0 && f.count + c.tokens_p <= kList)
    c.kind = kShort, c.edge = f.bin, c.tokens = f.count + c.tokens_p;
  else if (c.kind != kOther)  // (kWhole: what top_k leaves)
    c.kind = c.tokens_p <= kList ? kEdges : kOther;
  return c;
}
static_assert(kOctaves <= 0.034 * kBins, "a bin's weights are within a factor of 1.024 of each other");

// One end of the logits that go to lists (see Ranges): by one wave.  Of kShort's list, at[3] is where the tokens of bin edge_p end.
__device__ __forceinline__ float range_of(const Cut& c, const Weights& w, int which) {
  // the last bin of a range, or the one before its first
  const int ends[4] = {c.edge, c.edge - 1, c.end_p, c.edge_p - 1}, b = ends[which];
  const bool asked = (which < 2 ? c.edge : c.edge_p) >= 0 && !(c.kind == kShort && (which == 1 || which == 2));
  if (c.kind == kWhole || c.kind == kOther || !asked || b < 0) return INFINITY;
  return lowest_where([&](float x) { return bin_of(exponent_of(w, x)) <= b; });
}

// ---------------------------------------------------------------- lists

struct Lists {
  uint64_t list[kList], list_p[kList];
  int32_t listed, listed_p;
};

// Tokens of pieces begin ... end - 1 to lists, in any order.
template <int WAVES, typename T>
__device__ __forceinline__ void gather(Lists& l, const Row<T>& row, int begin, int end, const Ranges& r) {
  if (threadIdx.x == 0) l.listed = l.listed_p = 0;
  __syncthreads();
  row.each(begin + threadIdx.x, end, 64 * WAVES, [&](int i, float x) {
    if (x >= r.at[0] && x < r.at[1]) {
      const int at = atomicAdd(&l.listed, 1);
      if (at < kList) l.list[at] = order_of(x, i);
    }
    if (x >= r.at[2] && x < r.at[3]) {
      const int at = atomicAdd(&l.listed_p, 1);
      if (at < kList) l.list_p[at] = order_of(x, i);
    }
  });
  __syncthreads();
}

// A list of n numbers in ascending order, by kThreads threads.  (Its place from n to the next power of two is used up.)
__device__ __forceinline__ void put_in_order(uint64_t (&list)[kList], int n) {
  const int tid = threadIdx.x;
  if (n <= kRanked) {
    uint64_t x = 0;
    int rank = 0;
    if (tid < n) {
      x = list[tid];
#pragma unroll 8
      for (int j = 0; j < n; ++j) rank += list[j] < x;
    }
    __syncthreads();
    if (tid < n) list[rank] = x;
    __syncthreads();
    return;
  }
  // A merge's steps of 128 and more are exchanged through LDS, those below within a wave, whose lanes have two numbers each.
  int size = 2 * kRanked;
  while (size < n) size *= 2;
  for (int i = n + tid; i < size; i += kThreads) list[i] = ~0ull;
  __syncthreads();
  const bool mine = 2 * tid < size;  // (whole waves)
  uint64_t x = 0, y = 0;
  if (mine) x = list[2 * tid], y = list[2 * tid + 1];
  for (int run = 2; run <= size; run *= 2) {
    const bool up = (2 * tid & run) == 0;
    if (run > 128) {
      if (mine) list[2 * tid] = x, list[2 * tid + 1] = y;
      __syncthreads();
      for (int step = run / 2; step >= 128; step /= 2) {
        if (mine) {
          const int a = (tid & ~(step - 1)) * 2 + (tid & (step - 1)), b = a + step;
          const uint64_t v = list[a], w = list[b];
          if ((v > w) == ((a & run) == 0)) list[a] = w, list[b] = v;
        }
        __syncthreads();
      }
      if (mine) x = list[2 * tid], y = list[2 * tid + 1];
    }
    if (mine) {
      for (int step = min(run / 2, 64); step >= 2; step /= 2) {  // between lanes step / 2 apart
        const uint64_t v = __shfl_xor((unsigned long long)x, step / 2), w = __shfl_xor((unsigned long long)y, step / 2);
        const bool lower = ((2 * tid & step) == 0) == up;  // keeps the smaller
        x = (v < x) == lower ? v : x, y = (w < y) == lower ? w : y;
      }
      const bool turned = (x > y) == up;
      const uint64_t v = turned ? y : x;
      y = turned ? x : y, x = v;
    }
    if (run > 64) __syncthreads();  // (the list is read before the next merge writes it)
  }
  if (mine) list[2 * tid] = x, list[2 * tid + 1] = y;
  __syncthreads();
}

// A row's workgroup's LDS.
struct SampleLds {
  union {
    Bins bins;
    uint64_t list_p[kList];
    uint64_t mass[kList];  // of tokens in their order
  };
  uint64_t list[kList];
  Groups groups;
  Cut cut;
  Ranges ranges;
  uint64_t masses[kWavesOf];
  // what one thread or wave finds for all
  uint64_t order, total;
  int32_t count;
  Kept kept;
};

// Of n tokens of a list, in order, the one with which their running sums, counts or masses, pass `target`; left in l.order,
// with the mass before it in l.total.
__device__ __forceinline__ void find_listed(SampleLds& l, const uint64_t (&list)[kList], const Weights& w, int n, bool by_count,
                                            uint64_t target) {
  const auto find = [&](auto per, const auto& running_sum) {
    constexpr int PER = decltype(per)::value;
    uint64_t m[PER], sum = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = threadIdx.x * PER + i;
      m[i] = at < n ? weight_of(exponent_of(w, logit_of(list[at]))) : 0;
      sum += m[i];
    }
    uint64_t m0 = running_sum(sum) - sum;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = threadIdx.x * PER + i;
      const uint64_t before = by_count ? at : m0, with = before + (by_count ? 1 : m[i]);
      if (at < n && before <= target && target < with) l.order = list[at], l.total = m0;
      m0 += m[i];
    }
  };
  if (n > kRanked)
    find(std::integral_constant<int, kListEach>(), [&](uint64_t x) { return block_running_sum(l.masses, x); });
  else if (threadIdx.x < 64)
    find(std::integral_constant<int, kRanked / 64>(), [](uint64_t x) { return wave_running_sum(x); });
  __syncthreads();
}

// What is left: the order up to `last`, exponents from log2 min_p.  By one wave.
__device__ __forceinline__ Kept kept_of(const Weights& w, uint64_t last, const Limits& limits) {
  Kept k = last == ~0ull ? Kept{-INFINITY, -1} : Kept{logit_of(last), (int32_t)(uint32_t)last};
  if (limits.min_p > 0.0f) {
    const double least = least_of(limits);
    const float lowest = lowest_where([&](float x) { return exponent_of(w, x) >= least; });
    if (lowest > k.logit) k = {lowest, 0x7fffffff};
  }
  return k;
}
__device__ __forceinline__ uint64_t kept_weight(const Weights& w, const Kept& k, int i, float x) {
  return x > k.logit || (x == k.logit && i <= k.index) ? weight_of(exponent_of(w, x)) : 0;
}

// The token from the masses m of tokens x, kListEach to a thread (0: none): the masses are added for each 256 indexes, then for each
// index of the 256 that the target lies in.
__device__ __forceinline__ void pick_by_bins(const SampleArgs& a, int r, SampleLds& l, const Weights& w, const Limits& limits,
                             const uint64_t (&x)[kListEach], const uint64_t (&m)[kListEach]) {
  static_assert((kMaxVocab - 1) >> 8 < kBins, "a bin for each 256 indexes");
  uint64_t sum = 0;
#pragma unroll
  for (int i = 0; i < kListEach; ++i) sum += m[i];
  const uint64_t total = block_sum<kWavesOf>(l.masses, sum);
  uint64_t target = target_of(limits.u, total);
  uint32_t high = 0, token = 0;
#pragma unroll
  for (int level = 0; level < 2; ++level) {
    for (int i = threadIdx.x; i < kBins; i += kThreads) l.bins.mass[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kListEach; ++i) {
      const uint32_t index = (uint32_t)x[i];
      if (m[i] && (level == 0 || index >> 8 == high))
        atomicAdd(reinterpret_cast<unsigned long long*>(&l.bins.mass[level ? index & 255 : index >> 8]), (unsigned long long)m[i]);
    }
    __syncthreads();
    sum_groups<kWavesOf>(l.bins, l.groups);
    const Found f = find_bin(l.bins, l.groups, false, target);
    __syncthreads();
    target -= f.mass;
    token = high << 8 | (uint32_t)f.bin, high = (uint32_t)f.bin;
  }
#pragma unroll
  for (int i = 0; i < kListEach; ++i)
    if (m[i] && (uint32_t)x[i] == token) store_token(a, r, (int)token, exponent_of(w, logit_of(x[i])), total);
}

// The row's token from the list of its first tokens (more than the limits leave, see kShort).  edge: what the logits of the
// tokens of bin edge_p are below.
__device__ __forceinline__ void pick_from_list(const SampleArgs& a, int r, SampleLds& l, const Weights& w, const Limits& limits,
                                               const Cut& cut, float edge) {
  const int tid = threadIdx.x, n = (int)cut.tokens;
  const bool by_p = cut.edge_p >= 0;  // it ends with the bin in which top_p does, not top_k
  if (n > kRanked && by_p) {
    // only the tokens of its last bin are put in order
    uint64_t x[kListEach], m[kListEach];
    if (tid == 0) l.count = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kListEach; ++i) {
      const int at = tid + i * kThreads;
      x[i] = at < n ? l.list[at] : ~0ull;
      if (at < n && logit_of(x[i]) < edge) l.list_p[atomicAdd(&l.count, 1)] = x[i];
    }
    __syncthreads();
    const int some = l.count;
    put_in_order(l.list_p, some);
    find_listed(l, l.list_p, w, some, false, limit_of(limits.top_p, cut.total) - cut.mass_p);
    if (tid < 64) {
      const Kept k = kept_of(w, l.order, limits);
      if (tid == 0) l.kept = k;
    }
    __syncthreads();
    const Kept kept = l.kept;
#pragma unroll
    for (int i = 0; i < kListEach; ++i) m[i] = tid + i * kThreads < n ? kept_weight(w, kept, (int)(uint32_t)x[i], logit_of(x[i])) : 0;
    return pick_by_bins(a, r, l, w, limits, x, m);
  }
  put_in_order(l.list, n);
  const int most = by_p ? n : min(n, limits.top_k);
  // the masses of what is kept of PER tokens of the order
  const auto keep = [&](auto& x, auto& m, const auto& running_sum, const auto& sum_of) {
    constexpr int PER = sizeof(m) / 8;
    const double least = least_of(limits);
    uint64_t sum = 0;
    bool in[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = tid * PER + i;
      x[i] = l.list[min(at, n - 1)];
      const double z = exponent_of(w, logit_of(x[i]));
      m[i] = at < most ? weight_of(z) : 0;
      in[i] = z >= least;
      sum += m[i];
    }
    uint64_t before = running_sum(sum) - sum, limit = ~0ull;
    if (limits.top_p < 1.0f) limit = limit_of(limits.top_p, by_p ? cut.total : sum_of(sum));
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const uint64_t mass = m[i];
      if (!in[i] || before > limit) m[i] = 0;
      before += mass;
    }
  };
  if (n > kRanked) {
    uint64_t x[kListEach], m[kListEach];
    keep(x, m, [&](uint64_t y) { return block_running_sum(l.masses, y); },
         [&](uint64_t y) { return block_sum<kWavesOf>(l.masses, y); });
    return pick_by_bins(a, r, l, w, limits, x, m);
  }
  if (tid < 64) {
    uint64_t x[kRanked / 64], m[kRanked / 64], sum = 0;
    keep(x, m, [](uint64_t y) { return wave_running_sum(y); }, [](uint64_t y) { return wave_sum(y); });
#pragma unroll
    for (int i = 0; i < kRanked / 64; ++i) l.mass[tid * (kRanked / 64) + i] = m[i], sum += m[i];
    sum = wave_sum(sum);
    if (tid == 0) l.total = sum;
  }
  __syncthreads();
  if (tid >= n) return;
  const uint64_t total = l.total, target = target_of(limits.u, total), x = l.list[tid], mine = l.mass[tid];
  uint64_t before = 0;
#pragma unroll 8
  for (int j = 0; j < n; ++j) before += (uint32_t)l.list[j] < (uint32_t)x ? l.mass[j] : 0;
  if (before <= target && target < before + mine) store_token(a, r, (int)(uint32_t)x, exponent_of(w, logit_of(x)), total);
}

// The last token that the limits leave where the last bins' tokens tell (see kEdges); load(which): l.list from the row's list of
// those of bin edge, or of bins edge_p to end_p.
template <typename F>
__device__ __forceinline__ uint64_t last_of_edges(SampleLds& l, const Weights& w, const Limits& limits, const Cut& cut,
                                                  const F& load) {
  uint64_t last = ~0ull, kept = cut.total;
  if (cut.edge >= 0) {
    load(0);
    put_in_order(l.list, (int)cut.tokens);
    find_listed(l, l.list, w, (int)cut.tokens, true, cut.rank);
    last = l.order;
    kept = cut.mass + l.total + weight_of(exponent_of(w, logit_of(last)));
    __syncthreads();
  }
  if (cut.edge_p >= 0) {
    load(1);
    put_in_order(l.list, (int)cut.tokens_p);
    find_listed(l, l.list, w, (int)cut.tokens_p, false, limit_of(limits.top_p, kept) - cut.mass_p);
    last = l.order;  // (not after the last that top_k leaves)
  }
  return last;
}

// ---------------------------------------------------------------- what is left, by index

// The last token of bin `bin` that is left: the one with which the running sums of the bin's tokens in their order,
// counts or masses, pass `target`; left in l.order, with the mass before it in the bin in l.total.  (The bins are used up.)
template <typename T>
__device__ __forceinline__ void resolve(SampleLds& l, const Row<T>& row, const Weights& w, int bin, bool by_count, uint64_t target) {
  const int tid = threadIdx.x;
  // digit by digit of a token's place in the order, from the first in which the bin's tokens differ
  const auto each = [&](const auto& f) {
    row.each(tid, row.pieces, kThreads, [&](int i, float x) {
      const double z = exponent_of(w, x);
      if (x > -INFINITY && bin_of(z) == bin) f(order_of(x, i), z);
    });
  };
  uint64_t least = ~0ull, most = 0;
  each([&](uint64_t v, double) { least = v < least ? v : least, most = v > most ? v : most; });
  least = wave_least(least), most = ~wave_least(~most);
  __syncthreads();
  if (tid % 64 == 0) l.masses[tid / 64] = least, l.list[tid / 64] = most;
  __syncthreads();
  for (int v = 0; v < kWavesOf; ++v)
    least = l.masses[v] < least ? l.masses[v] : least, most = l.list[v] > most ? l.list[v] : most;
  constexpr int DIGIT = 11;
  static_assert(1 << DIGIT == kBins, "a bin for each value of a digit");
  int bits = least == most ? 0 : 64 - __builtin_clzll(least ^ most);
  uint64_t prefix = bits == 64 ? 0 : most >> bits << bits, mass_before = 0;
  while (bits > 0) {
    const int shift = max(bits - DIGIT, 0), top = bits;
    __syncthreads();
    for (int i = tid; i < kBins; i += kThreads) l.bins.mass[i] = 0, l.bins.count[i] = 0;
    __syncthreads();
    each([&](uint64_t v, double z) {
      if (top < 64 && v >> top != prefix >> top) return;
      const int d = (int)(v >> shift & (kBins - 1) & ((1u << (top - shift)) - 1));
      atomicAdd(&l.bins.count[d], 1u);
      atomicAdd(reinterpret_cast<unsigned long long*>(&l.bins.mass[d]), (unsigned long long)weight_of(z));
    });
    __syncthreads();
    sum_groups<kWavesOf>(l.bins, l.groups);
    const Found f = find_bin(l.bins, l.groups, by_count, target);
    prefix |= (uint64_t)f.bin << shift;
    target -= by_count ? f.count : f.mass;
    mass_before += f.mass;
    bits = shift;
  }
  __syncthreads();
  if (tid == 0) l.order = prefix, l.total = mass_before;
  __syncthreads();
}

// The last token that the limits leave, in the order, where no list holds what is to be known: from the row.
template <typename T>
__device__ __forceinline__ uint64_t last_of(SampleLds& l, const Row<T>& row, const Weights& w, const Limits& limits) {
  uint64_t last = ~0ull;
  fill_bins<kWavesOf>(l.bins, row, w, 0, row.pieces, true);
  sum_groups<kWavesOf>(l.bins, l.groups);
  uint64_t kept = wave_sum(threadIdx.x % 64 < kGroups ? l.groups.mass[threadIdx.x % 64] : 0);
  if (limits.top_k > 0) {
    const Found f = find_bin(l.bins, l.groups, true, (uint64_t)(limits.top_k - 1));
    if (f.bin >= 0 && f.bin < kBins - 1) {
      resolve(l, row, w, f.bin, true, (uint64_t)(limits.top_k - 1) - f.count);
      last = l.order;
      kept = f.mass + l.total + weight_of(exponent_of(w, logit_of(last)));
      fill_bins<kWavesOf>(l.bins, row, w, 0, row.pieces, true);
      sum_groups<kWavesOf>(l.bins, l.groups);
    }
  }
  const uint64_t limit = limits.top_p < 1.0f ? limit_of(limits.top_p, kept) : kept;
  if (limit < kept) {
    const Found f = find_bin(l.bins, l.groups, false, limit);
    resolve(l, row, w, f.bin, false, limit - f.mass);
    last = l.order < last ? l.order : last;
  }
  __syncthreads();
  return last;
}

// The token at which the masses kept, by index, pass the target.  They are added for 16 parts of the pieces, then for 16 parts
// of the one that the token lies in, until a wave has few enough to look at them one by one.  total: all masses of the row where
// they are known (then begin ... end is the part with the token, and `before` what is before it), else 0.
template <typename T>
__device__ __forceinline__ void pick_by_index(const SampleArgs& a, int r, uint64_t (&lds)[kWavesOf], const Row<T>& row,
                                              const Weights& w, const Limits& limits, const Kept& kept, int begin, int end,
                                              uint64_t before, uint64_t total) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint64_t target = total ? target_of(limits.u, total) : 0;
  while (!total || end - begin > 64) {
    const int part = (end - begin + kWavesOf - 1) / kWavesOf;
    const int from = min(begin + wave * part, end), to = min(from + part, end);
    uint64_t m = 0;
    row.each(from + lane, to, 64, [&](int i, float x) { m += kept_weight(w, kept, i, x); });
    m = wave_sum(m);
    if (lane == 0) lds[wave] = m;
    __syncthreads();
    const uint64_t mine = lane < kWavesOf ? lds[lane] : 0, run = wave_running_sum(mine);
    __syncthreads();
    if (!total) total = of_lane(run, 63), target = target_of(limits.u, total);
    const int v = __builtin_ctzll(__ballot(target < before + run));
    before += of_lane(run - mine, v);
    begin = min(begin + v * part, end), end = min(begin + part, end);
  }
  if (wave > 0) return;
  // a piece to a lane
  constexpr int V = Row<T>::V;
  uint64_t m[V], sum = 0;
  const int g = begin + lane;
  typename Row<T>::Piece p;
  if (g < end) p = row.load(g);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    m[e] = g < end ? kept_weight(w, kept, g * V - row.lead + e, row.logit(p, e)) : 0;
    sum += m[e];
  }
  uint64_t run = wave_running_sum(sum) + before - sum;
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if (run <= target && target < run + m[e])
      store_token(a, r, g * V - row.lead + e, exponent_of(w, row.logit(p, e)), total);
    run += m[e];
  }
}

// A row to a workgroup, in one launch.  Of the passes over the row (its first token; the bins; the tokens that go to a list) those
// that it does not ask for are left out; all but the first read from L2.
//   Latency bounds it, a compute unit's reading and a chain of searches.  A row of 50021 in 32 bits with top_k 40 and top_p: 25 us.
// With bins counted in 32-bit arithmetic it takes as long, so what a token costs does not count.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ SampleLds l;
  const int r = blockIdx.x, wave = threadIdx.x / 64;
  Row<T> row(a, r);
  const Limits limits = limits_of(a, r);
  const uint64_t first = first_of<kWavesOf>(l.masses, row, 0, row.pieces);
  if (settled(first, limits)) return store_first(a, r, first);
  const Weights w = weights_of(first, limits, row);
  uint64_t last = ~0ull;
  if (by_bins(limits)) {
    fill_bins<kWavesOf>(l.bins, row, w, 0, row.pieces, by_masses(limits));
    sum_groups<kWavesOf>(l.bins, l.groups);
    if (wave == 0) l.cut = cut_of(l.bins, l.groups, limits);
    __syncthreads();
    const Cut cut = l.cut;
    if (wave < 4) {
      const float at = range_of(cut, w, wave);
      if (threadIdx.x % 64 == 0) l.ranges.at[wave] = at;
    }
    __syncthreads();
    const Ranges ranges = l.ranges;
    const auto load = [&](int which) {
      const float from = ranges.at[2 * which], to = ranges.at[2 * which + 1];
      __syncthreads();
      if (threadIdx.x == 0) l.count = 0;
      __syncthreads();
      row.each(threadIdx.x, row.pieces, kThreads, [&](int i, float x) {
        if (x >= from && x < to) l.list[min(atomicAdd(&l.count, 1), kList - 1)] = order_of(x, i);
      });
      __syncthreads();
    };
    if (cut.kind == kShort) {
      load(0);
      return pick_from_list(a, r, l, w, limits, cut, ranges.at[3]);
    }
    if (cut.kind == kEdges) last = last_of_edges(l, w, limits, cut, load);
    if (cut.kind == kOther) last = last_of(l, row, w, limits);
  }
  pick_by_index(a, r, l.masses, row, w, limits, kept_of(w, last, limits), 0, row.pieces, 0, 0);
}

// ---------------------------------------------------------------- rows shared out over workgroups

struct Part {
  int r, part, begin, end;
  template <typename T>
  __device__ __forceinline__ Part(const SampleArgs& a, const Row<T>& row) {
    r = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const int per = (row.pieces + a.parts - 1) / a.parts;
    begin = min(part * per, row.pieces), end = min(begin + per, row.pieces);
  }
};

// 128 rows of 131001 in 16 bits that ask for all kinds of limits: 87 us in seven launches, sample_first 9, sample_bins 23 (21
// with four parts to a workgroup of four times the threads, a call 85), sample_cut 8, sample_gather 12, sample_order 18 (lists of
// up to 2048 tokens), sample_masses 11, sample_pick 7, of which about 3 are each launch's own.

// The first token of each part; the row's bins and its lists are emptied.
template <typename T>
__global__ __launch_bounds__(kPass) void sample_first(SampleArgs a) {
  __shared__ uint64_t lds[kWavesOf];
  Row<T> row(a, blockIdx.x / a.parts);
  const Part p(a, row);
  SampleSpace& s = a.space[p.r];
  for (int i = p.part * kPass + threadIdx.x; i < kBins; i += a.parts * kPass) s.count[i] = 0, s.mass[i] = 0;
  if (p.part == 0 && threadIdx.x == 0) s.listed = s.listed_p = 0;
  const uint64_t first = first_of<kPassWaves>(lds, row, p.begin, p.end);
  if (threadIdx.x == 0) s.firsts[p.part] = first;
}

// The parts' bins, added to the row's.  And, for the kernels after, what the row asks for and its first token.
template <typename T>
__global__ __launch_bounds__(kPass) void sample_bins(SampleArgs a) {
  __shared__ Bins b;
  Row<T> row(a, blockIdx.x / a.parts);
  const Part p(a, row);
  SampleSpace& s = a.space[p.r];
  const int lane = threadIdx.x % 64;
  const uint64_t mine = lane < a.parts ? s.firsts[lane] : ~0ull;
  const Limits limits = limits_of(a, p.r);
  const uint64_t first = wave_least(mine);
  const Weights w = weights_of(first, limits, row);
  if (p.part == 0 && threadIdx.x == 0) s.limits = limits, s.first = first, s.weights = w;
  if (settled(first, limits) || !by_bins(limits)) return;
  fill_bins<kPassWaves>(b, row, w, p.begin, p.end, by_masses(limits));
  for (int i = threadIdx.x; i < kBins; i += kPass) {
    if (b.count[i]) atomicAdd(&s.count[i], b.count[i]);
    if (b.mass[i]) atomicAdd(reinterpret_cast<unsigned long long*>(&s.mass[i]), (unsigned long long)b.mass[i]);
  }
}

// What the bins tell.
__global__ __launch_bounds__(kPass) void sample_cut(SampleArgs a) {
  __shared__ Bins b;
  __shared__ Groups g;
  __shared__ Cut cut;
  SampleSpace& s = a.space[blockIdx.x];
  const int wave = threadIdx.x / 64;
  const Limits limits = s.limits;
  const Weights w = s.weights;
  if (settled(s.first, limits) || !by_bins(limits)) return;
  for (int i = threadIdx.x; i < kBins; i += kPass) b.count[i] = s.count[i], b.mass[i] = s.mass[i];
  __syncthreads();
  sum_groups<kPassWaves>(b, g);
  if (wave == 0) cut = cut_of(b, g, limits);
  __syncthreads();
  const float at = range_of(cut, w, wave);
  if (threadIdx.x % 64 == 0) s.ranges.at[wave] = at;
  if (threadIdx.x == 0) s.cut = cut;
}
static_assert(kPassWaves == 4, "a wave for each end of a range");

// n tokens to a list in memory that other workgroups add to as well.
__device__ __forceinline__ void add_list(const uint64_t* from, int n, uint64_t* list, int32_t* listed, int32_t& place) {
  if (n == 0) return;
  if (threadIdx.x == 0) place = atomicAdd(listed, n);
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPass)
    if (place + i < kList) list[place + i] = from[i];
  __syncthreads();
}

// The tokens that are put in order to the row's lists.
template <typename T>
__global__ __launch_bounds__(kPass) void sample_gather(SampleArgs a) {
  __shared__ Lists l;
  __shared__ int32_t place;
  Row<T> row(a, blockIdx.x / a.parts);
  const Part p(a, row);
  SampleSpace& s = a.space[p.r];
  const uint64_t first = s.first;
  const CutKind kind = s.cut.kind;
  const Ranges ranges = s.ranges;
  if (settled(first, s.limits) || !by_bins(s.limits) || (kind != kShort && kind != kEdges)) return;
  row.infinite = logit_of(first) == INFINITY;
  gather<kPassWaves>(l, row, p.begin, p.end, ranges);
  add_list(l.list, l.listed, s.list, &s.listed, place);
  add_list(l.list_p, l.listed_p, s.list_p, &s.listed_p, place);
}

// The tokens of rows whose lists hold what is left; of the others what that is.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_order(SampleArgs a) {
  __shared__ SampleLds l;
  const int r = blockIdx.x;
  SampleSpace& s = a.space[r];
  const uint64_t first = s.first;
  const Limits limits = s.limits;
  const Weights w = s.weights;
  Cut cut = s.cut;
  if (settled(first, limits)) return store_first(a, r, first);
  if (!by_bins(limits)) cut.kind = kWhole;
  const auto load = [&](int which) {
    const uint64_t* list = which ? s.list_p : s.list;
    for (int i = threadIdx.x; i < (int)(which ? cut.tokens_p : cut.tokens); i += kThreads) l.list[i] = list[i];
    __syncthreads();
  };
  if (cut.kind == kShort) {
    load(0);
    return pick_from_list(a, r, l, w, limits, cut, s.ranges.at[3]);
  }
  uint64_t last = ~0ull;
  if (cut.kind == kEdges) last = last_of_edges(l, w, limits, cut, load);
  if (cut.kind == kOther) {
    Row<T> row(a, r);
    row.infinite = logit_of(first) == INFINITY;
    last = last_of(l, row, w, limits);
  }
  if (threadIdx.x >= 64) return;
  const Kept k = kept_of(w, last, limits);
  if (threadIdx.x == 0) s.kept = k;
}

// The parts' masses of what is left, where no list holds it.
template <typename T>
__global__ __launch_bounds__(kPass) void sample_masses(SampleArgs a) {
  __shared__ uint64_t lds[kWavesOf];
  Row<T> row(a, blockIdx.x / a.parts);
  const Part p(a, row);
  SampleSpace& s = a.space[p.r];
  const uint64_t first = s.first;
  const Weights w = s.weights;
  const Kept kept = s.kept;
  if (settled(first, s.limits) || (by_bins(s.limits) && s.cut.kind == kShort)) return;
  row.infinite = logit_of(first) == INFINITY;
  uint64_t m = 0;
  row.each(p.begin + threadIdx.x, p.end, kPass, [&](int i, float x) { m += kept_weight(w, kept, i, x); });
  m = block_sum<kPassWaves>(lds, m);
  if (threadIdx.x == 0) s.masses[p.part] = m;
}

// Their tokens.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_pick(SampleArgs a) {
  __shared__ uint64_t lds[kWavesOf];
  const int r = blockIdx.x, lane = threadIdx.x % 64;
  Row<T> row(a, r);
  const SampleSpace& s = a.space[r];
  const uint64_t first = s.first, mine = lane < a.parts ? s.masses[lane] : 0;  // (where not written, not used)
  const Limits limits = s.limits;
  const Weights w = s.weights;
  const Kept kept = s.kept;
  if (settled(first, limits) || (by_bins(limits) && s.cut.kind == kShort)) return;
  row.infinite = logit_of(first) == INFINITY;
  const uint64_t run = wave_running_sum(mine), total = of_lane(run, 63);
  const int p = __builtin_ctzll(__ballot(target_of(limits.u, total) < run));
  const int per = (row.pieces + a.parts - 1) / a.parts, begin = min(p * per, row.pieces);
  pick_by_index(a, r, lds, row, w, limits, kept, begin, min(begin + per, row.pieces), of_lane(run - mine, p), total);
}

template <typename T>
hipError_t start(const SampleArgs& a, int32_t rows, hipStream_t stream) {
  if (a.parts == 0) {
    sample_kernel<T><<<(unsigned)rows, kThreads, 0, stream>>>(a);
    return hipGetLastError();
  }
  const unsigned parts = (unsigned)(rows * a.parts);
  sample_first<T><<<parts, kPass, 0, stream>>>(a);
  sample_bins<T><<<parts, kPass, 0, stream>>>(a);
  sample_cut<<<(unsigned)rows, kPass, 0, stream>>>(a);
  sample_gather<T><<<parts, kPass, 0, stream>>>(a);
  sample_order<T><<<(unsigned)rows, kThreads, 0, stream>>>(a);
  sample_masses<T><<<parts, kPass, 0, stream>>>(a);
  sample_pick<T><<<(unsigned)rows, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const void* logits, int64_t row_stride, int dtype, int32_t rows, int32_t vocab, const float* u,
                         const sdnn_sampling& settings, int32_t* token, float* logprob, float* workspace, hipStream_t stream) {
  if (!launchable(rows, kThreads)) return hipErrorInvalidConfiguration;
  SampleArgs a = {};
  a.logits = logits, a.row_stride = row_stride, a.vocab = vocab, a.u = u, a.settings = settings;
  a.token = token, a.logprob = logprob;
  a.parts = sample_parts(rows, vocab), a.space = reinterpret_cast<SampleSpace*>(workspace);
  return dtype == SDNN_F32   ? start<float>(a, rows, stream)
         : dtype == SDNN_F16 ? start<_Float16>(a, rows, stream)
                             : start<__bf16>(a, rows, stream);
}

}  // namespace sdnn
